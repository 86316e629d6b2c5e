/*
 * rgd.h -- C ABI of the refusal-gated decode step on GB300 (sm_103a).
 *
 * Refusal-gated decoding (arxiv 2607.20791) runs, for every prompt, one greedy
 * "probe" row and N high-temperature sample rows.  All rows of a prompt attend
 * to the prompt's KV cache, which is computed once and reused (Sec. 3), plus
 * their own generated-suffix KV.  The greedy probe is checked token by token
 * against a set P of refusal prefixes (the compatibility predicate C, Sec. 3;
 * matched on token prefixes, a detection needing at least two tokens, App. D);
 * the hard gate of Alg. 1 then either keeps the greedy refusal or discards the
 * probe and keeps the high-temperature samples.
 *
 * This library implements one decode step of that loop as CUDA kernels:
 *   rgd_prefix_decode_attn  shared-prefix split-KV decode attention,
 *   rgd_sample_head         greedy argmax / temperature + min-p + Philox sample,
 *   rgd_probe_gate          per-token refusal-prefix gate on a token trie,
 *   rgd_sample_head_gated   the two above in one kernel,
 *   rgd_decode_step         attention, then the gated head: one whole step,
 *   rgd_soft_gate           its soft variant (the appendix ablation, Alg. 2),
 *   rgd_residual_precheck   the residual-stream classifier that lets a prompt
 *                           skip the probe (App. A), once per prompt.
 * A step whose rows decode several drafted tokens at once has beside them:
 *   rgd_w4_matvec           products of a few rows with 4-bit weights, as an
 *                           output matrix or a draft model keeps them,
 *   rgd_verify_draft        drafted tokens against the target's probabilities,
 *   rgd_cache_*             the pages of the KV cache: reserved and written for
 *                           new tokens, forked, trimmed, copied and compacted.
 *
 * Conventions for every entry point
 *   - Tensor pointers are DEVICE pointers owned by the caller unless a comment
 *     says "host".  The library never frees them.  bf16 values are passed as
 *     their 16-bit patterns (rgd_bf16).  All tensors are dense, row-major, with
 *     the shapes given, and 16-byte aligned base addresses.
 *   - Calls are asynchronous on `stream` (a cudaStream_t; NULL = the legacy
 *     default stream) and use the device that is current on the calling thread.
 *     Their kernels are launched as programmatic dependents of the previous
 *     kernel on the stream: they are scheduled while it finishes and wait for it
 *     before they read or write anything (the head inside rgd_decode_step reads
 *     its inputs, complete by then, while the step's attention runs).
 *   - The return value is a host status: RGD_OK, or an RGD_ERR_* code when the
 *     arguments are rejected (nothing is launched) or a launch fails;
 *     rgd_last_error_string() then describes the error (per thread).
 *   - Errors found on the device (an out-of-range page id, an invalid
 *     temperature, a wait that timed out) never trap: the kernel ORs an
 *     RGD_DEV_* bit into *dev_status (a caller-owned device int32, may be NULL)
 *     and skips the offending work.  Read it after synchronising.
 */
#ifndef RGD_H
#define RGD_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* host status codes */
#define RGD_OK 0
#define RGD_ERR_INVALID_ARG 1
#define RGD_ERR_CUDA 2
#define RGD_ERR_UNSUPPORTED 3

/* device status bits (ORed into *dev_status) */
#define RGD_DEV_BAD_PAGE 1      /* block-table entry outside [0, num_pages): read as zeros */
#define RGD_DEV_BAD_TOKEN 2     /* negative probe token that is not the stop token: skipped */
#define RGD_DEV_WAIT_TIMEOUT 4  /* a bounded wait on a copy gave up; outputs of that block are missing */
#define RGD_DEV_BAD_PARAM 8     /* temperature < 0 or not finite, min_p outside [0, 1], or non-finite logits max */
#define RGD_DEV_NO_PAGE 16      /* the pool has fewer free pages than rgd_cache_reserve was asked for */

/* logits element types */
#define RGD_F32 0
#define RGD_BF16 1

/* gate decisions (Sec. 3 / Alg. 1 outcomes) */
#define RGD_PENDING 0
#define RGD_REFUSAL 1      /* the greedy probe stays refusal-compatible: return the greedy refusal */
#define RGD_NON_REFUSAL 2  /* the probe became incompatible: discard it, keep the samples */

typedef uint16_t rgd_bf16;
typedef void* rgd_stream_t;

/* Description of the last error on this thread ("" if none). */
const char* rgd_last_error_string(void);
/* Library version string. */
const char* rgd_version(void);

/* ------------------------------------------------------------------------ */
/* Shared-prefix decode attention (Sec. 3: prompt KV reused by the probe and   */
/* the sampling stage; here read once per prompt group and kv head)            */
/* ------------------------------------------------------------------------ */

/* Shape of one attention call.  R = num_groups * rows_per_group rows; row
 * g*rows_per_group is the probe of group g, the next rows_per_group-1 rows are
 * its sample rows.  Query head j uses kv head j / (num_q_heads/num_kv_heads). */
typedef struct {
  int32_t num_groups;        /* G >= 1                                          */
  int32_t rows_per_group;    /* 1 + N >= 1                                      */
  int32_t num_q_heads;       /* Hq, a multiple of num_kv_heads                  */
  int32_t num_kv_heads;      /* Hkv >= 1                                        */
  int32_t head_dim;          /* D: 64 or 128                                    */
  int32_t page_size;         /* tokens per KV page: 16                          */
  int32_t num_pages;         /* pages in each of the K and V pools              */
  int32_t max_prompt_pages;  /* columns of prompt_block_table (>= 1)            */
  int32_t max_suffix_pages;  /* columns of suffix_block_table (>= 1)            */
  int32_t num_ctas;          /* persistent blocks (<= 65535); 0 = one per SM     */
  int32_t reserved;          /* must be 0                                       */
} rgd_attn_shape;

/* Sets how long the attention kernel's blocks wait for one another (a split
 * job's merger for its other pieces) and for their own copies and MMAs before
 * giving up with RGD_DEV_WAIT_TIMEOUT, for every later call on any thread; 0
 * restores the default of 2 s.  The kernel never traps: a wait that gives up
 * stops that block's work, drains its copies in flight and returns.  A short
 * limit serves tests of that path; in service a limit must stay far above a
 * call's run time. */
int rgd_set_wait_limit_ns(uint64_t limit_ns);

/* Bytes of device workspace rgd_prefix_decode_attn needs for this shape (it
 * depends on the current device's SM count when num_ctas is 0). */
size_t rgd_prefix_decode_attn_workspace_size(const rgd_attn_shape* shape);

/* Decode attention of every active row over [prompt KV of its group | its own
 * suffix KV] (the concatenation; no causal mask; no rotary embedding):
 *   out[r, j, :] = softmax(softmax_scale * K q[r, j]) V,
 *   lse[r, j]    = ln sum exp(softmax_scale * K q[r, j])   (natural log).
 * Every prompt KV page of a group is read once and attended by all
 * rows_per_group * Hq/Hkv queries of that group and kv head; a row's suffix
 * pages are attended by that row's queries.  The pages of all (group, kv head)
 * jobs are divided over num_ctas persistent blocks (evenly, a job's end counting
 * as some pages where groups are few); a job split across blocks is merged from
 * its partial results by log-sum-exp.
 *
 *   q                  bf16 [R, Hq, D]
 *   k_pages, v_pages   bf16 [num_pages, Hkv, page_size, D].  Slots past a length in
 *                      a listed page have no weight, but their V must be finite: a
 *                      NaN or infinity there (or in another row's suffix) makes
 *                      outputs of the group and kv head NaN (0 x NaN in the MMA)
 *   prompt_block_table int32 [G, max_prompt_pages]: page ids of prompt tokens
 *                      (token t in page table[t / page_size], slot t % page_size)
 *   prompt_len         int32 [G], 0 <= prompt_len <= max_prompt_pages*page_size
 *   suffix_block_table int32 [R, max_suffix_pages]
 *   suffix_len         int32 [R], 0 <= suffix_len <= max_suffix_pages*page_size
 *   row_active         uint8 [R] or NULL (all active); inactive rows read no KV
 *                      and their out/lse are left untouched
 *   softmax_scale      > 0 (1/sqrt(D) for standard attention)
 *   out                bf16 [R, Hq, D]; lse float [R, Hq] or NULL
 *   workspace          device memory of rgd_prefix_decode_attn_workspace_size()
 *                      bytes, 256-byte aligned, zero-filled before its first
 *                      use.  It starts with an area of max(J, 8192) int32
 *                      counters, J = num_groups * num_kv_heads (one per (group,
 *                      kv head) job), which every call leaves at zero again
 *                      unless it reports RGD_DEV_WAIT_TIMEOUT (then zero-fill it
 *                      before reuse); the rest is scratch that a call writes
 *                      before reading.  So one workspace, sized for the largest
 *                      shape, may serve calls of any shapes with J <= 8192;
 *                      a call with J > 8192 moves the scratch, so zero-fill the
 *                      workspace whenever the shape changes across it.  Calls
 *                      that share a workspace must not overlap in time.
 * One kernel runs on `stream`, launched as a programmatic dependent of the
 * previous kernel on the stream (it is scheduled while that kernel finishes and
 * waits for it before reading any input).  A job split across blocks is merged by the
 * block holding its first page, which waits (bounded) for the job's other
 * pieces; those are the first pieces of later blocks and wait on no other
 * block, so the wait ends as long as blocks start in index order (num_ctas
 * above the number of blocks the device holds at once relies on that).
 * A group with prompt_len 0 and a row with suffix_len 0 are valid; a row with
 * neither gets out = 0, lse = -inf.  Page ids outside [0, num_pages) read as
 * zeros and set RGD_DEV_BAD_PAGE.  Lengths beyond the table are rejected on the
 * device (RGD_DEV_BAD_PAGE) because the host does not read device lengths. */
int rgd_prefix_decode_attn(const rgd_attn_shape* shape, const rgd_bf16* q,
                           const rgd_bf16* k_pages, const rgd_bf16* v_pages,
                           const int32_t* prompt_block_table, const int32_t* prompt_len,
                           const int32_t* suffix_block_table, const int32_t* suffix_len,
                           const uint8_t* row_active, float softmax_scale, rgd_bf16* out,
                           float* lse, void* workspace, size_t workspace_bytes,
                           int32_t* dev_status, rgd_stream_t stream);

/* Allocation-free form of rgd_prefix_decode_attn (the paper has no counterpart;
 * this is a deployment convenience).  Same arguments and results, minus the
 * workspace: the split partials live in one fixed 8 MiB device
 * array inside the library (one per device, held by every process that loads the
 * library until it exits).  It is for callers that cannot call cudaMalloc: for
 * example a serving engine whose KV-cache manager has already reserved the free
 * device memory (a new allocation would fail or break its memory accounting),
 * or a latency-critical decode loop where cudaMalloc / cudaFree would
 * synchronise the device.  The caller still passes every input and output.
 *   - Shapes whose workspace (rgd_prefix_decode_attn_workspace_size) exceeds
 *     8 MiB, or with more than 8192 (group, kv head) jobs, are rejected with
 *     RGD_ERR_UNSUPPORTED.
 *   - The first call on a device looks up the array's device address (once per
 *     device, with that device current); make that first call before any stream
 *     capture.
 *   - Nothing is allocated or cleared: the array starts zeroed when the library
 *     is loaded; its first 32 KiB hold the job counters of every call, whatever
 *     the shape, and every call leaves the counters of its jobs at zero, unless
 *     it reports RGD_DEV_WAIT_TIMEOUT (after which this entry point must not be
 *     used again in the process).  Every call shares the one array, so calls
 *     that overlap on the GPU (other streams, other threads) race: serialise
 *     them. */
int rgd_prefix_decode_attn_noalloc(const rgd_attn_shape* shape, const rgd_bf16* q,
                                   const rgd_bf16* k_pages, const rgd_bf16* v_pages,
                                   const int32_t* prompt_block_table, const int32_t* prompt_len,
                                   const int32_t* suffix_block_table, const int32_t* suffix_len,
                                   const uint8_t* row_active, float softmax_scale, rgd_bf16* out,
                                   float* lse, int32_t* dev_status, rgd_stream_t stream);

/* ------------------------------------------------------------------------ */
/* Sample head: G_M's greedy token and S_{T,theta}'s truncated sample          */
/* (Sec. 3, Alg. 1; truncation = min-p, Sec. 1)                                */
/* ------------------------------------------------------------------------ */

/* For every active row r of logits [rows, vocab] (RGD_F32 or RGD_BF16):
 *   greedy rows (is_probe[r] != 0 or temperature[r] == 0):
 *     token = argmax, lowest index on ties; kept_count = 1.
 *   sample rows: l_max = max logit; cutoff c = fl32(l_max + fl32(T ln p_min))
 *     (T ln p_min evaluated in double, rounded once to float; p_min = 0 keeps
 *     everything); kept set K = {i : l_i >= c} (this is {p_i >= p_min p_max}
 *     for p = softmax(l/T)); w_i = exp((l_i - l_max)/T); u = Philox4x32-10
 *     uniform with key = seed[r] (low word first) and counter = (step low,
 *     step high, 0, 0): u = (word0 >> 8) * 2^-24; token = the smallest i in K
 *     with sum_{j in K, j <= i} w_j > u * sum_K w.
 *   token_out int32 [rows] (-1 for inactive rows and rejected parameters);
 *   kept_count int32 [rows] or NULL: |K| (0 for inactive and rejected rows);
 *   kept_mask uint8 [rows, vocab] or NULL: 1 where i in K (sample rows only;
 *     rows that are greedy, inactive or rejected are not written).
 * is_probe may be NULL (no probe rows); row_active may be NULL (all active).
 * vocab must satisfy vocab * element size <= 2 MiB.  A wait that gives up sets
 * RGD_DEV_WAIT_TIMEOUT in dev_status; outputs of rows then are missing. */
int rgd_sample_head(int32_t rows, int32_t vocab, int32_t dtype, const void* logits,
                    const uint8_t* is_probe, const float* temperature, const float* min_p,
                    const uint64_t* seed, uint64_t step, const uint8_t* row_active,
                    int32_t* token_out, int32_t* kept_count, uint8_t* kept_mask,
                    int32_t* dev_status, rgd_stream_t stream);

/* ------------------------------------------------------------------------ */
/* Refusal-prefix gate (compatibility predicate C, Sec. 3; hard gate, Alg. 1)  */
/* ------------------------------------------------------------------------ */

/* Token trie of the refusal-prefix set P, built on the host and uploaded to the
 * current device.  Library-owned; release with rgd_trie_destroy. */
typedef struct rgd_trie rgd_trie;

/* tokens (host) int32 [offsets[n_seq]]: the sequences back to back, each token
 * >= 0; offsets (host) int64 [n_seq + 1], offsets[0] = 0, strictly increasing
 * (every sequence non-empty).  Duplicates and sequences that are prefixes of
 * others are allowed.  min_confirm >= 1 is the minimum length of a refusal
 * prefix whose full match confirms a refusal (2 in the paper, App. D).
 * n_seq = 0 gives the empty set (every probe is incompatible). */
int rgd_trie_create(const int32_t* tokens, const int64_t* offsets, int32_t n_seq,
                    int32_t min_confirm, rgd_trie** out);
int rgd_trie_destroy(rgd_trie* trie);
/* Node and edge counts of a trie (root included). */
int rgd_trie_info(const rgd_trie* trie, int32_t* num_nodes, int32_t* num_edges);

/* Per-group gate state, in device memory owned by the caller. */
typedef struct {
  int32_t node;           /* trie node of the probe q (root = 0)                    */
  int32_t length;         /* |q|: probe tokens appended (stop token excluded)        */
  int32_t steps;          /* probe tokens consumed (stop token included)             */
  int32_t decisive_step;  /* 0-based index of the token that decided; -1 if pending  */
  uint8_t decision;       /* RGD_PENDING / RGD_REFUSAL / RGD_NON_REFUSAL             */
  uint8_t confirmed;      /* some refusal prefix of length >= min_confirm prefixes q */
  uint8_t done;           /* the probe has ended (stop token, length cap, discarded) */
  uint8_t reserved;       /* 0 between calls (rgd_sample_head_gated counts rows here) */
} rgd_gate_state;

/* Reset `groups` states to the empty probe (node 0, pending). */
int rgd_gate_state_init(rgd_gate_state* state, int32_t groups, rgd_stream_t stream);

/* Feed n_tokens greedy probe tokens per group to the hard gate.  Token k of
 * group g is probe_tokens[g * token_stride + k] (token_stride >= n_tokens; use
 * the sample head's token_out with token_stride = rows_per_group and n_tokens =
 * 1 to gate the probe row of every group).  For each token of a group whose
 * probe has not ended:
 *   - the stop token (eos_token >= 0) ends the probe: REFUSAL if q is
 *     compatible (q non-empty, or P non-empty), else NON_REFUSAL;
 *   - otherwise q <- q || y; if q is not compatible: NON_REFUSAL, the probe
 *     ends; if a refusal prefix of length >= min_confirm is now a prefix of q:
 *     confirmed, REFUSAL (the probe continues to produce its text); if |q|
 *     reaches max_len: the probe ends, REFUSAL if still pending.
 * Then row_active [groups*rows_per_group] (updated in place, may be NULL):
 * the probe row is cleared once the probe has ended; the sample rows of a group
 * are cleared once its decision is REFUSAL.  Negative tokens other than the
 * stop token are skipped and set RGD_DEV_BAD_TOKEN. */
int rgd_probe_gate(const rgd_trie* trie, int32_t groups, int32_t rows_per_group,
                   const int32_t* probe_tokens, int32_t n_tokens, int64_t token_stride,
                   int32_t eos_token, int32_t max_len, rgd_gate_state* state,
                   uint8_t* row_active, int32_t* dev_status, rgd_stream_t stream);

/* The sample head and the hard gate of one decode step in one kernel (Alg. 1:
 * the greedy step G_M and the sample rows' S_{T,theta} draw, then the probe
 * token through the compatibility gate).  Same results as rgd_sample_head
 * (without kept_mask) followed by
 *   rgd_probe_gate(trie, rows / rows_per_group, rows_per_group, token_out, 1,
 *                  rows_per_group, eos_token, max_len, state, row_active, ...):
 * every active row draws its token first, and only then are the rows of a
 * group masked by its gate outcome (the gate of group g runs once all
 * rows_per_group rows of the group have their tokens).  Rows g*rows_per_group
 * .. +rows_per_group-1 form group g; row g*rows_per_group is its probe (pass
 * is_probe with those rows set, or temperature 0 there, for a greedy probe).
 *   row_active   uint8 [rows] or NULL: read as by rgd_sample_head, then
 *                updated in place by the gate
 *   state        device rgd_gate_state [rows / rows_per_group], 4-byte
 *                aligned; its `reserved` byte must be 0 between calls (the
 *                kernel counts a group's finished rows there during the call
 *                and leaves it at 0; rgd_gate_state_init sets it)
 *   rows_per_group in [1, 255], dividing rows; max_len >= 1; trie non-NULL.
 * One kernel on `stream`, launched as a programmatic dependent of the previous
 * kernel on the stream (it is scheduled while that kernel finishes and waits
 * for it before reading any input). */
int rgd_sample_head_gated(int32_t rows, int32_t vocab, int32_t dtype, const void* logits,
                          const uint8_t* is_probe, const float* temperature, const float* min_p,
                          const uint64_t* seed, uint64_t step, uint8_t* row_active, int32_t* token_out,
                          int32_t* kept_count, const rgd_trie* trie, int32_t rows_per_group,
                          int32_t eos_token, int32_t max_len, rgd_gate_state* state, int32_t* dev_status,
                          rgd_stream_t stream);

/* One whole decode step of the gated loop: rgd_prefix_decode_attn over the
 * step's rows, then rgd_sample_head_gated over the step's logits (two kernels
 * on `stream`; the head's blocks are scheduled while the attention finishes).
 * The logits are the caller's: this call has no part of the model between the
 * attention output and the next-token logits (projections, MLP, LM head; for
 * 4-bit weights there is rgd_w4_matvec); the head reads its inputs while the
 * attention finishes (the attention writes none of them).
 * Arguments are those of the two calls, with rows = num_groups *
 * rows_per_group and one row_active shared by both (the attention reads it,
 * the gate updates it); out and lse receive the attention output.  The first
 * error stops the step (nothing after it is launched). */
int rgd_decode_step(const rgd_attn_shape* shape, const rgd_bf16* q, const rgd_bf16* k_pages,
                    const rgd_bf16* v_pages, const int32_t* prompt_block_table, const int32_t* prompt_len,
                    const int32_t* suffix_block_table, const int32_t* suffix_len, float softmax_scale,
                    rgd_bf16* out, float* lse, void* workspace, size_t workspace_bytes, int32_t vocab,
                    int32_t dtype, const void* logits, const uint8_t* is_probe, const float* temperature,
                    const float* min_p, const uint64_t* seed, uint64_t step, uint8_t* row_active,
                    int32_t* token_out, int32_t* kept_count, const rgd_trie* trie, int32_t eos_token,
                    int32_t max_len, rgd_gate_state* state, int32_t* dev_status, rgd_stream_t stream);

/* Soft compatibility gate (the appendix ablation's Alg. 2): one probe step per
 * group from the probe row's logits.  With y the greedy token (argmax, lowest
 * index on ties): after the first c probe steps, or when y is the stop token,
 * or when q || y stays refusal-compatible, this is the hard gate's step with
 * y.  Otherwise the top_k tokens of softmax(logits) (larger logit first, lower
 * index first on ties) that keep q compatible -- the trie children of q's node,
 * and the stop token, which does not change q -- form A_ref with mass m (their
 * softmax probabilities summed); when A_ref is non-empty and m >= rho the most
 * probable of them, a*, is appended instead of y (the caller feeds it back as
 * the probe's token), else the probe is discarded: NON_REFUSAL at this step.
 *   probe_logits   device [groups rows of row_stride elements]: group g's probe
 *                  logits at probe_logits + g * row_stride (RGD_F32 / RGD_BF16);
 *                  use the step's logits with row_stride = rows_per_group * vocab
 *   token_out      device int32 [groups]: the token appended this step (y or
 *                  a*), -1 when none (probe discarded or already ended)
 *   mass_out       device float [groups] or NULL: m when the soft branch ran,
 *                  else -1
 * State and row_active as for rgd_probe_gate.  m is accumulated in fp32 with
 * e^x taken as 2^(x log2 e) by the SFU (the decision can differ from exact
 * arithmetic only when m is within ~1e-5 relative of rho).  dev_status (may
 * be NULL) gets RGD_DEV_WAIT_TIMEOUT when a bounded wait on a copy of the
 * logits gave up; that step's outputs are then not valid.
 * RGD_ERR_UNSUPPORTED when a trie node has more than 2047 children.  One
 * kernel on `stream`: a cluster of 6, 4 or 2 blocks per group, each block reading
 * an equal share of the probe row. */
int rgd_soft_gate(const rgd_trie* trie, int32_t groups, int32_t rows_per_group, int32_t vocab, int32_t dtype,
                  const void* probe_logits, int64_t row_stride, int32_t top_k, float rho, int32_t c,
                  int32_t eos_token, int32_t max_len, rgd_gate_state* state, uint8_t* row_active,
                  int32_t* token_out, float* mass_out, int32_t* dev_status, rgd_stream_t stream);

/* ------------------------------------------------------------------------ */
/* Residual-stream precheck (App. A)                                          */
/* ------------------------------------------------------------------------ */

/* Logistic readout of each group's last-prompt-token activation, run once
 * before the probe's first token:
 *   z_g = sum_i w[i] * h[g, i] + bias,  p_g = 1 / (1 + exp(-z_g)),
 * and a group with p_g <= theta skips the greedy probe (App. A: the prompt
 * decodes directly at high temperature).  For such a group whose state is
 * still the fresh empty probe (pending, no token consumed), the state becomes
 * decision RGD_NON_REFUSAL, done = 1, decisive_step -1 (decided before any
 * probe token), and its probe row (row g * rows_per_group) is cleared in
 * row_active; the sample rows stay on.  Other groups are left unchanged.
 *   h           device, [groups, d], dtype RGD_F32 or RGD_BF16, row-major
 *   w           device float [d]; bias, theta in [0, 1] by value
 *   prob_out    device float [groups] (p_g) or NULL
 *   state       device rgd_gate_state [groups]; row_active device
 *               uint8 [groups * rows_per_group] or NULL
 * z is accumulated in fp32 (the decision can differ from exact arithmetic
 * only when z is within the fp32 rounding of its sum from the threshold's
 * logit).  One kernel on `stream`, one block per group. */
int rgd_residual_precheck(int32_t groups, int32_t d, int32_t dtype, const void* h, const float* w, float bias,
                          float theta, int32_t rows_per_group, float* prob_out, rgd_gate_state* state,
                          uint8_t* row_active, int32_t* dev_status, rgd_stream_t stream);

/* ------------------------------------------------------------------------ */
/* Verification of drafted tokens                                             */
/* ------------------------------------------------------------------------ */

/* Bytes of device workspace rgd_verify_draft needs (0 on a negative argument). */
size_t rgd_verify_draft_workspace_size(int32_t rows, int32_t max_draft);

/* Row r has n = n_draft[r] drafted tokens d_0 .. d_{n-1} (a draft model's, a
 * phrase list's, the refusal trie's own continuation) and the target's logits at
 * the n + 1 positions they lead to: position k follows the row's prefix and d_0 ..
 * d_{k-1}.  Sample rows (as in rgd_sample_head): with p_k and q_k the target's and
 * the draft's softmax(l / T) over their min-p kept sets {l >= c}, c = fl32(l_max +
 * fl32(T ln p_min)), in order of k
 *   d_k is accepted if accept_u[r, k] q_k(d_k) < p_k(d_k);
 *   at the first that is not, the row's last token is drawn from max(0, p_k - q_k)
 *   (from p_k should that be 0 everywhere); if all are accepted it is drawn from p_n:
 *   token = the smallest i whose cumulative weight exceeds draw_u[r] times their sum.
 * The tokens that come out are distributed as p, up to rounding (see below), if d_k was
 * drawn from q_k - that is with the row's temperature and min_p - or, without draft
 * logits, was chosen in any way that does not look at the uniforms.  Greedy rows
 * (is_probe or temperature 0): d_k is accepted if it is the argmax (lowest index on
 * ties), and the last token is the argmax; draft_logits, min_p and the uniforms are
 * not read.
 *   target_logits  [rows, max_draft + 1] rows of vocab logits, target_stride elements
 *                  apart (>= vocab), dtype RGD_F32 or RGD_BF16
 *   draft_logits   [rows, max_draft] rows of vocab logits of the same dtype,
 *                  draft_stride elements apart; NULL: every draft was certain
 *                  (q_k(d_k) = 1).  Rows that all start on 16 bytes are read fastest
 *   draft_tokens   int32 [rows, max_draft]; one outside [0, vocab) is rejected, the
 *                  draw there is from p_k, and it sets RGD_DEV_BAD_TOKEN, also at a
 *                  position of finite logits that the row does not get to
 *   n_draft        int32 [rows], in [0, max_draft]; NULL: max_draft each
 *   is_probe       uint8 [rows] or NULL; temperature, min_p float [rows]
 *   accept_u       float [rows, max_draft], draw_u float [rows]: independent
 *                  uniforms in [0, 1)
 *   row_active     uint8 [rows] or NULL (all active)
 *   token_out      int32 [rows, max_draft + 1]: the accepted drafts, the last token,
 *                  then -1; all -1 for inactive and rejected rows.  (rgd_probe_gate
 *                  skips the -1 of a probe row that is given to it as it is, and sets
 *                  RGD_DEV_BAD_TOKEN for them)
 *   accepted_out   int32 [rows]: accepted drafts (0 for inactive and rejected rows);
 *                  token_out[r] holds accepted_out[r] + 1 tokens
 *   accept_prob    float [rows, max_draft] or NULL: min(1, p_k(d_k) / q_k(d_k)) of
 *                  every drafted position (1 or 0 in greedy rows), whether the row
 *                  gets there or not; 0 past n_draft
 *   workspace      rgd_verify_draft_workspace_size() bytes, 4-byte aligned, zero-filled
 *                  before its first use; a call leaves it all zero again, so one sized
 *                  for the largest call serves calls of any shape.  Calls that share
 *                  it must not overlap.  RGD_DEV_WAIT_TIMEOUT: a wait within the kernel
 *                  gave up after 2 s, and the row it was for is rejected; rely on no
 *                  output of the call then, and fill the workspace anew
 * A row with n_draft, temperature, min_p or draw_u out of range, or with a position it
 * gets to whose accept_u is out of range or whose largest logit is not finite, is rejected
 * and sets RGD_DEV_BAD_PARAM.  NaN logits have no weight.  Weights are 2^((l - l_max)
 * log2(e)/T) in fp32, rounded to multiples of 2^-31 and summed exactly, so the
 * outputs do not depend on how a call is cut.  (rgd_sample_head keeps 43 binary places
 * of them: of the same uniform it can draw another token where the mark lies next to an
 * edge.)  max(0, p_k - q_k) is rounded to multiples of 2^-31 as well - of probability 1,
 * not of its own largest value: where p and q are flat and nearly the same, its small
 * values lose digits or vanish.  The rest alone is then off by 0.4 % in total variation
 * at a vocab of 262144, T = 10 and draft logits off by 0.05, by 4 % with 0.005, and 5e-5
 * at T = 1 and 0.5; as such rests are drawn from as rarely, what is emitted is off by
 * 1e-5 at most in each.  RGD_ERR_UNSUPPORTED above a vocab of 2^20.  One kernel on
 * `stream`. */
int rgd_verify_draft(int32_t rows, int32_t max_draft, int32_t vocab, int32_t dtype, const void* target_logits,
                     int64_t target_stride, const void* draft_logits, int64_t draft_stride,
                     const int32_t* draft_tokens, const int32_t* n_draft, const uint8_t* is_probe,
                     const float* temperature, const float* min_p, const float* accept_u, const float* draw_u,
                     const uint8_t* row_active, int32_t* token_out, int32_t* accepted_out, float* accept_prob,
                     void* workspace, size_t workspace_bytes, int32_t* dev_status, rgd_stream_t stream);

/* ------------------------------------------------------------------------ */
/* Products with 4-bit weights                                                */
/* ------------------------------------------------------------------------ */

/* y[i, j] = sum_k x[i, k] W[j, k],  W[j, k] = (q[j, k] - z[j, k / G]) s[j, k / G],
 * for a few rows of activations (any m is right; above 16 rows the weights are read and
 * converted once more for every 16, so that many rows are better served as a dense product).
 *   x        bf16 [m, k]
 *   weights  uint8 [n, ceil(k / 2)]: q in 4 bits, the even k in the low half of its
 *            byte; the last high half of an odd k is not read as a weight
 *   scales   [n, ceil(k / G)], scale_dtype RGD_F32 or RGD_BF16, finite; G = group_size
 *            = 32, 64 or 128; the last group of a row may be short
 *   zeros    uint8 [n, ceil(k / G)], 0 to 15, or NULL (8 everywhere)
 *   y        [m] rows of n elements, y_stride elements apart (>= n; the rest of a row
 *            is left alone), out_dtype RGD_F32 or RGD_BF16
 * Products of bf16 activations with the whole numbers q - z are exact and are summed,
 * and scaled group by group, in fp32; the result is rounded once.  The order of the sums
 * is the same for every call of the same m, n and k, but goes by all three: a row's y may
 * differ in its last bits from that of a call with fewer or more rows.  dev_status gets
 * RGD_DEV_WAIT_TIMEOUT when a bounded wait on a copy gave up; y is then not valid.  One
 * kernel on `stream`. */
int rgd_w4_matvec(int32_t m, int32_t n, int32_t k, int32_t group_size, const rgd_bf16* x, const uint8_t* weights,
                  int32_t scale_dtype, const void* scales, const uint8_t* zeros, int32_t out_dtype, void* y,
                  int64_t y_stride, int32_t* dev_status, rgd_stream_t stream);

/* ------------------------------------------------------------------------ */
/* Pages of the KV cache                                                      */
/* ------------------------------------------------------------------------ */

/* The pools of a paged cache: for every layer K and V bf16 [num_pages, Hkv,
 * page_size, D] as rgd_prefix_decode_attn reads them (layer l of k_pages starts at
 * k_pages + l * layer_stride).  Page i stands for the same tokens in every layer.
 * page_refs, device int32 [num_pages], counts the rows whose table lists a page; a page
 * is free exactly if its count is 0.  Whoever fills a table by other means sets the
 * counts too. */
typedef struct {
  int32_t num_layers;    /* >= 1, at most 4096                                      */
  int32_t num_pages;     /* pages in each pool                                      */
  int32_t num_kv_heads;  /* Hkv, at most 4096                                       */
  int32_t page_size;     /* tokens per page: 16                                     */
  int32_t head_dim;      /* D: a multiple of 8, at most 1024                        */
  int32_t reserved;      /* must be 0                                               */
  int64_t layer_stride;  /* elements from a layer's pool to the next; 0: no gap     */
} rgd_cache_shape;

/* Bytes of device workspace rgd_cache_reserve (for up to `rows` rows) and
 * rgd_cache_compact need; 16-byte aligned, its contents do not matter.  Calls that
 * share it must not overlap.  0 on an invalid shape. */
size_t rgd_cache_workspace_size(const rgd_cache_shape* shape, int32_t rows);

/* Makes room for n_new[r] tokens after the length[r] that row r has: every page that
 * tokens length .. length + n_new - 1 fall into is the row's own afterwards.  A table
 * entry < 0 there gets a free page; a page that other rows list too (count > 1) is
 * replaced by a free page, into which the row's tokens in it (length % page_size of
 * them) are copied in every layer.  (So for every row of the call that writes it, the last
 * one too: a page that all its rows write in one call is free afterwards.)  Free pages
 * are taken in order of their number, by rows in order and within a row by column.
 *   block_table  int32 [rows, max_pages], updated; length, n_new int32 [rows]
 *   row_active   uint8 [rows] or NULL (all); other rows are left alone
 *   page_refs    updated; k_pages, v_pages every layer's pools
 *   row_ok       uint8 [rows] or NULL: 1 where an active row and those before it have
 *                their room, else 0
 * Rows are served in order: where the pool runs out, a row whose pages and those of the
 * rows before it (those refused included) exceed the free pages is left as it was, also
 * one that needs none itself, and RGD_DEV_NO_PAGE is set.  A row of a negative length or n_new, or past the table, or with an entry >=
 * num_pages there, is left as it was and sets RGD_DEV_BAD_PAGE.  RGD_ERR_UNSUPPORTED for
 * rows * max_pages of 2^31 or more.  One kernel, and one for the copies unless they are
 * few. */
int rgd_cache_reserve(const rgd_cache_shape* shape, int32_t rows, int32_t max_pages, int32_t* block_table,
                      const int32_t* length, const int32_t* n_new, const uint8_t* row_active, int32_t* page_refs,
                      rgd_bf16* k_pages, rgd_bf16* v_pages, uint8_t* row_ok, void* workspace, size_t workspace_bytes,
                      int32_t* dev_status, rgd_stream_t stream);

/* Writes one layer's keys and values of new tokens into reserved pages: token i <
 * n_new[r] of row r becomes token length[r] + i of the row (the lengths stay the
 * caller's to raise).
 *   k_new, v_new  bf16, the Hkv x D values of (r, i) at r * row_stride + i *
 *                 token_stride elements (both multiples of 8): views of a fused
 *                 projection's output do
 *   n_new         int32 [rows], in [0, max_new]; of a row of more, the first max_new
 *                 are written and RGD_DEV_BAD_PAGE is set, as for one of less than 0
 *   row_active    uint8 [rows] or NULL: rows to write (rgd_cache_reserve's row_ok)
 * A token whose page is not listed is skipped and sets RGD_DEV_BAD_PAGE. */
int rgd_cache_write(const rgd_cache_shape* shape, int32_t layer, int32_t rows, int32_t max_new, const rgd_bf16* k_new,
                    const rgd_bf16* v_new, int64_t row_stride, int64_t token_stride, const int32_t* n_new,
                    int32_t max_pages, const int32_t* block_table, const int32_t* length, const uint8_t* row_active,
                    rgd_bf16* k_pages, rgd_bf16* v_pages, int32_t* dev_status, rgd_stream_t stream);

/* Gives back every page of a row that lies wholly past its length (all of them at
 * length 0): entries from ceil(length / page_size) on become -1 and their counts fall
 * by one.  After rejected drafts, with the lengths raised by what was accepted; for
 * rows that have ended, with length 0.  Rows with row_active 0 are left alone. */
int rgd_cache_trim(int32_t rows, int32_t max_pages, int32_t num_pages, int32_t* block_table, const int32_t* length,
                   const uint8_t* row_active, int32_t* page_refs, int32_t* dev_status, rgd_stream_t stream);

/* Makes row child[i] a copy of row parent[i]: the parent's length and the pages of its
 * tokens, shared (their counts rise by one; nothing is copied until one of them
 * writes, see rgd_cache_reserve).  A child's row is overwritten: trim it to length 0
 * first.  No row may be a child twice, or a child and a parent, in one call.  A pair
 * outside [0, rows) is skipped and sets RGD_DEV_BAD_PAGE. */
int rgd_cache_fork(int32_t pairs, const int32_t* parent, const int32_t* child, int32_t rows, int32_t max_pages,
                   int32_t num_pages, int32_t* block_table, int32_t* length, int32_t* page_refs, int32_t* dev_status,
                   rgd_stream_t stream);

/* Copies page src[i] onto page dst[i] for i < n, keys and values in every layer (device
 * int32 arrays; no target may be another pair's source or target).  A pair outside
 * the pool is skipped and sets RGD_DEV_BAD_PAGE. */
int rgd_cache_copy(const rgd_cache_shape* shape, int32_t n, const int32_t* src, const int32_t* dst, rgd_bf16* k_pages,
                   rgd_bf16* v_pages, int32_t* dev_status, rgd_stream_t stream);

/* Moves the pages in use to the front of the pool.  With L pages in use, the i-th of
 * them at or above L goes to the i-th free page below L, in every layer; the counts
 * move along and the entries of up to two tables (int32 [rows, max_pages]; NULL: none;
 * every table of the pool has to be given) are renumbered.  *num_live (device) = L: pages
 * from L on are free afterwards.  An entry that names a free page at or above L becomes
 * -1 and sets RGD_DEV_BAD_PAGE.  Two kernels. */
int rgd_cache_compact(const rgd_cache_shape* shape, int32_t rows_a, int32_t max_pages_a, int32_t* block_table_a,
                      int32_t rows_b, int32_t max_pages_b, int32_t* block_table_b, int32_t* page_refs,
                      rgd_bf16* k_pages, rgd_bf16* v_pages, int32_t* num_live, void* workspace,
                      size_t workspace_bytes, int32_t* dev_status, rgd_stream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* RGD_H */
