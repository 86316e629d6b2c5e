// Verification of drafted tokens.  Row r has n drafted tokens d_0 .. d_{n-1} and the
// target's logits at the n + 1 positions they lead to; the draft's logits (or nothing,
// where each draft was certain) say what the tokens were drawn from.  With p and q the
// two sides' truncated softmax of temperature T and min-p,
//   d_k is accepted if u_k q(d_k) < p(d_k); at the first k that is not, the row's last
//   token is drawn from max(0, p - q); after n acceptances it is drawn from p,
// which leaves the emitted tokens distributed as if each were drawn from p.
//
// One thread-block cluster of C CTAs handles one position (a "unit": the target's row
// and, for k < n, the draft's), every warp a contiguous share of each row:
//   1 the two maxima, a stream from HBM (a greedy row then needs the argmax only).  A
//     lane keeps the maximum of every group of its vectors;
//   2 the sums of the kept weights, and with them p(d), q(d) and the acceptance.  The rows
//     were just read and lie in L2, and only vectors whose group reaches the cutoff are
//     read again: under min-p a few, without truncation all;
//   3 where the draft is rejected, the sums of max(0, p - q), likewise.
// Each is joined over the CTA's warps in shared memory and over the cluster by one 8-byte
// push from every CTA into every CTA.  A draw then picks the CTA and the warp by prefix
// sums and that warp searches its own share.  The last unit of a row to finish joins the
// row's results.
//
// Rows held in shared memory instead were read from HBM no less, but 152 SMs hold 64 such
// pairs of rows, each for three exchanges over its cluster: a third of the copy rate with
// every CTA's memory loaded once, less with two buffers each.
//
// Sums are exact in any order, and so is every token, whatever the cluster's size: a
// weight 2^x <= 1 is rounded once to a whole number of 2^-31 and summed in 64 bits.  The
// rounding is what a sum in fp32 does to a small weight too: it loses at most 2^-32 of
// the largest weight, 3e-5 of the sum in the worst case over 131072 tokens, where each
// is below 2.4e-10 of the largest.  max(0, p - q) goes by the same multiples, of probability
// 1 (a scale of its own would take one exchange more, finer multiples a third sum).  A rest of small mass over many tokens
// loses digits so (262144 tokens, T = 10, draft logits off by 0.05: a rest of mass 2e-3 is off by
// 0.4 % in total variation; off by 0.005: 2e-4 and 4 %, a tenth of its tokens have no weight),
// but is drawn from as rarely as its mass says: what is emitted is off by 8e-6 in both.
#include <cuda_bf16.h>

#include <algorithm>
#include <cmath>

#include "common.h"
#include "log_pair.cuh"
#include "logit_rows.cuh"
#include "ptx.cuh"

namespace rgd {
namespace {

constexpr int kVerifyWarps = 8;
constexpr int kVerifyThreads = kVerifyWarps * 32;
constexpr int kVerifyCluster = 16;                           // CTAs of a unit at most
constexpr int32_t kTaken = -1, kRejectedRow = -2;            // results of a unit other than a token + 1

struct VerifyParams {
  const uint8_t* target;
  const uint8_t* draft;  // NULL: every draft was certain
  int64_t target_stride, draft_stride;  // bytes
  int32_t rows, max_draft, vocab;
  int32_t stripes;  // of 32 vectors, in a warp's share
  const int32_t* tokens;
  const int32_t* n_draft;
  const uint8_t* is_probe;
  const float* temperature;
  const float* min_p;
  const float* accept_u;
  const float* draw_u;
  const uint8_t* row_active;
  int32_t* token_out;
  int32_t* accepted_out;
  float* accept_prob;
  int32_t* count;   // workspace: finished units of each row
  int32_t* result;  // workspace: each unit's result
  int32_t* dev_status;
};

struct VerifyShared {
  // of this CTA's warps, and pushed by every CTA of the cluster into every other
  float warp_top[2][kVerifyWarps], top[2][kVerifyCluster];
  uint64_t warp_sum[3][kVerifyWarps], sum[3][kVerifyCluster];  // target's and draft's weights, max(0, p - q)
  uint64_t part_sum[kVerifyWarps];  // of the parts of the share that a draw falls into
  uint64_t arrived[3];  // barriers of the exchanges: maxima; weights (or argmax); max(0, p - q)
  int lost;             // a wait has given up
  float theta, tl, ql;  // T ln p_min, the drafted token's logits
};

// The whole warp: a row's finished unit is counted, and the last one to finish writes the row.
// Results are never 0 and start at 0, so that the last one needs no other order than each
// result's own: it reads them until all are there.  (A counter that released and acquired
// them took 1 us more.)
__device__ __noinline__ void finish_unit(const VerifyParams& p, int row, int pos, int n, int32_t result) {
  const int lane = threadIdx.x & 31;
  int32_t* res = p.result + (int64_t)row * (p.max_draft + 1);
  const int32_t* drafts = p.tokens + (int64_t)row * p.max_draft;
  const int32_t draft = lane < n ? drafts[lane] : -1;
  int last = 0;
  if (lane == 0) {
    asm volatile("st.relaxed.gpu.global.s32 [%0], %1;" ::"l"(res + pos), "r"(result) : "memory");
    int32_t old;
    asm volatile("atom.relaxed.gpu.global.add.s32 %0, [%1], 1;" : "=r"(old) : "l"(p.count + row) : "memory");
    last = old == n;
  }
  if (!__shfl_sync(0xffffffffu, last, 0)) return;
  int taken = n;
  int32_t token = kRejectedRow;
  const uint64_t t0 = globaltimer_ns();
  bool there = true;
  for (int base = 0; base <= n; base += 32) {
    int32_t v = kTaken;
    if (base + lane <= n) {
      do {
        asm volatile("ld.relaxed.gpu.global.s32 %0, [%1];" : "=r"(v) : "l"(res + base + lane) : "memory");
      } while (v == 0 && globaltimer_ns() - t0 < kWaitLimitNs);
      asm volatile("st.relaxed.gpu.global.s32 [%0], 0;" ::"l"(res + base + lane) : "memory");
    }
    there = __all_sync(0xffffffffu, v != 0) && there;
    const uint32_t stop = __ballot_sync(0xffffffffu, v != kTaken);
    if (stop && taken == n && token == kRejectedRow) {
      const int at = __ffs(stop) - 1;
      taken = base + at;
      token = __shfl_sync(0xffffffffu, v, at);
      if (token == kRejectedRow) taken = -1;
    }
  }
  const bool good = there && taken >= 0;
  for (int i = lane; i <= p.max_draft; i += 32)
    p.token_out[(int64_t)row * (p.max_draft + 1) + i] =
        !good || i > taken ? -1 : i < taken ? (i < 32 ? draft : drafts[i]) : token - 1;
  if (lane == 0) {
    p.accepted_out[row] = good ? taken : 0;
    p.count[row] = 0;
    // (a position that the row does not get to is nobody's error)
    if (!good && p.dev_status) atomicOr(p.dev_status, there ? RGD_DEV_BAD_PARAM : RGD_DEV_WAIT_TIMEOUT);
  }
}

// The whole CTA: a wait has run out, so the position has no result and no other one joins its row.
// (Which row it is is read again, so that it costs the kernel no registers.)
__device__ __noinline__ void give_up(const VerifyParams& p) {
  uint32_t unit;
  asm volatile("mov.u32 %0, %%clusterid.x;" : "=r"(unit));
  const int K = p.max_draft, row = (int)unit / (K + 1), pos = (int)unit % (K + 1);
  if (threadIdx.x >= 32) return;
  for (int i = threadIdx.x; i <= K; i += 32) p.token_out[(int64_t)row * (K + 1) + i] = -1;
  if (threadIdx.x != 0) return;
  p.accepted_out[row] = 0;
  if (pos < K && p.accept_prob) p.accept_prob[(int64_t)row * K + pos] = 0.f;
}

// An exchange over the cluster: every CTA pushes a value (or two) into every CTA, counted by
// the receiver's barrier of that exchange.  (With stores and a cluster barrier instead, which
// waits for the stores' return, 80 rows of 5 positions by 128256 bf16 took 38.2 us for 36.8.)
__device__ __forceinline__ void push(VerifyShared& sh, int exchange, uint64_t* slot, uint64_t v, uint32_t csize, uint32_t to) {
  if (csize == 1) *slot = v;
  else
    asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.b64 [%0], %1, [%2];" ::"r"(peer_addr(smem_u32(slot), to)),
                 "l"(v), "r"(peer_addr(smem_u32(&sh.arrived[exchange]), to))
                 : "memory");
}
__device__ __forceinline__ void push(VerifyShared& sh, int exchange, float* slot, float v, uint32_t csize, uint32_t to) {
  if (csize == 1) *slot = v;
  else
    asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.b32 [%0], %1, [%2];" ::"r"(peer_addr(smem_u32(slot), to)),
                 "r"(__float_as_uint(v)), "r"(peer_addr(smem_u32(&sh.arrived[exchange]), to))
                 : "memory");
}
// The whole CTA: what is pushed into it has arrived; false after 2 s, once no CTA of the cluster
// can push any more.
__device__ __forceinline__ bool exchanged(VerifyShared& sh, int exchange, uint32_t csize, int32_t* dev_status) {
  if (csize > 1 && threadIdx.x == 0) {
    const uint64_t t0 = globaltimer_ns();
    uint32_t done = 0;
    for (uint32_t i = 1; !done; ++i) {
      asm volatile(
          "{\n\t.reg .pred p;\n\t"
          "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], 0;\n\t"
          "selp.u32 %0, 1, 0, p;\n\t}"
          : "=r"(done)
          : "r"(smem_u32(&sh.arrived[exchange]))
          : "memory");
      if (!done && (i & 63u) == 0 && globaltimer_ns() - t0 > kWaitLimitNs) break;
    }
    if (!done) sh.lost = 1;
  }
  __syncthreads();
  if (csize == 1 || !sh.lost) return true;
  if (threadIdx.x == 0 && dev_status) atomicOr(dev_status, RGD_DEV_WAIT_TIMEOUT);
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");  // (a CTA that has ended counts as arrived)
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  return false;
}

template <typename T, bool kAligned>
__global__ void __launch_bounds__(kVerifyThreads, 4) verify_kernel(const VerifyParams p) {
  constexpr int E = 16 / (int)sizeof(T);
  using V = Vec<T>;
  __shared__ VerifyShared sh;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint32_t rank, csize, unit;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(csize));
  asm volatile("mov.u32 %0, %%clusterid.x;" : "=r"(unit));
  const int K = p.max_draft, row = (int)unit / (K + 1), pos = (int)unit % (K + 1);
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");  // (a dependent waits for this kernel's end)
  asm volatile("griddepcontrol.wait;" ::: "memory");
  // The row's parameters; every thread of the cluster takes the same decisions.
  const bool active = !p.row_active || p.row_active[row];
  const float temp = p.temperature[row], min_p = p.min_p[row], draw_u = p.draw_u[row];
  const bool greedy = (p.is_probe && p.is_probe[row]) || temp == 0.f;
  const int n = p.n_draft ? p.n_draft[row] : K;
  bool good = n >= 0 && n <= K;
  if (!greedy) good = good && temp > 0.f && temp < INFINITY && min_p >= 0.f && min_p <= 1.f && draw_u >= 0.f && draw_u < 1.f;
  const bool leader = rank == 0 && warp == 0, has_draft = active && good && pos < n;
  float* prob = pos < K && p.accept_prob ? p.accept_prob + (int64_t)row * K + pos : nullptr;
  if (leader && lane == 0 && prob && !has_draft) *prob = 0.f;
  if (!active || !good) {
    if (leader && pos == 0) {
      for (int i = lane; i <= K; i += 32) p.token_out[(int64_t)row * (K + 1) + i] = -1;
      if (lane == 0) {
        p.accepted_out[row] = 0;
        if (active && p.dev_status) atomicOr(p.dev_status, RGD_DEV_BAD_PARAM);
      }
    }
    return;
  }
  if (pos > n) return;
  const int32_t d = has_draft ? p.tokens[(int64_t)row * K + pos] : -1;
  const bool d_in = d >= 0 && d < p.vocab;  // (a draft outside the vocabulary is rejected, q = 0 everywhere)
  const float u = has_draft && !greedy ? p.accept_u[(int64_t)row * K + pos] : 0.f;
  const bool two = p.draft != nullptr && has_draft && !greedy;
  if (csize > 1) {
    if (threadIdx.x == 0) {
      sh.lost = 0;
#pragma unroll
      for (int i = 0; i < 3; ++i) mbar_init(&sh.arrived[i], 1);
      fence_mbar_init();
      mbar_arrive_expect_tx(&sh.arrived[0], csize * 8);
      mbar_arrive_expect_tx(&sh.arrived[1], csize * (two ? 16 : 8));
      mbar_arrive_expect_tx(&sh.arrived[2], csize * 8);
    }
    __syncwarp();
    cluster_arrive_relaxed();
  }
  const int64_t trow = ((int64_t)row * (K + 1) + pos) * p.target_stride, qrow = ((int64_t)row * K + pos) * p.draft_stride;

  // This warp's share, in the order of the elements over the cluster.
  const int64_t share = (int64_t)p.stripes * 32 * E;
  const int64_t e0 = ((int64_t)rank * kVerifyWarps + warp) * share;
  const int64_t count = min(share, p.vocab - e0);
  const Share<T, kAligned> tv(p.target + trow, e0, count);
  const Share<T, kAligned> qv(two ? p.draft + qrow : p.target + trow, e0, two ? count : 0);

  // Pass 1: the maxima (NaN never wins).
  if (warp == kVerifyWarps - 1 && lane == 0) {
    sh.theta = scaled_log(temp, greedy ? 1.f : min_p);  // (the token is still on its way)
    sh.tl = d_in && !greedy ? one_logit<T>(p.target + trow, d) : 0.f;
    sh.ql = d_in && two ? one_logit<T>(p.draft + qrow, d) : 0.f;
  }
  Kept tkept, qkept;
  {
    const float tm = find_maxima(tv, tkept, p.stripes, lane);
    const float qm = find_maxima(qv, qkept, two ? p.stripes : 0, lane);
    if (lane == 0) {
      sh.warp_top[0][warp] = tm;
      sh.warp_top[1][warp] = qm;
    }
  }
  __syncthreads();
  if (csize > 1) cluster_wait();  // every CTA of the cluster has started
  if (warp < 2) {
    const float m = warp_max(sh.warp_top[warp][lane % kVerifyWarps]);
    if (lane < (int)csize) push(sh, 0, &sh.top[warp][rank], m, csize, lane);
  }
  if (!exchanged(sh, 0, csize, p.dev_status)) return give_up(p);
  Side t, q;
  t.top = warp_max(sh.top[0][lane % csize]);
  q.top = warp_max(sh.top[1][lane % csize]);
  if (!two) q.top = 0.f;
  if (!(fabsf(t.top) < INFINITY && fabsf(q.top) < INFINITY && u >= 0.f && u < 1.f)) {
    if (leader) {
      if (lane == 0 && prob) *prob = 0.f;
      finish_unit(p, row, pos, n, kRejectedRow);
    }
    return;
  }
  if (has_draft && !d_in && leader && lane == 0 && p.dev_status) atomicOr(p.dev_status, RGD_DEV_BAD_TOKEN);

  if (greedy) {  // the lowest index of the largest logit
    uint32_t best = 0xffffffffu;
    auto look = [&](const uint4& w, int i) {
#pragma unroll
      for (int e = E - 1; e >= 0; --e)
        if (elem<T>(w, e) == t.top) best = min(best, (uint32_t)e0 + i * E + e);
    };
    Walk walk(groups_reaching(tkept, t.top), p.stripes, tv.whole, lane);
#pragma unroll 1
    for (int i = walk.next(); i >= 0; i = walk.next()) look(tv.get(i), i);
    look(tkept.rest, tv.whole);
    best = __reduce_min_sync(0xffffffffu, best);
    if (lane == 0) sh.warp_sum[0][warp] = best;
    __syncthreads();
    if (warp == 0) {
      best = __reduce_min_sync(0xffffffffu, (uint32_t)sh.warp_sum[0][lane % kVerifyWarps]);
      if (lane == 0) push(sh, 1, &sh.sum[0][rank], best, csize, 0);
    }
    if (rank != 0) return;
    if (!exchanged(sh, 1, csize, p.dev_status)) return give_up(p);
    if (leader) {
      best = __reduce_min_sync(0xffffffffu, (uint32_t)sh.sum[0][lane % csize]);
      const bool same = has_draft && (int32_t)best == d;
      if (lane == 0 && prob && has_draft) *prob = same ? 1.f : 0.f;
      finish_unit(p, row, pos, n, same ? kTaken : (int32_t)best + 1);
    }
    return;
  }

  // A sum of every warp over the cluster: by warp for the CTA's own, by CTA for all.
  auto join = [&](int which, uint64_t mine) {
    if (lane == 0) sh.warp_sum[which][warp] = mine;
  };
  auto exchange = [&](int first, int last) {
    __syncthreads();
    if (warp >= first && warp <= last) {
      const uint64_t v = warp_sum(lane < kVerifyWarps ? sh.warp_sum[warp][lane] : 0);
      if (lane < (int)csize) push(sh, first ? 2 : 1, &sh.sum[warp][rank], v, csize, lane);
    }
    return exchanged(sh, first ? 2 : 1, csize, p.dev_status);
  };
  auto over_cluster = [&](int which) { return warp_sum(lane < (int)csize ? sh.sum[which][lane] : 0); };

  // Pass 2: the sums of the weights.
  t.kexp = q.kexp = fminf(__fdiv_rn(1.4426950408889634f, temp), 3e38f);  // (finite: 0 times it is 0)
  t.cut = __fadd_rn(t.top, sh.theta);
  q.cut = __fadd_rn(q.top, sh.theta);
  join(0, sum_weights(tv, tkept, t, p.stripes, lane));
  if (two) join(1, sum_weights(qv, qkept, q, p.stripes, lane));
  if (!exchange(0, two ? 1 : 0)) return give_up(p);
  uint64_t total = over_cluster(0);
  t.inv = __fdiv_rn(1.f, __ull2float_rn(total) * 0x1p-31f);
  if (two) q.inv = __fdiv_rn(1.f, __ull2float_rn(over_cluster(1)) * 0x1p-31f);
  int which = 0;  // the sums that the draw goes by: the target's weights, or the rest
  if (has_draft) {
    const float pd = d_in ? t.prob(sh.tl) : 0.f;
    const float qp = !d_in ? 0.f : two ? q.prob(sh.ql) : 1.f;
    const bool taken = d_in && __fmul_rn(u, qp) < pd;
    if (leader && lane == 0 && prob) *prob = qp > 0.f ? fminf(__fdiv_rn(pd, qp), 1.f) : pd > 0.f ? 1.f : 0.f;
    if (taken) {
      if (leader) finish_unit(p, row, pos, n, kTaken);
      return;
    }
    // Pass 3: the sums of max(0, p - q); a certain draft takes its own token's p alone.
    if (d_in) {
      WholeSum rest;
      auto add = [&](const uint4& a, const uint4& c, int i) {
#pragma unroll
        for (int e = 0; e < V::kPairs; ++e) {
          float x, y, q0, q1;
          V::get(a, e, x, y);
          V::get(c, e, q0, q1);
          const int32_t at = (int32_t)e0 + i * E + 2 * e;
          q0 = two ? q.prob(q0) : at == d ? 1.f : 0.f;
          q1 = two ? q.prob(q1) : at + 1 == d ? 1.f : 0.f;
          rest.add(pair(fmaxf(t.prob(x) - q0, 0.f), fmaxf(t.prob(y) - q1, 0.f)));
        }
        rest.count(V::kPairs);
      };
      Walk walk(groups_reaching(tkept, t.cut), p.stripes, tv.whole, lane);  // (p is 0 elsewhere)
      uint4 a = tkept.rest, c = two ? qkept.rest : a;
      int i = tv.whole, ahead = walk.next();
#pragma unroll 1
      for (;;) {
        uint4 a1 = V::nothing(), c1 = a1;
        if (ahead >= 0) {
          a1 = tv.get(ahead);
          if (two) c1 = qv.get(ahead);
        }
        add(a, c, i);
        if (ahead < 0) break;
        i = ahead;
        ahead = walk.next();
        a = a1, c = c1;
      }
      join(2, warp_sum(rest.total()));
      if (!exchange(2, 2)) return give_up(p);
      const uint64_t rz = over_cluster(2);
      if (rz > 0) {  // (p and q may be equal but for rounding: then p itself)
        which = 2;
        total = rz;
      }
    }
  }

  // The draw: the CTA, then the share, that holds the mark; every warp of the CTA takes a part
  // of that share, and the one whose part holds the mark finds the element.
  const uint64_t mark = (uint64_t)((double)draw_u * (double)total);
  uint64_t before = warp_sum(lane < (int)rank ? sh.sum[which][lane] : 0);
  if (!(before <= mark && mark < before + sh.sum[which][rank])) return;
  int owner = 0;
  for (; owner + 1 < kVerifyWarps && before + sh.warp_sum[which][owner] <= mark; ++owner) before += sh.warp_sum[which][owner];
  const int64_t o0 = ((int64_t)rank * kVerifyWarps + owner) * share, left = min(share, p.vocab - o0);
  const Share<T, kAligned> ot(p.target + trow, o0, left), oq(two ? p.draft + qrow : p.target + trow, o0, two ? left : 0);
  const int stripes = (p.stripes + kVerifyWarps - 1) / kVerifyWarps;  // of a part
  uint64_t part = 0;
  uint4 a1, c1;
  auto fetch = [&](int s) {
    const int i = (warp * stripes + s) * 32 + lane;
    a1 = c1 = V::nothing();
    if (i < ot.whole) {
      a1 = ot.get(i);
      if (two) c1 = oq.get(i);
    } else if (i == ot.whole) {
      a1 = ot.rest(lane);
      if (two) c1 = oq.rest(lane);
    }
  };
  fetch(0);
#pragma unroll 1
  for (int pass = 0; pass < 2; ++pass) {  // the parts' sums, then the element
#pragma unroll 1
    for (int s = 0; s < stripes; ++s) {
      const int i = (warp * stripes + s) * 32 + lane;
      const uint4 a = a1, c = c1;
      fetch(s + 1 < stripes ? s + 1 : 0);  // (the next, or the first again)
      uint32_t w[E];
      uint64_t sum = 0;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        float x = t.weight(elem<T>(a, e));
        if (which == 2) {
          const float qe = two ? q.prob(elem<T>(c, e)) : o0 + i * E + e == d ? 1.f : 0.f;
          x = fmaxf(__fmul_rn(x, t.inv) - qe, 0.f);
        }
        w[e] = whole(x);
        sum += w[e];
      }
      const uint64_t stripe = warp_sum(sum);
      if (pass == 0) {
        part += stripe;
      } else if (mark < before + stripe) {
        uint64_t upto = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const uint64_t v = __shfl_up_sync(0xffffffffu, upto, o);
          if (lane >= o) upto += v;
        }
        upto += before;
        const int at = __ffs(__ballot_sync(0xffffffffu, upto > mark)) - 1;
        int32_t token = 0;
#pragma unroll
        for (int e = E - 1; e >= 0; --e) {  // (from behind: the first element whose sum up to it exceeds the mark stays)
          if (upto > mark) token = (int32_t)o0 + i * E + e;
          upto -= w[e];
        }
        finish_unit(p, row, pos, n, __shfl_sync(0xffffffffu, token, at) + 1);
        return;
      } else {
        before += stripe;
      }
    }
    if (pass == 1) return;
    if (lane == 0) sh.part_sum[warp] = part;
    __syncthreads();
    before += warp_sum(lane < warp ? sh.part_sum[lane] : 0);
    if (!(before <= mark && mark < before + part)) return;
  }
}

template <typename T, bool kAligned>
int launch_verify(VerifyParams& p, cudaStream_t st) {
  static std::atomic<bool> wide[kMaxDevices];  // clusters of 16 are allowed
  auto k = verify_kernel<T, kAligned>;
  const int64_t nvec = ((int64_t)p.vocab * sizeof(T) + 15) / 16;
  const int64_t units = (int64_t)p.rows * (p.max_draft + 1);
  auto stripes = [&](int c) { return (int)((nvec + (int64_t)c * kVerifyWarps * 32 - 1) / ((int64_t)c * kVerifyWarps * 32)); };
  // CTAs of a unit.  A CTA pays for three exchanges however little it reads, and reads
  // nothing meanwhile: its warps' shares are up to 40 stripes (20 KB), shorter (16) only to
  // have a few CTAs for each of the 608 that fit the SMs, so that they are at different
  // stages, and 8 only to fill the SMs.  Measured: 400 units of 2 x 128256 bf16 40 us with 4,
  // 47 with 2, 51 with 8 (fp32: 55.4 with 4, 57.6 with 8); 1024 of 3 x 152064 192 us with 2, 196 with 4; 192 of 262144
  // fp32 58 us with 8, 80 with 4.  Few units are cut further until the SMs have two CTAs each, but
  // a CTA on its own needs no cluster's barriers: 9 units of 4096 fp32 8.4 us with 1, 9.4 with 2.
  int c = 1;
  while (c < kVerifyCluster && stripes(c) > 40) c *= 2;
  while (c < 8 && ((units * c < 1600 && stripes(2 * c) >= 16) || (units * c < 608 && stripes(2 * c) >= 8))) c *= 2;
  while (c < kVerifyCluster && units * c < 304 && stripes(c) > 4) c *= 2;
  if (c > 8) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return cuda_error(e, "cudaGetDevice");
    if (dev >= kMaxDevices || !wide[dev].load(std::memory_order_acquire)) {
      e = cudaFuncSetAttribute(k, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
      if (e != cudaSuccess) return cuda_error(e, "verify attributes");
      if (dev < kMaxDevices) wide[dev].store(true, std::memory_order_release);
    }
  }
  p.stripes = stripes(c);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(units * c));
  cfg.blockDim = dim3(kVerifyThreads);
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim = {(unsigned)c, 1, 1};
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  cudaError_t e = cudaLaunchKernelEx(&cfg, k, p);
  if (e == cudaSuccess) e = cudaGetLastError();
  return e == cudaSuccess ? RGD_OK : cuda_error(e, "verify launch");
}

}  // namespace
}  // namespace rgd

using namespace rgd;

extern "C" size_t rgd_verify_draft_workspace_size(int32_t rows, int32_t max_draft) {
  clear_error();
  if (rows < 0 || max_draft < 0) {
    set_error(RGD_ERR_INVALID_ARG, "rgd_verify_draft_workspace_size: rows and max_draft must not be negative");
    return 0;
  }
  return (size_t)std::max(rows, 1) * ((size_t)max_draft + 2) * 4;
}

extern "C" int rgd_verify_draft(int32_t rows, int32_t max_draft, int32_t vocab, int32_t dtype, const void* target_logits,
                                int64_t target_stride, const void* draft_logits, int64_t draft_stride,
                                const int32_t* draft_tokens, const int32_t* n_draft, const uint8_t* is_probe,
                                const float* temperature, const float* min_p, const float* accept_u,
                                const float* draw_u, const uint8_t* row_active, int32_t* token_out,
                                int32_t* accepted_out, float* accept_prob, void* workspace, size_t workspace_bytes,
                                int32_t* dev_status, rgd_stream_t stream) {
  clear_error();
  const char* fn = "rgd_verify_draft";
  RGD_CHECK_ARG(rows >= 0 && max_draft >= 0, "%s: rows and max_draft must not be negative", fn);
  RGD_CHECK_ARG(vocab >= 1, "%s: vocab < 1", fn);
  RGD_CHECK_ARG(dtype == RGD_F32 || dtype == RGD_BF16, "%s: dtype must be RGD_F32 or RGD_BF16", fn);
  RGD_CHECK_ARG(target_stride >= vocab && (!draft_logits || draft_stride >= vocab), "%s: a stride is below vocab", fn);
  if (rows == 0) return RGD_OK;
  RGD_CHECK_ARG(target_logits && temperature && min_p && draw_u && token_out && accepted_out && workspace,
                "%s: target_logits/temperature/min_p/draw_u/token_out/accepted_out/workspace must be non-NULL", fn);
  RGD_CHECK_ARG(max_draft == 0 || (draft_tokens && accept_u), "%s: draft_tokens/accept_u must be non-NULL", fn);
  RGD_CHECK_ARG(aligned16(target_logits) && aligned16(draft_logits), "%s: logits must be 16-byte aligned", fn);
  RGD_CHECK_ARG((reinterpret_cast<uintptr_t>(workspace) & 3u) == 0, "%s: workspace must be 4-byte aligned", fn);
  RGD_CHECK_ARG(workspace_bytes >= rgd_verify_draft_workspace_size(rows, max_draft), "%s: workspace too small", fn);
  // (a lane has at most 512 of them then, and its sums are exact)
  if (vocab > 1 << 20) return set_error(RGD_ERR_UNSUPPORTED, "%s: vocab %d too large (max %d)", fn, vocab, 1 << 20);
  if ((int64_t)rows * ((int64_t)max_draft + 1) > 0x7fffffff / kVerifyCluster)
    return set_error(RGD_ERR_UNSUPPORTED, "%s: too many positions", fn);
  const int es = dtype == RGD_F32 ? 4 : 2;
  VerifyParams p{};
  p.target = static_cast<const uint8_t*>(target_logits);
  p.draft = max_draft ? static_cast<const uint8_t*>(draft_logits) : nullptr;
  p.target_stride = target_stride * es;
  p.draft_stride = draft_stride * es;
  p.rows = rows;
  p.max_draft = max_draft;
  p.vocab = vocab;
  p.tokens = draft_tokens;
  p.n_draft = n_draft;
  p.is_probe = is_probe;
  p.temperature = temperature;
  p.min_p = min_p;
  p.accept_u = accept_u;
  p.draw_u = draw_u;
  p.row_active = row_active;
  p.token_out = token_out;
  p.accepted_out = accepted_out;
  p.accept_prob = accept_prob;
  p.count = static_cast<int32_t*>(workspace);
  p.result = p.count + rows;
  p.dev_status = dev_status;
  cudaStream_t st = (cudaStream_t)stream;
  const bool aligned = p.target_stride % 16 == 0 && (!p.draft || p.draft_stride % 16 == 0);
  if (dtype == RGD_F32) return aligned ? launch_verify<float, true>(p, st) : launch_verify<float, false>(p, st);
  return aligned ? launch_verify<__nv_bfloat16, true>(p, st) : launch_verify<__nv_bfloat16, false>(p, st);
}
