// Verification of drafted tokens.  Row r has n drafted tokens d_0 .. d_{n-1} and the
// target's logits at the n + 1 positions they lead to; the draft's logits (or nothing,
// where each draft was certain) say what the tokens were drawn from.  With p and q the
// two sides' truncated softmax of temperature T and min-p,
//   d_k is accepted if u_k q(d_k) < p(d_k); at the first k that is not, the row's last
//   token is drawn from max(0, p - q); after n acceptances it is drawn from p,
// which leaves the emitted tokens distributed as if each were drawn from p.
//
// One thread-block cluster of C CTAs handles one position (a "unit": the target's row
// and, for k < n, the draft's).  Both rows are read from HBM once, into shared memory,
// each warp's contiguous share by a bulk copy of its own.  Three passes follow, with one
// exchange over the cluster after each:
//   1 the two maxima (a greedy row needs the argmax only);
//   2 the sums of the kept weights, and with them p(d), q(d) and the acceptance;
//   3 where the draft is rejected, the sums of max(0, p - q).
// A draw then picks the warp by prefix sums over the cluster and that warp searches its
// own share.  The last unit of a row to finish joins the row's results.
//
// Sums are exact in any order, and so is every token, whatever the cluster's size: a
// weight 2^x <= 1 is rounded once to a whole number of 2^-31 and summed in 64 bits.  The
// rounding is what a sum in fp32 does to a small weight too: it loses at most 2^-32 of
// the largest weight, 3e-5 of the sum in the worst case over 131072 tokens, where each
// is below 2.4e-10 of the largest.
#include <cuda_bf16.h>

#include <algorithm>
#include <cmath>

#include "common.h"
#include "ptx.cuh"

namespace rgd {
namespace {

constexpr int kVerifyWarps = 8;
constexpr int kVerifyThreads = kVerifyWarps * 32;
constexpr int kVerifyCluster = 16;                           // CTAs of a unit at most
constexpr int kSlots = kVerifyCluster * kVerifyWarps;        // warps of a unit at most
constexpr int kVerifySmem = 220 * 1024;                      // rows' bytes in one CTA at most
constexpr int32_t kTaken = -1, kRejectedRow = -2;            // results of a unit other than a token

struct VerifyParams {
  const uint8_t* target;
  const uint8_t* draft;  // NULL: every draft was certain
  int64_t target_stride, draft_stride;  // bytes
  int32_t rows, max_draft, vocab;
  int32_t wvec;  // 16-byte vectors of a row per warp (a multiple of 32)
  int32_t copy_target, copy_draft;  // the rows start on 16 bytes: bulk copies
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
  uint64_t sum[3][kSlots];   // pushed by every warp of the cluster: target's and draft's weights, the rest
  float top[2][kSlots];      // ... and the maxima
  uint64_t copied[kVerifyWarps];
  float theta;
};

// Element i of a 16-byte vector.
template <typename T>
__device__ __forceinline__ float elem(const uint4& w, int i);
template <>
__device__ __forceinline__ float elem<float>(const uint4& w, int i) {
  return __uint_as_float(i == 0 ? w.x : i == 1 ? w.y : i == 2 ? w.z : w.w);
}
template <>
__device__ __forceinline__ float elem<__nv_bfloat16>(const uint4& w, int i) {
  const uint32_t u = (i >> 1) == 0 ? w.x : (i >> 1) == 1 ? w.y : (i >> 1) == 2 ? w.z : w.w;
  return __uint_as_float((i & 1) ? (u & 0xffff0000u) : (u << 16));
}
template <typename T>
__device__ __forceinline__ T neg_inf();
template <>
__device__ __forceinline__ float neg_inf<float>() { return -INFINITY; }
template <>
__device__ __forceinline__ __nv_bfloat16 neg_inf<__nv_bfloat16>() { return __ushort_as_bfloat16(0xff80u); }
template <typename T>
__device__ __forceinline__ float one_logit(const uint8_t* row, int32_t i) {
  return (float)reinterpret_cast<const T*>(row)[i];
}

// One side's softmax: weights 2^((l - top) kexp) of the logits at or above the cutoff,
// and the reciprocal of their sum.
struct Side {
  float top, cut, kexp, inv;
  __device__ float weight(float l) const { return l >= cut ? ex2_approx((l - top) * kexp) : 0.f; }
  __device__ float prob(float l) const { return __fmul_rn(weight(l), inv); }
};

// w 2^31, rounded to the nearest whole number, for 0 <= w <= 1.  Up to 2^-8 the sum with
// 2^23 does the rounding and holds the number in its low bits; above, w 2^31 is whole.
__device__ __forceinline__ uint32_t whole(float w) {
  if (w > 0x1p-8f) return __float2uint_rz(w * 0x1p31f);
  return __float_as_uint(fmaf(w, 0x1p31f, 0x1p23f)) - 0x4b000000u;
}

// Two fp32 values in one 64-bit register, and arithmetic on both at once.
__device__ __forceinline__ uint64_t pair(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void unpair(uint64_t v, float& a, float& b) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v));
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint32_t word_sum(uint64_t v) { return (uint32_t)v + (uint32_t)(v >> 32); }

// A lane's sum of whole(w), exact for up to 512 numbers.  Small ones (w <= 2^-8) are added
// as the bits of w 2^31 + 2^23.  Others go in two halves, w = a 2^-15 + r with a the
// nearest whole number, and w 2^31 = a 2^16 + r 2^31, both again read off the bits of a sum
// (2^23, and 1.5 2^23 for r's sign).  Conversions to integers would take the special
// function unit's time, which the exponentials need.
struct WholeSum {
  uint32_t low = 0, a = 0, b = 0;
  __device__ void small(uint64_t w2) {
    low += word_sum(fma2(w2, pair(0x1p31f, 0x1p31f), pair(0x1p23f, 0x1p23f))) - 2u * 0x4b000000u;
  }
  __device__ void any(uint64_t w2) {
    const uint64_t h = fma2(w2, pair(0x1p15f, 0x1p15f), pair(0x1p23f, 0x1p23f));
    const uint64_t n = add2(h, pair(-0x1p23f, -0x1p23f));
    const uint64_t r = fma2(n, pair(-0x1p-15f, -0x1p-15f), w2);
    a += word_sum(h) - 2u * 0x4b000000u;
    b += word_sum(fma2(r, pair(0x1p31f, 0x1p31f), pair(0x1.8p23f, 0x1.8p23f))) - 2u * 0x4b400000u;
  }
  __device__ uint64_t total() const { return (uint64_t)low + ((uint64_t)a << 16) + (uint64_t)(int64_t)(int32_t)b; }
};

// 16 bytes of logits: pairs of them, their maximum, and whether any is at or above a bound.
template <typename T>
struct Vec;
template <>
struct Vec<float> {
  static constexpr int kPairs = 2;
  using Max = float;
  struct Bound {
    float v;
    __device__ explicit Bound(float x) : v(x) {}
  };
  __device__ static Max lowest() { return -INFINITY; }
  __device__ static Max max_of(const uint4& w, Max m) {
    return fmaxf(fmaxf(fmaxf(fmaxf(m, __uint_as_float(w.x)), __uint_as_float(w.y)), __uint_as_float(w.z)), __uint_as_float(w.w));
  }
  __device__ static float value(Max m) { return m; }
  __device__ static bool reaches(Max m, const Bound& b) { return m >= b.v; }
  __device__ static void get(const uint4& w, int i, float& a, float& b) {
    a = __uint_as_float(i ? w.z : w.x);
    b = __uint_as_float(i ? w.w : w.y);
  }
};
template <>
struct Vec<__nv_bfloat16> {
  static constexpr int kPairs = 4;
  using Max = __nv_bfloat162;
  // (a bf16 is >= an fp32 bound exactly if it is >= the bound rounded up to bf16)
  struct Bound {
    __nv_bfloat162 v;
    __device__ explicit Bound(float x) : v(__bfloat162bfloat162(__float2bfloat16_ru(x))) {}
  };
  __device__ static __nv_bfloat162 b2(uint32_t u) { return *reinterpret_cast<const __nv_bfloat162*>(&u); }
  __device__ static Max lowest() { return b2(0xff80ff80u); }
  __device__ static Max max_of(const uint4& w, Max m) {  // (NaN never wins, as with fmaxf)
    return __hmax2(__hmax2(__hmax2(b2(w.x), b2(w.y)), __hmax2(b2(w.z), b2(w.w))), m);
  }
  __device__ static float value(Max m) {
    const uint32_t u = *reinterpret_cast<const uint32_t*>(&m);
    return fmaxf(__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u));
  }
  __device__ static bool reaches(Max m, const Bound& b) { return __hge2_mask(m, b.v) != 0; }
  __device__ static void get(const uint4& w, int i, float& a, float& b) {
    const uint32_t u = i == 0 ? w.x : i == 1 ? w.y : i == 2 ? w.z : w.w;
    a = __uint_as_float(u << 16);
    b = __uint_as_float(u & 0xffff0000u);
  }
};

// The sum of a share's weights, in whole multiples of 2^-31.
template <typename T>
__device__ __forceinline__ uint64_t sum_weights(const uint4* v, int mine, const Side& side, int lane) {
  using V = Vec<T>;
  WholeSum sum;
  const bool open = side.cut == -INFINITY;  // no truncation
  const typename V::Bound cut(side.cut), big(side.top - 8.001f / side.kexp);  // (below `big` a weight is under 2^-8)
  const uint64_t top = pair(-side.top, -side.top), kexp = pair(side.kexp, side.kexp);
  for (int i = lane; i < mine; i += 32) {
    const uint4 w = v[i];
    const typename V::Max m = V::max_of(w, V::lowest());
    if (!open && !V::reaches(m, cut)) continue;
    const bool small = open && !V::reaches(m, big);
#pragma unroll
    for (int e = 0; e < V::kPairs; ++e) {
      float a, b;
      V::get(w, e, a, b);
      unpair(mul2(add2(pair(a, b), top), kexp), a, b);
      // (2^-200 is 0; NaN and -inf end there too)
      if (open) {
        a = fmaxf(a, -200.f);
        b = fmaxf(b, -200.f);
      } else {
        float la, lb;
        V::get(w, e, la, lb);
        a = la >= side.cut ? a : -200.f;
        b = lb >= side.cut ? b : -200.f;
      }
      const uint64_t w2 = pair(ex2_approx(a), ex2_approx(b));
      if (small) sum.small(w2);
      else sum.any(w2);
    }
  }
  return sum.total();
}

__device__ __forceinline__ uint64_t warp_sum(uint64_t v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}

__device__ __forceinline__ uint32_t peer_addr(uint32_t addr, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
  return r;
}
__device__ __forceinline__ void push(const uint64_t* slot, uint64_t v, uint32_t rank) {
  asm volatile("st.shared::cluster.b64 [%0], %1;" ::"r"(peer_addr(smem_u32(slot), rank)), "l"(v) : "memory");
}
__device__ __forceinline__ void push(const float* slot, float v, uint32_t rank) {
  asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(peer_addr(smem_u32(slot), rank)), "f"(v) : "memory");
}
// What was pushed before is seen by every CTA of the cluster after it.
__device__ __forceinline__ void cluster_exchange() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// The whole warp: a row's finished unit is counted, and the last one to finish writes the row.
__device__ void finish_unit(const VerifyParams& p, int row, int pos, int n, int32_t result) {
  const int lane = threadIdx.x & 31;
  int32_t* res = p.result + (int64_t)row * (p.max_draft + 1);
  int last = 0;
  if (lane == 0) {
    res[pos] = result;
    int32_t old;
    asm volatile("atom.acq_rel.gpu.global.add.s32 %0, [%1], 1;" : "=r"(old) : "l"(p.count + row) : "memory");
    last = old == n;
  }
  if (!__shfl_sync(0xffffffffu, last, 0)) return;
  __syncwarp();
  int taken = n;
  int32_t token = kRejectedRow;
  for (int base = 0; base <= n; base += 32) {
    const int32_t v = base + lane <= n ? __ldcg(res + base + lane) : kTaken;
    const uint32_t stop = __ballot_sync(0xffffffffu, v != kTaken);
    if (stop) {
      const int at = __ffs(stop) - 1;
      taken = base + at;
      token = __shfl_sync(0xffffffffu, v, at);
      break;
    }
  }
  const bool good = token != kRejectedRow;
  for (int i = lane; i <= p.max_draft; i += 32)
    p.token_out[(int64_t)row * (p.max_draft + 1) + i] =
        !good || i > taken ? -1 : i < taken ? p.tokens[(int64_t)row * p.max_draft + i] : token;
  if (lane == 0) {
    p.accepted_out[row] = good ? taken : 0;
    p.count[row] = 0;
  }
}

// One warp's share of one row into shared memory; elements past the row's end read as
// -inf.  Bulk copies where the row starts on 16 bytes.
template <typename T>
__device__ __forceinline__ uint32_t fetch_share(uint4* dst, const uint8_t* row, int32_t vocab, int32_t v0, int32_t wvec,
                                                bool bulk, uint64_t* bar, int lane) {
  constexpr int E = 16 / (int)sizeof(T);
  const int32_t e0 = v0 * E;                                   // first element
  const int32_t ne = min(max(vocab - e0, 0), wvec * E);        // elements of the row here
  const int32_t nv = bulk ? ne / E : 0;
  if (lane == 0 && nv) bulk_load(dst, row + (int64_t)e0 * sizeof(T), (uint32_t)nv * 16, bar);
  T* d = reinterpret_cast<T*>(dst);
  const T* s = reinterpret_cast<const T*>(row) + e0;
  const int32_t end = (ne + E - 1) / E * E;  // whole vectors
#pragma unroll 8
  for (int32_t i = nv * E + lane; i < end; i += 32) d[i] = i < ne ? s[i] : neg_inf<T>();
  return (uint32_t)nv * 16;
}

template <typename T>
__global__ void __launch_bounds__(kVerifyThreads) verify_kernel(const VerifyParams p) {
  constexpr int E = 16 / (int)sizeof(T);
  extern __shared__ __align__(16) uint8_t dyn[];
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
  const float temp = p.temperature[row], min_p = p.min_p[row];
  const bool greedy = (p.is_probe && p.is_probe[row]) || temp == 0.f;
  const int n = p.n_draft ? p.n_draft[row] : K;
  const float draw_u = p.draw_u[row];
  bool good = n >= 0 && n <= K;
  if (!greedy) good = good && temp > 0.f && temp < INFINITY && min_p >= 0.f && min_p <= 1.f && draw_u >= 0.f && draw_u < 1.f;
  const bool leader = rank == 0 && warp == 0;
  const bool has_draft = good && pos < n;
  if (leader && lane == 0 && pos < K && p.accept_prob && !(active && has_draft)) p.accept_prob[(int64_t)row * K + pos] = 0.f;
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
  const uint8_t* trow = p.target + ((int64_t)row * (K + 1) + pos) * p.target_stride;
  const uint8_t* qrow = two ? p.draft + ((int64_t)row * K + pos) * p.draft_stride : nullptr;

  // This warp's share, and its place among the cluster's warps (in index order).
  const int slot = (int)rank * kVerifyWarps + warp, slots = (int)csize * kVerifyWarps;
  const int32_t v0 = slot * p.wvec;
  const int32_t mine = min(max((p.vocab + E - 1) / E - v0, 0), p.wvec);  // its vectors
  uint4* tv = reinterpret_cast<uint4*>(dyn) + (int64_t)warp * p.wvec;
  uint4* qv = reinterpret_cast<uint4*>(dyn) + (int64_t)(kVerifyWarps + warp) * p.wvec;
  uint64_t* bar = &sh.copied[warp];
  if (lane == 0) {
    mbar_init(bar, 1);
    fence_mbar_init();
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  __syncwarp();
  cluster_arrive_relaxed();
  uint32_t bytes = fetch_share<T>(tv, trow, p.vocab, v0, p.wvec, p.copy_target, bar, lane);
  if (two) bytes += fetch_share<T>(qv, qrow, p.vocab, v0, p.wvec, p.copy_draft, bar, lane);
  if (lane == 0) mbar_arrive_expect_tx(bar, bytes);
  const float td = d_in && !greedy ? one_logit<T>(trow, d) : 0.f;
  const float qd = d_in && two ? one_logit<T>(qrow, d) : 0.f;
  if (threadIdx.x == 0) sh.theta = (float)((double)temp * log((double)min_p));
  __syncwarp();
  bool copied = mbar_wait(bar, 0);
  if (!copied) {
    if (p.dev_status) atomicOr(p.dev_status, RGD_DEV_WAIT_TIMEOUT);
    copied = mbar_wait(bar, 0);  // (the copy in flight, before this block may end)
  }
  __syncwarp();

  // Pass 1: the maxima (NaN never wins).
  using V = Vec<T>;
  typename V::Max tmax = V::lowest(), qmax = V::lowest();
  for (int i = lane; i < mine; i += 32) tmax = V::max_of(tv[i], tmax);
  if (two)
    for (int i = lane; i < mine; i += 32) qmax = V::max_of(qv[i], qmax);
  float tm = V::value(tmax), qm = V::value(qmax);
  tm = warp_max(tm);
  if (two) qm = warp_max(qm);
  cluster_wait();  // every CTA of the cluster has started
  if (lane < (int)csize) {
    push(&sh.top[0][slot], tm, lane);
    if (two) push(&sh.top[1][slot], qm, lane);
  }
  cluster_exchange();
  Side t, q;
  t.top = q.top = -INFINITY;
  for (int i = lane; i < slots; i += 32) {
    t.top = fmaxf(t.top, sh.top[0][i]);
    if (two) q.top = fmaxf(q.top, sh.top[1][i]);
  }
  t.top = warp_max(t.top);
  if (two) q.top = warp_max(q.top);
  const bool finite = fabsf(t.top) < INFINITY && (!two || fabsf(q.top) < INFINITY) && (!has_draft || greedy || (u >= 0.f && u < 1.f));
  if (!finite) {
    if (leader) {
      if (lane == 0 && p.dev_status) atomicOr(p.dev_status, RGD_DEV_BAD_PARAM);
      if (lane == 0 && has_draft && p.accept_prob) p.accept_prob[(int64_t)row * K + pos] = 0.f;
      finish_unit(p, row, pos, n, kRejectedRow);
    }
    return;
  }
  if (has_draft && !d_in && leader && lane == 0 && p.dev_status) atomicOr(p.dev_status, RGD_DEV_BAD_TOKEN);

  if (greedy) {  // the lowest index of the largest logit
    uint32_t best = 0xffffffffu;
    for (int i = lane; i < mine && best == 0xffffffffu; i += 32) {
      const uint4 a = tv[i];
      if (V::value(V::max_of(a, V::lowest())) != t.top) continue;
#pragma unroll
      for (int e = E - 1; e >= 0; --e)
        if (elem<T>(a, e) == t.top) best = (uint32_t)(v0 + i) * E + e;
    }
    best = __reduce_min_sync(0xffffffffu, best);
    if (lane == 0) push(&sh.sum[0][slot], best, 0);
    cluster_exchange();
    if (leader) {
      uint32_t b = 0xffffffffu;
      for (int i = lane; i < slots; i += 32) b = min(b, (uint32_t)sh.sum[0][i]);
      b = __reduce_min_sync(0xffffffffu, b);
      const bool same = has_draft && (int32_t)b == d;
      if (lane == 0 && has_draft && p.accept_prob) p.accept_prob[(int64_t)row * K + pos] = same ? 1.f : 0.f;
      finish_unit(p, row, pos, n, same ? kTaken : (int32_t)b);
    }
    return;
  }

  // Pass 2: the sums of the weights.
  t.kexp = q.kexp = fminf(__fdiv_rn(1.4426950408889634f, temp), 3e38f);  // (finite: 0 times it is 0)
  t.cut = __fadd_rn(t.top, sh.theta);
  q.cut = __fadd_rn(q.top, sh.theta);
  uint64_t ts = sum_weights<T>(tv, mine, t, lane), qs = 0;
  if (two) qs = sum_weights<T>(qv, mine, q, lane);
  ts = warp_sum(ts);
  if (two) qs = warp_sum(qs);
  if (lane < (int)csize) {
    push(&sh.sum[0][slot], ts, lane);
    if (two) push(&sh.sum[1][slot], qs, lane);
  }
  cluster_exchange();
  uint64_t tz = 0, qz = 0;
  for (int i = lane; i < slots; i += 32) {
    tz += sh.sum[0][i];
    if (two) qz += sh.sum[1][i];
  }
  tz = warp_sum(tz);
  t.inv = __fdiv_rn(1.f, __ull2float_rn(tz) * 0x1p-31f);
  if (two) {
    qz = warp_sum(qz);
    q.inv = __fdiv_rn(1.f, __ull2float_rn(qz) * 0x1p-31f);
  }
  int which = 0;  // the sums that the draw goes by: the target's weights, or the rest
  if (has_draft) {
    const float pd = d_in ? t.prob(td) : 0.f;
    const float qp = !d_in ? 0.f : two ? q.prob(qd) : 1.f;
    const bool taken = d_in && __fmul_rn(u, qp) < pd;
    if (leader && lane == 0 && p.accept_prob)
      p.accept_prob[(int64_t)row * K + pos] = qp > 0.f ? fminf(__fdiv_rn(pd, qp), 1.f) : pd > 0.f ? 1.f : 0.f;
    if (taken) {
      if (leader) finish_unit(p, row, pos, n, kTaken);
      return;
    }
    // Pass 3: the sums of max(0, p - q); a certain draft takes its own token's p alone.
    if (d_in) {
      WholeSum rest;
      const typename V::Bound cut(t.cut);
      for (int i = lane; i < mine; i += 32) {
        const uint4 a = tv[i];
        if (!V::reaches(V::max_of(a, V::lowest()), cut)) continue;  // (p is 0 there)
        const uint4 b = two ? qv[i] : a;
#pragma unroll
        for (int e = 0; e < V::kPairs; ++e) {
          float x, y, u0 = 0.f, u1 = 0.f;
          V::get(a, e, x, y);
          if (two) {
            V::get(b, e, u0, u1);
            u0 = q.prob(u0);
            u1 = q.prob(u1);
          } else {
            u0 = (v0 + i) * E + 2 * e == d ? 1.f : 0.f;
            u1 = (v0 + i) * E + 2 * e + 1 == d ? 1.f : 0.f;
          }
          rest.any(pair(fmaxf(t.prob(x) - u0, 0.f), fmaxf(t.prob(y) - u1, 0.f)));
        }
      }
      uint64_t rs = rest.total();
      rs = warp_sum(rs);
      if (lane < (int)csize) push(&sh.sum[2][slot], rs, lane);
      cluster_exchange();
      uint64_t rz = 0;
      for (int i = lane; i < slots; i += 32) rz += sh.sum[2][i];
      if (warp_sum(rz) > 0) which = 2;  // (p and q may be equal but for rounding: then p itself)
    }
  }

  // The draw: the warp whose share holds the mark, by prefix sums over the cluster's warps.
  uint64_t total = 0, before = 0;
  for (int i = lane; i < slots; i += 32) {
    total += sh.sum[which][i];
    before += i < slot ? sh.sum[which][i] : 0;
  }
  total = warp_sum(total);
  before = warp_sum(before);
  const uint64_t mark = (uint64_t)((double)draw_u * (double)total);
  const uint64_t here = sh.sum[which][slot];
  if (!(before <= mark && mark < before + here)) return;
  for (int base = 0; base < mine; base += 32) {
    const int i = base + lane;
    uint32_t w[E];
    uint64_t s = 0;
    const uint4 a = i < mine ? tv[i] : make_uint4(0, 0, 0, 0);
    const uint4 b = two && i < mine ? qv[i] : a;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      float x = t.weight(elem<T>(a, e));
      if (which == 2) {
        const float qe = two ? q.prob(elem<T>(b, e)) : (v0 + i) * E + e == d ? 1.f : 0.f;
        x = fmaxf(__fmul_rn(x, t.inv) - qe, 0.f);
      }
      w[e] = i < mine ? whole(x) : 0u;
      s += w[e];
    }
    uint64_t incl = s;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint64_t v = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += v;
    }
    const uint32_t hit = __ballot_sync(0xffffffffu, before + incl > mark);
    if (hit) {
      const int at = __ffs(hit) - 1;
      uint64_t c = before + incl - s;
      int32_t token = 0;
#pragma unroll
      for (int e = E - 1; e >= 0; --e) {
        uint64_t upto = c;
#pragma unroll
        for (int f = 0; f <= e; ++f) upto += w[f];
        if (upto > mark) token = (v0 + i) * E + e;
      }
      finish_unit(p, row, pos, n, __shfl_sync(0xffffffffu, token, at));
      return;
    }
    before += __shfl_sync(0xffffffffu, incl, 31);
  }
}

template <typename T>
int launch_verify(VerifyParams& p, bool two, cudaStream_t st) {
  static std::atomic<bool> done[kMaxDevices];
  auto k = verify_kernel<T>;
  if (int rc = ensure_smem(k, kVerifySmem, done)) return rc;
  const int64_t nvec = ((int64_t)p.vocab * sizeof(T) + 15) / 16;
  const int64_t units = (int64_t)p.rows * (p.max_draft + 1);
  auto share = [&](int c) { return (int)((nvec + (int64_t)c * kVerifyWarps * 32 - 1) / ((int64_t)c * kVerifyWarps * 32)) * 32; };
  auto bytes = [&](int c) { return (int64_t)share(c) * kVerifyWarps * 16 * (two ? 2 : 1); };
  // CTAs of a unit: three to an SM, so that one's passes run behind another's copies; more
  // where the units alone do not fill the SMs.
  int c = 1;
  while (c < kVerifyCluster && (bytes(c) > 72 * 1024 || (units * c < 304 && share(c) > 32))) c *= 2;
  if (bytes(c) > kVerifySmem)
    return set_error(RGD_ERR_UNSUPPORTED, "rgd_verify_draft: vocab %d too large", p.vocab);
  if (c > 8) {
    const cudaError_t e = cudaFuncSetAttribute(k, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess) return cuda_error(e, "verify attributes");
  }
  p.wvec = share(c);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(units * c));
  cfg.blockDim = dim3(kVerifyThreads);
  cfg.dynamicSmemBytes = (size_t)bytes(c);
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
  p.copy_target = p.target_stride % 16 == 0;
  p.copy_draft = p.draft_stride % 16 == 0;
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
  const bool two = p.draft != nullptr;
  return dtype == RGD_F32 ? launch_verify<float>(p, two, (cudaStream_t)stream)
                          : launch_verify<__nv_bfloat16>(p, two, (cudaStream_t)stream);
}
