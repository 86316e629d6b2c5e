// Sampling with temperature, top-k, top-p and min-p from given uniforms.  Tokens are ordered
// by their logits, the largest first, equal ones by their index.  S is the first k of those
// that min-p leaves; the kept tokens are the shortest run of S from its front whose weights
// reach p times S's; the token is drawn from them in the order of their indices.
//
// Weights 2^((l - top) log2(e)/T) are whole multiples of 2^-31 and summed in 64 bits, so that
// every sum, every cut and every token is the same whatever order it is worked out in.
//
// One cluster of CTAs a row, every warp with a contiguous share of it:
//   1 the maximum, a stream from HBM; and a bound that enough tokens surely reach: a warp's
//     r-th largest lane maximum, the smallest over all warps, is reached by r tokens of each;
//   2 the tokens that reach the bound are listed, and the lists meet in the first CTA's shared
//     memory (the row lies in L2 now, and only vectors whose group reaches the bound are read); top-p
//     alone needs all the weights' sum as well.  The first CTA sorts the list.  Where k, or the
//     mass p, lies within it the row is done: the usual case, two exchanges.
//   3 else the cut is searched for: a range of logits, at first from a sample of the row, is
//     divided into 512 by a histogram of counts or weights; the part that holds the cut is the
//     next range, until what it holds fits the list or is one value.  Then a pass for the kept
//     tokens' sums by warp, and one warp finds the token.
// No sorting of whole rows, no limit on k or on how flat a row is.
//
// Measured: 80 rows of 128256 with the usual filters 19 us (bf16) and 21 us (fp32), fp32 with top-p
// alone 92 us; 512 of 152064 bf16 with filters of all kinds 106 us, with top-p alone 158 us; 5 of
// 32001 fp32 with top-p alone 34 us.  A row's stages
// follow one another, and the first CTA works while the others of its cluster wait: that bounds
// few rows and rows whose list suffices (15 % of HBM in the second case); rows that are searched
// are bound by the instructions for every token's weight and place, three times each.
#include <cuda_bf16.h>

#include <algorithm>
#include <cmath>

#include "common.h"
#include "log_pair.cuh"
#include "logit_rows.cuh"
#include "ptx.cuh"

namespace rgd {
namespace {

constexpr int kTopWarps = 8;
constexpr int kTopThreads = kTopWarps * 32;
constexpr int kTopCluster = 16;  // CTAs of a row at most
constexpr int kList = 2048;      // tokens that the list holds at most,
constexpr int kSorted = 1024;    // and that are sorted together
constexpr int kEnough = 128;     // tokens that the first list shall hold at least for top-p
constexpr int kBins = 512;
constexpr int kCopies = 3, kCopyPitch = kBins + 8;  // (the same bin lies on another bank in each)
constexpr int kSampleShift = 3;  // 1 stripe of 8 is sampled
constexpr int kMostRounds = 64;

struct TopParams {
  const uint8_t* logits;
  int64_t stride;  // bytes
  int32_t rows, vocab, stripes;
  const uint8_t* is_probe;
  const float* temperature;
  const int32_t* top_k;
  const float* top_p;
  const float* min_p;
  const float* draw_u;
  const uint8_t* row_active;
  int32_t* token_out;
  int32_t* kept_count;
  float* prob_out;
  int32_t* dev_status;
};

// What the first CTA tells the others to do next.
enum Next { kDone, kRange, kDraw };
struct Order {
  int next;
  int by_count;         // the cut is at a count, not a mass
  int list;             // the range's tokens go into the list, in case that they fit
  uint32_t from, to;    // range of keys' distances from the largest
  uint32_t last_key;    // the last kept value, and how many of it are kept (0: all)
  uint32_t of_last;
  int pad;
  uint64_t need;        // count or mass up to the cut, the last token included
};
static_assert(sizeof(Order) % 8 == 0, "");

struct TopShared {
  float warp_top[kTopWarps], warp_low[kTopWarps], top[kTopCluster], low[kTopCluster];
  uint64_t warp_sum[kTopWarps], sum[kTopCluster], part_sum[kTopWarps];
  uint32_t warp_count[kTopWarps], count[kTopCluster], part_count[kTopWarps];
  uint32_t warp_larger[kTopWarps], larger[kTopCluster];  // (of the first CTA only)
  uint64_t scan[kTopWarps];
  uint32_t lo[kBins], hi[kBins];  // sums of the weights' low 16 bits and of the rest, or counts
  uint32_t listed;                // tokens that belong into the list
  uint32_t list_from;             // where this CTA's go in the first one's
  Order order;
  float theta;
  int found;
  union {
    uint64_t list[kList];
    uint32_t copies[kCopies][kCopyPitch];  // of the bins, for counts while there is no list
  };
};

__device__ __forceinline__ void cluster_barrier() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t load_peer(uint32_t addr) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ void store_peer(uint32_t addr, uint32_t v) {
  asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}
__device__ __forceinline__ void store_peer(uint32_t addr, uint64_t v) {
  asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(addr), "l"(v) : "memory");
}

// Keys in the order of the logits, consecutive for consecutive values of the type; -0 and 0 have
// the same.  key_of an fp32 that is no bf16: the key of the next bf16 above.
template <typename T>
__device__ __forceinline__ uint32_t key_of(float l) {
  if (sizeof(T) == 2) l = __bfloat162float(__float2bfloat16_ru(l));
  const uint32_t u = __float_as_uint(l == 0.f ? 0.f : l), key = u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
  return sizeof(T) == 2 ? key >> 16 : key;
}
template <typename T>
__device__ __forceinline__ float of_key(uint32_t k) {
  if (sizeof(T) == 2) return __uint_as_float((k & 0x8000u) ? (k & 0x7fffu) << 16 : (~k & 0xffffu) << 16);
  return __uint_as_float((k & 0x80000000u) ? k ^ 0x80000000u : ~k);
}
// The key of element e of a vector that is no NaN.
template <typename T>
__device__ __forceinline__ uint32_t key_at(const uint4& w, int e) {
  if (sizeof(T) == 4) return key_of<T>(elem<T>(w, e));
  const uint32_t pair = (e >> 1) == 0 ? w.x : (e >> 1) == 1 ? w.y : (e >> 1) == 2 ? w.z : w.w;
  const uint32_t u = (e & 1) ? pair >> 16 : pair & 0xffffu, key = u ^ ((u & 0x8000u) ? 0xffffu : 0x8000u);
  return key == 0x7fffu ? 0x8000u : key;
}

// Those of all its elements (a NaN's is above every other one or below).
template <typename T>
__device__ __forceinline__ void keys_of(const uint4& w, uint32_t (&key)[16 / (int)sizeof(T)]) {
  const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 4) {
      key[i] = key_of<T>(__uint_as_float(v[i]));
    } else {
      const __nv_bfloat162 z = __hadd2(*reinterpret_cast<const __nv_bfloat162*>(&v[i]), __nv_bfloat162(0.f, 0.f));  // (no -0)
      const uint32_t u = *reinterpret_cast<const uint32_t*>(&z), k = u ^ ((u >> 15 & 0x10001u) * 0xffffu | 0x80008000u);
      key[2 * i] = k & 0xffffu;
      key[2 * i + 1] = k >> 16;
    }
  }
}

template <typename T>
__device__ __forceinline__ bool one_value(const uint4& w) {
  return w.x == w.y && w.x == w.z && w.x == w.w && (sizeof(T) == 4 || w.x >> 16 == (w.x & 0xffffu));
}

// The bins of a sample, by how many octaves a weight lies below the largest: 1/32 octave each for the
// first eight (at high temperatures nearly all tokens are there), then 1/16; the last one holds the rest.
constexpr int kFine = kBins / 2;
__device__ __forceinline__ int octave_bin(float octaves) {
  return (int)fminf(octaves < 8.f ? octaves * 32.f : kFine + (octaves - 8.f) * 16.f, (float)(kBins - 1));
}
__device__ __forceinline__ float octaves_of(int bin) {  // where it starts
  return bin < kFine ? (float)bin * 0.03125f : 8.f + (float)(bin - kFine) * 0.0625f;
}

// Which elements of a vector are in [from, below), as bits (NaN is nowhere).
template <typename T>
__device__ __forceinline__ uint32_t elements_in(const uint4& w, float from, float below) {
  uint32_t m = 0;
#pragma unroll
  for (int e = 0; e < 16 / (int)sizeof(T); ++e) {
    const float l = elem<T>(w, e);
    m |= l >= from && !(l >= below) ? 1u << e : 0u;
  }
  return m;
}

// f(vector, its number) for every vector of a lane's part that may reach `bound`.
template <typename T, bool kAligned, typename F>
__device__ __forceinline__ void visit(const Share<T, kAligned>& v, const Kept& kept, float bound, int stripes, int lane, F&& f) {
  using V = Vec<T>;
  const uint32_t mask = groups_reaching(kept, bound);
  const int steps = (int)__reduce_max_sync(0xffffffffu, (uint32_t)__popc(mask)) * ((stripes + kGroups - 1) / kGroups);
  if (7 * steps > 4 * stripes) {  // all of them, in order
#pragma unroll 1
    for (int i = lane; i < v.whole; i += 32 * 4) {
      uint4 x[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        x[k] = V::nothing();
        if (i + 32 * k < v.whole) x[k] = v.get(i + 32 * k);
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) f(x[k], i + 32 * k);
    }
  } else {
    Walk walk(mask, stripes, v.whole, lane);
    int i = walk.next();
    uint4 w = V::nothing();
    if (i >= 0) w = v.get(i);
#pragma unroll 1
    while (i >= 0) {
      const int ahead = walk.next();
      uint4 w1 = V::nothing();
      if (ahead >= 0) w1 = v.get(ahead);
      f(w, i);
      w = w1;
      i = ahead;
    }
  }
  f(kept.rest, v.whole);
}

// The same with code for one vector alone, two on their way.  (A range's pass, unrolled four times, does not
// stay in the instruction cache: 45 us of a row of 152064 among 512, 29 so.)
template <typename T, bool kAligned, typename F>
__device__ __forceinline__ void visit_each(const Share<T, kAligned>& v, const Kept& kept, float bound, int stripes, int lane, F&& f) {
  using V = Vec<T>;
  Walk walk(groups_reaching(kept, bound), stripes, v.whole, lane);
  int i = walk.next(), i1 = walk.next();
  uint4 w = V::nothing(), w1 = w;
  if (i >= 0) w = v.get(i);
  if (i1 >= 0) w1 = v.get(i1);
#pragma unroll 1
  for (;;) {
    const int i2 = walk.next();
    uint4 w2 = V::nothing();
    if (i2 >= 0) w2 = v.get(i2);
    const bool end = i < 0;
    if (end) w = kept.rest;
    f(w, end ? v.whole : i);
    if (end) break;
    w = w1, w1 = w2;
    i = i1, i1 = i2;
  }
}

// Sorts the first n = 256 R numbers or fewer (a power of two from 32 on) of a list in shared memory,
// the largest first, those from `count` on taken as 0.  The whole CTA, R numbers a thread; they
// pass through shared memory only from warp to warp.  (All in shared memory, with a barrier a
// step, 1024 numbers took 12 us.)
template <int R>
__device__ __forceinline__ void sort_numbers(uint64_t* list, int n, int count) {
  const int first = threadIdx.x * R;
  uint64_t v[R];
#pragma unroll
  for (int r = 0; r < R; ++r) v[r] = first + r < count ? list[first + r] : 0;
#pragma unroll 1
  for (int size = 2; size <= n; size *= 2) {
#pragma unroll 1
    for (int gap = size / 2; gap >= 32 * R; gap /= 2) {
      __syncthreads();
#pragma unroll
      for (int r = 0; r < R; ++r) list[first + r] = v[r];
      __syncthreads();
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const int i = first + r;
        const uint64_t other = i < n ? list[i ^ gap] : 0;
        const bool larger = ((i & gap) == 0) == ((i & size) == 0);  // this place gets the larger one
        v[r] = larger == (v[r] > other) ? v[r] : other;
      }
    }
#pragma unroll 1
    for (int gap = min(size / 2, 16 * R); gap >= R; gap /= 2) {
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const int i = first + r;
        const uint64_t other = __shfl_xor_sync(0xffffffffu, v[r], gap / R);
        const bool larger = ((i & gap) == 0) == ((i & size) == 0);
        v[r] = larger == (v[r] > other) ? v[r] : other;
      }
    }
#pragma unroll
    for (int gap = R / 2; gap > 0; gap /= 2) {
      if (gap >= size) continue;
#pragma unroll
      for (int r = 0; r < R; ++r) {
        if (r & gap) continue;
        const bool down = ((first + r) & size) == 0;
        const uint64_t x = v[r], y = v[r | gap];
        if ((x < y) == down) {
          v[r] = y;
          v[r | gap] = x;
        }
      }
    }
  }
  __syncthreads();
#pragma unroll
  for (int r = 0; r < R; ++r) list[first + r] = v[r];
  __syncthreads();
}
// The whole CTA; at most kSorted numbers.
__device__ __noinline__ void sort_down(uint64_t* list, int count) {
  int n = 32;
  while (n < count) n *= 2;
  if (n <= 256) sort_numbers<1>(list, n, count);
  else if (n <= 512) sort_numbers<2>(list, n, count);
  else sort_numbers<4>(list, n, count);
}

// Sum over the threads before this one, and over all.  The whole CTA.
__device__ __forceinline__ uint64_t scan_before(TopShared& sh, uint64_t v, uint64_t& all) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint64_t upto = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint64_t x = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += x;
  }
  __syncthreads();  // (may still be read from the scan before)
  if (lane == 31) sh.scan[warp] = upto;
  __syncthreads();
  uint64_t before = 0;
  all = 0;
#pragma unroll
  for (int w = 0; w < kTopWarps; ++w) {
    before += w < warp ? sh.scan[w] : 0;
    all += sh.scan[w];
  }
  return before + upto - v;
}

// The n-th largest (from 1) of the first `count` lanes' values, -inf if there are fewer.
__device__ __forceinline__ float nth_largest(float v, int n, int count) {
  const int lane = threadIdx.x & 31;
  int larger = 0;
#pragma unroll 8
  for (int o = 0; o < count; ++o) {
    const float x = __shfl_sync(0xffffffffu, v, o);
    larger += x > v || (x == v && o < lane);
  }
  return warp_max(lane < count && larger == n - 1 ? v : -INFINITY);
}

__device__ __forceinline__ uint32_t whole_weight(const Side& side, float l) { return whole(side.weight(l)); }
__device__ __forceinline__ uint64_t share_of(float p, uint64_t total) {  // ceil(p total), at least 1
  const uint64_t need = (uint64_t)ceil((double)p * (double)total);
  return need ? need : 1;
}

// The first CTA: the first `keep` tokens of the sorted list of n are kept; draws from them and
// writes the row's results.
template <typename T>
__device__ __noinline__ void finish_list(const TopParams& p, TopShared& sh, const Side& side, int row, int keep, float u) {
  if (threadIdx.x == 0 && p.kept_count) p.kept_count[row] = keep;
  if (keep <= 32) {  // one warp, a token a lane: the weights of lower indices are added up as they are
    if (threadIdx.x >= 32) return;
    const int lane = threadIdx.x;
    const uint64_t t = lane < keep ? sh.list[lane] : 0;
    const uint32_t index = ~(uint32_t)t, w = lane < keep ? whole_weight(side, of_key<T>((uint32_t)(t >> 32))) : 0;
    uint64_t before = 0, total = 0;
    for (int i = 0; i < keep; ++i) {
      const uint32_t other = __shfl_sync(0xffffffffu, index, i), x = __shfl_sync(0xffffffffu, w, i);
      total += x;
      before += other < index ? x : 0;
    }
    const uint64_t mark = (uint64_t)((double)u * (double)total);
    if (before <= mark && mark < before + w) {
      p.token_out[row] = (int32_t)index;
      if (p.prob_out) p.prob_out[row] = __fdiv_rn((float)w, __ull2float_rn(total));
    }
    return;
  }
  for (int i = threadIdx.x; i < keep; i += kTopThreads) {
    const uint64_t t = sh.list[i];
    // (the complement of the index, and the weight)
    sh.list[i] = t << 32 | whole_weight(side, of_key<T>((uint32_t)(t >> 32)));
  }
  __syncthreads();
  sort_down(sh.list, keep);  // by index
  const int each = (keep + kTopThreads - 1) / kTopThreads, first = threadIdx.x * each;
  uint64_t mine = 0, total;
  for (int i = 0; i < each; ++i)
    if (first + i < keep) mine += (uint32_t)sh.list[first + i];
  uint64_t before = scan_before(sh, mine, total);
  const uint64_t mark = (uint64_t)((double)u * (double)total);
  for (int i = 0; i < each; ++i) {
    if (first + i >= keep) break;
    const uint64_t e = sh.list[first + i];
    const uint32_t w = (uint32_t)e;
    if (before <= mark && mark < before + w) {
      p.token_out[row] = (int32_t)~(uint32_t)(e >> 32);
      if (p.prob_out) p.prob_out[row] = __fdiv_rn((float)w, __ull2float_rn(total));
    }
    before += w;
  }
}

template <typename T, bool kAligned>
__global__ void __launch_bounds__(kTopThreads, 4) sample_top_kernel(const TopParams p) {
  constexpr int E = 16 / (int)sizeof(T);
  using V = Vec<T>;
  __shared__ TopShared sh;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint32_t rank, csize, urow;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(csize));
  asm volatile("mov.u32 %0, %%clusterid.x;" : "=r"(urow));
  const int row = (int)urow;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");  // (a dependent waits for this kernel's end)
  asm volatile("griddepcontrol.wait;" ::: "memory");
  // The row's parameters; every thread of the cluster takes the same decisions.
  const bool active = !p.row_active || p.row_active[row];
  const float temp = p.temperature[row], u = p.draw_u[row];
  const float min_p = p.min_p ? p.min_p[row] : 0.f, top_p = p.top_p ? p.top_p[row] : 1.f;
  const bool greedy = (p.is_probe && p.is_probe[row]) || temp == 0.f;
  const int k = p.top_k && p.top_k[row] > 0 && p.top_k[row] < p.vocab ? p.top_k[row] : 0;
  bool good = true;
  if (!greedy)
    good = temp > 0.f && temp < INFINITY && min_p >= 0.f && min_p <= 1.f && top_p >= 0.f && top_p <= 1.f && u >= 0.f && u < 1.f;
  auto nothing = [&](bool bad) {
    if (rank != 0 || threadIdx.x != 0) return;
    p.token_out[row] = -1;
    if (p.kept_count) p.kept_count[row] = 0;
    if (p.prob_out) p.prob_out[row] = 0.f;
    if (bad && p.dev_status) atomicOr(p.dev_status, RGD_DEV_BAD_PARAM);
  };
  if (!active || !good) return nothing(active);
  const bool cut_mass = !greedy && top_p < 1.f;

  // This warp's share, in the order of the elements over the cluster.
  const uint8_t* logits = p.logits + row * p.stride;
  const int64_t share = (int64_t)p.stripes * 32 * E;
  const int64_t e0 = ((int64_t)rank * kTopWarps + warp) * share;
  const Share<T, kAligned> v(logits, e0, min(share, p.vocab - e0));
  if (threadIdx.x == 0) {
    sh.listed = 0;
    sh.theta = scaled_log(greedy ? 1.f : temp, greedy ? 1.f : min_p);
  }

  // Pass 1: the maximum (NaN never wins), and a bound that `wanted` tokens reach.
  Kept kept;
  // (A bound that `wanted` tokens reach, by the lanes' maxima: the each-th largest of a warp; the fourth
  // of a CTA's warps; the some-th of the CTAs.  So half of the row may hold nothing of interest.  A
  // warp takes part if every lane has a vector.)
  const bool full_share = (int64_t)p.vocab - e0 >= 32 * E;
  const int wanted = greedy ? 0 : k ? k : cut_mass ? min(kEnough, p.vocab) : 0;
  const int half = ((int)csize + 1) / 2, each = min(max((wanted + 4 * half - 1) / (4 * half), 1), 32);
  const int some = (wanted + 4 * each - 1) / (4 * each);
  const bool bounded = some <= (int)csize;
  {
    const float mine = find_lane_maxima(v, kept, p.stripes, lane), top = warp_max(mine);
    float low = -INFINITY;
    if (wanted && bounded && full_share) {  // the each-th largest of the lanes' maxima
      low = nth_largest(mine, each, 32);
    }
    if (lane == 0) {
      sh.warp_top[warp] = top;
      sh.warp_low[warp] = low;
    }
  }
  __syncthreads();
  cluster_arrive_relaxed();  // every CTA of the cluster has started
  cluster_wait();
  if (warp == 0) {
    const float t = warp_max(sh.warp_top[lane % kTopWarps]);
    const float l = nth_largest(lane < kTopWarps ? sh.warp_low[lane] : -INFINITY, 4, kTopWarps);
    if (lane < (int)csize) {
      store_peer(peer_addr(smem_u32(&sh.top[rank]), lane), __float_as_uint(t));
      store_peer(peer_addr(smem_u32(&sh.low[rank]), lane), __float_as_uint(l));
    }
  }
  cluster_barrier();
  Side side;
  side.top = warp_max(sh.top[lane % csize]);
  const float low = nth_largest(lane < (int)csize ? sh.low[lane] : -INFINITY, max(some, 1), (int)csize);
  if (!(fabsf(side.top) < INFINITY)) return nothing(true);

  if (greedy) {  // the lowest index of the largest logit
    uint32_t best = 0xffffffffu;
    auto look = [&](const uint4& w, int i) {
#pragma unroll
      for (int e = E - 1; e >= 0; --e)
        if (elem<T>(w, e) == side.top) best = min(best, (uint32_t)e0 + i * E + e);
    };
    Walk walk(groups_reaching(kept, side.top), p.stripes, v.whole, lane);
#pragma unroll 1
    for (int i = walk.next(); i >= 0; i = walk.next()) look(v.get(i), i);
    look(kept.rest, v.whole);
    best = __reduce_min_sync(0xffffffffu, best);
    if (lane == 0) sh.warp_count[warp] = best;
    __syncthreads();
    if (warp == 0) {
      best = __reduce_min_sync(0xffffffffu, sh.warp_count[lane % kTopWarps]);
      if (lane == 0) store_peer(peer_addr(smem_u32(&sh.count[rank]), 0), best);
    }
    cluster_barrier();
    if (rank == 0 && warp == 0) {
      best = __reduce_min_sync(0xffffffffu, sh.count[lane % csize]);
      if (lane == 0) {
        p.token_out[row] = (int32_t)best;
        if (p.kept_count) p.kept_count[row] = 1;
        if (p.prob_out) p.prob_out[row] = 1.f;
      }
    }
    return;
  }
  side.kexp = fminf(__fdiv_rn(1.4426950408889634f, temp), 3e38f);  // (finite: 0 times it is 0)
  side.cut = fmaxf(__fadd_rn(side.top, sh.theta), -3.4028234663852886e38f);  // (-inf is never kept)
  const uint32_t top_key = key_of<T>(side.top);

  const uint32_t list_count = peer_addr(smem_u32(&sh.listed), 0), list_at = peer_addr(smem_u32(&sh.list[0]), 0);
  // Every CTA lists its own tokens, and what the others have listed then goes to the first one together (a count
  // there for each token's sake takes 0.5 us a token and warp).  The lanes that come together count together; a
  // lane that has seen the list full adds no more: the count is above kList then.
  bool full = false;
  auto enlist = [&](float l, uint32_t index) {
    if (full) return;
    const uint32_t with = __activemask();
    const int first = __ffs(with) - 1;
    uint32_t at = 0;
    if (lane == first) at = atomicAdd(&sh.listed, __popc(with));
    at = __shfl_sync(with, at, first) + __popc(with & ((1u << lane) - 1));
    if (at < kList) sh.list[at] = (uint64_t)key_of<T>(l) << 32 | (uint32_t)~index;
    else full = true;
  };
  auto hand_over = [&]() {
    if (rank == 0) return;
    __syncthreads();
    const uint32_t n = sh.listed;
    if (n == 0) return;
    if (threadIdx.x == 0)
      asm volatile("atom.relaxed.cluster.shared::cluster.add.u32 %0, [%1], %2;" : "=r"(sh.list_from) : "r"(list_count), "r"(n) : "memory");
    __syncthreads();
    const uint32_t to = sh.list_from;
    for (uint32_t i = threadIdx.x; i < n && to + i < kList; i += kTopThreads) store_peer(list_at + 8 * (to + i), sh.list[i]);
    if (threadIdx.x == 0) sh.listed = 0;
  };
  // Every CTA's sum and count into every CTA.
  auto exchange = [&](uint64_t sum, uint32_t count, uint32_t larger) {
    if (lane == 0) {
      sh.warp_larger[warp] = larger;
      sh.warp_sum[warp] = sum;
      sh.warp_count[warp] = count;
    }
    __syncthreads();
    if (warp == 0) {
      const uint64_t s = warp_sum(lane < kTopWarps ? sh.warp_sum[lane] : 0);
      const uint32_t c = __reduce_add_sync(0xffffffffu, lane < kTopWarps ? sh.warp_count[lane] : 0);
      const uint32_t l = __reduce_add_sync(0xffffffffu, lane < kTopWarps ? sh.warp_larger[lane] : 0);
      if (lane == 0) store_peer(peer_addr(smem_u32(&sh.larger[rank]), 0), l);
      if (lane < (int)csize) {
        store_peer(peer_addr(smem_u32(&sh.sum[rank]), lane), s);
        store_peer(peer_addr(smem_u32(&sh.count[rank]), lane), c);
      }
    }
    cluster_barrier();
  };
  auto sum_all = [&]() { return warp_sum(lane < (int)csize ? sh.sum[lane] : 0); };
  auto count_all = [&]() { return __reduce_add_sync(0xffffffffu, lane < (int)csize ? sh.count[lane] : 0); };
  // The first CTA's order into every CTA.
  auto publish = [&]() {
    __syncthreads();
    if (warp == 0 && lane < (int)csize && lane > 0) {
      const uint64_t* from = reinterpret_cast<const uint64_t*>(&sh.order);
      const uint32_t to = peer_addr(smem_u32(&sh.order), lane);
#pragma unroll
      for (int i = 0; i < (int)sizeof(Order) / 8; ++i) store_peer(to + 8 * i, from[i]);
    }
  };
  auto clear_bins = [&]() {
    for (int i = threadIdx.x; i < kBins; i += kTopThreads) sh.lo[i] = sh.hi[i] = 0;
    __syncthreads();
  };
  // A bin's sum over the cluster (the first CTA).
  auto bin_sum = [&](int b, bool high) {
    uint64_t s = 0;
    for (uint32_t r = 0; r < csize; ++r) {
      s += load_peer(peer_addr(smem_u32(&sh.lo[b]), r));
      if (high) s += (uint64_t)load_peer(peer_addr(smem_u32(&sh.hi[b]), r)) << 16;
    }
    return s;
  };

  uint64_t total = 0;  // of S's weights, once known
  if (k || cut_mass) {
    // Pass 2.
    const float bound = bounded ? fmaxf(low, side.cut) : INFINITY;
    const bool sampled = !k || bound == INFINITY;
    if (sampled) clear_bins();
    WholeSum sum;
    const float scale = side.kexp;
    // (What few tokens need is done one token after another, in code that is there once: unrolled
    // into the stream of vectors it took seven times as long as the sums.  And where all vectors are
    // streamed, only after it, for the vectors of a lane that reach the bound: two warps in three have
    // one among 32, a lane one in 30.)
    const typename V::Bound at_bound(bound);
    auto list_vector = [&](const uint4& w, int i) {
      uint32_t m = elements_in<T>(w, bound, INFINITY);
#pragma unroll 1
      for (; m; m &= m - 1) {
        const int e = __ffs(m) - 1;
        enlist(elem<T>(w, e), (uint32_t)e0 + i * E + e);
      }
    };
    if (sampled) {
      uint64_t hits = 0;  // the lane's stripes (64 at most)
      visit(v, kept, side.cut, p.stripes, lane, [&](const uint4& w, int i) {
        if (!k) add_weights<T>(w, side, typename V::Bound(side.cut), sum);
        if (((i >> 5) & ((1 << kSampleShift) - 1)) == 0) {
#pragma unroll
          for (int e = 0; e < E; ++e) {
            const float l = elem<T>(w, e);
            if (l >= side.cut && !(l >= bound))
              atomicAdd(&sh.lo[octave_bin((side.top - l) * scale)], k ? 1u : whole_weight(side, l) >> 13);
          }
        }
        if (i < v.whole && V::reaches(V::max_of(w, V::lowest()), at_bound)) hits |= 1ull << (i >> 5);
      });
      list_vector(kept.rest, v.whole);
#pragma unroll 1
      while (hits) {
        const int i = (__ffsll(hits) - 1) * 32 + lane;
        hits &= hits - 1;
        list_vector(v.get(i), i);
      }
    } else {
      visit_each(v, kept, bound, p.stripes, lane, [&](const uint4& w, int i) {
        if (V::reaches(V::max_of(w, V::lowest()), at_bound)) list_vector(w, i);
      });
    }
    hand_over();
    exchange(k ? 0 : warp_sum(sum.total()), 0, 0);
    if (rank == 0) {
      total = sum_all();
      const uint32_t listed = sh.listed;
      const int n = (int)min(listed, (uint32_t)kList);
      int keep = -1;  // known to be cut within the list
      uint64_t in_list = 0, need = k ? (uint64_t)k : share_of(top_p, total);
      if (listed <= kList && bound < INFINITY) {
        bool within = n <= kSorted;
        if (!k) {
          uint64_t mine = 0;
          for (int i = threadIdx.x; i < n; i += kTopThreads) mine += whole_weight(side, of_key<T>((uint32_t)(sh.list[i] >> 32)));
          scan_before(sh, mine, in_list);
          within = within && need <= in_list;
        }
        if (within) sort_down(sh.list, n);
        const int m = k ? min(k, n) : n;  // of S
        const int per = (n + kTopThreads - 1) / kTopThreads, first = threadIdx.x * per;
        uint64_t mine = 0;
        if (cut_mass && within) {
          for (int i = 0; i < per; ++i)
            if (first + i < m) mine += whole_weight(side, of_key<T>((uint32_t)(sh.list[first + i] >> 32)));
          uint64_t before = scan_before(sh, mine, in_list);
          if (k) {
            total = in_list;
            need = share_of(top_p, total);
          }
          if (threadIdx.x == 0) sh.found = -1;
          __syncthreads();
          for (int i = 0; i < per; ++i) {
            if (first + i >= m) break;
            const uint32_t w = whole_weight(side, of_key<T>((uint32_t)(sh.list[first + i] >> 32)));
            if (before < need && need <= before + w) sh.found = first + i + 1;
            before += w;
          }
          __syncthreads();
          keep = sh.found;
        } else if (within) {
          keep = m;
        }
      }
      if (threadIdx.x == 0) {
        sh.order.next = keep >= 0 ? kDone : kRange;
        sh.order.by_count = k > 0;
        sh.order.list = 0;
        sh.order.need = need;
        sh.order.from = 0;
        // (weights 33 octaves down are 0)
        sh.order.to = top_key - key_of<T>(k ? side.cut : fmaxf(side.cut, side.top - 33.f / side.kexp));
      }
      __syncthreads();
      if (keep < 0 && bound < INFINITY && listed <= kList && (k || need <= in_list)) {  // within a long list
        if (threadIdx.x == 0) sh.order.to = top_key - key_of<T>(bound);
      } else if (keep < 0 && (k == 0 || bound == INFINITY) && (bound == INFINITY || listed <= kList)) {
        // Where the cut is likely to be, from the sample: what it holds below the list stands for the rest.
        const uint64_t b0 = bin_sum(2 * threadIdx.x, false), b1 = bin_sum(2 * threadIdx.x + 1, false);
        uint64_t all;
        uint64_t upto = scan_before(sh, b0 + b1, all);
        const uint64_t rest = k ? 0 : total - in_list;
        // (a stripe in 8, or in as many as a share has; what of k's sample stands for is not known better)
        const float at = k ? (float)need / (float)min(1 << kSampleShift, p.stripes)
                           : rest ? (float)(need - in_list) / (float)rest * (float)all : 0.f;
        // A sum over a sample that each token is in by chance has the variance sum w^2 (of those in it).
        // Bins from three deviations before the cut to three behind it are searched.
        uint64_t squares;
        scan_before(sh, k ? b0 + b1 : (uint64_t)((float)b0 * exp2f(18.f - octaves_of(2 * threadIdx.x)) + (float)b1 * exp2f(18.f - octaves_of(2 * threadIdx.x + 1))),
                    squares);
        const float off = (float)all * 0.005f + 3.f * sqrtf((float)squares);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int bin = 2 * threadIdx.x + i;
          const float before = (float)upto, after = (float)(upto += i ? b1 : b0);
          if (before <= at - off && at - off < after)
            sh.order.from = top_key - key_of<T>(fminf(side.top - octaves_of(bin) / side.kexp, side.top));
          if (before < at + off && at + off <= after && bin + 1 < kBins) {
            const float lo = side.top - octaves_of(bin + 1) / side.kexp;
            if (lo > side.cut) sh.order.to = top_key - key_of<T>(lo);
          }
        }
        __syncthreads();
        if (threadIdx.x == 0 && sh.order.from > sh.order.to) sh.order.from = 0;
      }
      publish();
      if (keep >= 0) {
        cluster_barrier();
        finish_list<T>(p, sh, side, row, keep, u);
        return;
      }
      if (threadIdx.x == 0) sh.listed = 0;
    }
    cluster_barrier();
    if (sh.order.next == kDone) return;

    // Pass 3, until the cut is found: what lies above the range, and in each of its parts.
    // (A round leaves 1/512 of a range of less than 2^32: four, and four more for the mass of what a count leaves.
    // Before them, a sampled range that misses the cut is followed by one next to it, at least eight times as wide:
    // eleven reach over every key.  No search of a row that stays as it is takes kMostRounds.)
    int rounds = 0;
#pragma unroll 1
    while (sh.order.next == kRange) {
      if (++rounds > kMostRounds) {  // (uniform over the cluster)
        nothing(false);
        if (rank == 0 && threadIdx.x == 0 && p.dev_status) atomicOr(p.dev_status, RGD_DEV_WAIT_TIMEOUT);
        return;
      }
      const uint32_t from = sh.order.from, to = sh.order.to;
      const bool by_count = sh.order.by_count, list = sh.order.list;
      int shift = 0;
      while (((to - from) >> shift) >= (uint32_t)kBins) ++shift;
      const float in_range = of_key<T>(top_key - to);                          // the smallest of it,
      const float above = from ? of_key<T>(top_key - from + 1) : INFINITY;     // and of what lies above it
      // Counts of few values meet at the same places: lanes take turns over four sets of bins.
      const bool counts = by_count || shift == 0;  // (of a value, the count tells the mass)
      const bool apart = counts && !list;
      const bool masses = !by_count || cut_mass;
      __syncthreads();
      if (apart)
        for (int i = threadIdx.x; i < kCopies * kCopyPitch; i += kTopThreads) (&sh.copies[0][0])[i] = 0;
      clear_bins();
      uint32_t* const my_bins = apart && (lane & 3) ? sh.copies[(lane & 3) - 1] : sh.lo;
      const uint32_t bins_at = smem_u32(my_bins);
      WholeSum over;
      full = false;
      uint32_t count = 0;
      visit_each(v, kept, in_range, p.stripes, lane, [&](const uint4& w, int i) {
        if (from) {
          if (masses) add_weights<T>(w, side, typename V::Bound(above), over);
          if (by_count) count += __popc(elements_in<T>(w, above, INFINITY));
        }
        auto add = [&](float l, uint32_t key, uint32_t times) {
          const uint32_t b = (top_key - key - from) >> shift;
          if (counts) {
            atomicAdd(&my_bins[b], times);
          } else {
            const uint32_t x = whole_weight(side, l);
            if (x & 0xffffu) atomicAdd(&sh.lo[b], (x & 0xffffu) * times);
            if (x >> 16) atomicAdd(&sh.hi[b], (x >> 16) * times);
          }
        };
        if (one_value<T>(w) && !list) {  // (as in a row of few values: they would all wait for one bin)
          const float l = elem<T>(w, 0);
          if (l >= in_range && !(l >= above)) add(l, key_at<T>(w, 0), E);
          return;
        }
        if (counts) {  // without a branch for each element (512 x 152064 with top-p alone: 158 us so, 179 with)
          uint32_t key[E];
          keys_of<T>(w, key);
#pragma unroll
          for (int e = 0; e < E; ++e) {
            const uint32_t d = top_key - from - key[e];  // (what lies above the range wraps to more than its width)
            asm volatile("{\n\t.reg .pred p;\n\tsetp.le.u32 p, %0, %1;\n\t@p red.shared.add.u32 [%2], 1;\n\t}" ::"r"(d), "r"(to - from), "r"(bins_at + (d >> shift) * 4) : "memory");
          }
        } else {
#pragma unroll
          for (int e = 0; e < E; ++e) {
            const float l = elem<T>(w, e);
            if (l >= in_range && !(l >= above)) add(l, key_at<T>(w, e), 1);
          }
        }
        if (!list || full) return;
        uint32_t m = elements_in<T>(w, in_range, above);
#pragma unroll 1
        for (; m; m &= m - 1) {
          const int e = __ffs(m) - 1;
          enlist(elem<T>(w, e), (uint32_t)e0 + i * E + e);
        }
      });
      if (apart) {
        __syncthreads();
        for (int i = threadIdx.x; i < kBins; i += kTopThreads)
          for (int c = 0; c < kCopies; ++c) sh.lo[i] += sh.copies[c][i];
      }
      if (list) hand_over();
      exchange(warp_sum(over.total()), __reduce_add_sync(0xffffffffu, count), 0);
      if (rank == 0) {
        const uint64_t mass = sum_all();
        const uint32_t counted = count_all(), listed = sh.listed;
        const uint64_t before = by_count ? counted : mass, need = sh.order.need;
        const int bin = 2 * threadIdx.x;
        uint64_t b0 = bin_sum(bin, !by_count && shift > 0), b1 = bin_sum(bin + 1, !by_count && shift > 0);
        uint64_t mass_before = 0;  // of this thread's bins, where a count's cut needs it
        if (shift == 0 && (cut_mass || !by_count)) {
          const uint32_t key = top_key - from - bin;
          const uint64_t m0 = b0 ? b0 * whole_weight(side, of_key<T>(key)) : 0, m1 = b1 ? b1 * whole_weight(side, of_key<T>(key - 1)) : 0;
          if (by_count) {
            uint64_t all;
            mass_before = mass + scan_before(sh, m0 + m1, all);
          } else {
            b0 = m0;
            b1 = m1;
          }
        }
        uint64_t inside;
        uint64_t upto = before + scan_before(sh, b0 + b1, inside);
        __syncthreads();  // (every thread has read the order)
        bool cut = false;      // found, at (last_key, of_last), by this thread
        uint32_t last_key = 0, of_last = 0;
        uint64_t mass_upto = 0;  // up to the cut, known where the cut is at a count
        // (A sampled range that misses the cut: next to it, eight times as wide.)
        const uint32_t wider = (to - from) < 0x0fffffffu ? 8 * (to - from) + 8 : 0xffffffffu;
        if (need <= before) {
          if (threadIdx.x == 0) {
            sh.order.from = from > wider ? from - wider : 0;
            sh.order.to = from - 1;
          }
        } else if (need > before + inside) {  // (by a count: fewer than k tokens, if the range reaches down to the cutoff)
          const uint32_t lowest = top_key - key_of<T>(side.cut);
          if (to < lowest) {
            if (threadIdx.x == 0) {
              sh.order.from = to + 1;
              sh.order.to = lowest - to > wider ? to + wider : lowest;
            }
          } else if (threadIdx.x == 0) {
            sh.order.need = before + inside;  // all of them
          }
        } else if (list && listed <= kSorted) {
          const int n = (int)listed;
          sort_down(sh.list, n);
          const int per = (n + kTopThreads - 1) / kTopThreads, first = threadIdx.x * per;
          uint64_t mine = 0, all;
          for (int i = 0; i < per; ++i)
            if (first + i < n) mine += whole_weight(side, of_key<T>((uint32_t)(sh.list[first + i] >> 32)));
          uint64_t at = mass + scan_before(sh, mine, all);
          for (int i = 0; i < per; ++i) {
            const int j = first + i;
            if (j >= n) break;
            const uint32_t key = (uint32_t)(sh.list[j] >> 32), w = whole_weight(side, of_key<T>(key));
            if (by_count ? counted + j + 1 == need : at < need && need <= at + w) {
              cut = true;
              last_key = key;
              int f = j;  // the first of this value
              while (f > 0 && (uint32_t)(sh.list[f - 1] >> 32) == key) --f;
              of_last = (uint32_t)(j - f + 1);
              mass_upto = at + w;
            }
            at += w;
          }
        } else {  // the part that holds the cut
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const uint64_t b = i ? b1 : b0;
            if (upto < need && need <= upto + b && shift == 0) {  // one value
              last_key = top_key - from - (bin + i);
              const uint64_t w = whole_weight(side, of_key<T>(last_key)), unit = by_count ? 1 : w;
              cut = true;
              of_last = (uint32_t)((need - upto + unit - 1) / unit);
              mass_upto = mass_before + of_last * w;
              if (i) mass_upto += b0 * whole_weight(side, of_key<T>(last_key + 1));  // (by a count: b0 is one)
            } else if (upto < need && need <= upto + b) {
              const uint32_t start = from + ((uint32_t)(bin + i) << shift);
              sh.order.from = start;
              sh.order.to = min(to, start + ((1u << shift) - 1));
              // (bf16s are few values, found within another round; a mass does not tell of how many tokens)
              sh.order.list = sizeof(T) == 4 && (!by_count || b <= kSorted);
            }
            upto += b;
          }
        }
        if (cut) {
          if (by_count && cut_mass) {  // S is known now; next where its mass is cut
            sh.order.by_count = 0;
            sh.order.need = share_of(top_p, mass_upto);
            sh.order.from = 0;
            sh.order.to = top_key - last_key;
          } else {
            sh.order.next = kDraw;
            sh.order.last_key = last_key;
            sh.order.of_last = of_last;
          }
        }
        publish();
        if (threadIdx.x == 0) sh.listed = 0;
      }
      cluster_barrier();
    }
  } else if (threadIdx.x == 0) {  // all that the cutoff leaves
    sh.order.last_key = key_of<T>(side.cut);
    sh.order.of_last = 0;
  }
  __syncthreads();

  // The kept tokens' sums by warp: those above the last kept value, and the lowest indices of it.
  const uint32_t of_last = sh.order.of_last;
  const float last = of_key<T>(sh.order.last_key), above = of_last ? of_key<T>(sh.order.last_key + 1) : side.cut;
  const uint64_t last_weight = of_last ? whole_weight(side, last) : 0;
  WholeSum sum;
  uint32_t ties = 0, larger = 0;
  visit(v, kept, of_last ? last : above, p.stripes, lane, [&](const uint4& w, int) {
    add_weights<T>(w, side, typename V::Bound(above), sum);
    larger += __popc(elements_in<T>(w, above, INFINITY));
    if (of_last) ties += __popc(elements_in<T>(w, last, above));
  });
  exchange(warp_sum(sum.total()), __reduce_add_sync(0xffffffffu, ties), __reduce_add_sync(0xffffffffu, larger));
  total = sum_all() + (uint64_t)of_last * last_weight;
  if (rank == 0 && p.kept_count && warp == 0) {
    const uint32_t n = __reduce_add_sync(0xffffffffu, lane < (int)csize ? sh.larger[lane] : 0);
    if (lane == 0) p.kept_count[row] = (int32_t)(n + of_last);
  }
  // The CTA, then the share, that holds the mark.
  const uint64_t mark = (uint64_t)((double)u * (double)total);
  auto held = [&](uint64_t s, uint64_t before_ties, uint32_t n) {  // a stretch's mass, with the ties that are kept
    const uint64_t left = before_ties < of_last ? of_last - before_ties : 0;
    return s + (of_last ? min((uint64_t)n, left) * last_weight : 0);
  };
  uint64_t before = 0, tied = 0;
  for (uint32_t r = 0; r < rank; ++r) {
    before += held(sh.sum[r], tied, sh.count[r]);
    tied += sh.count[r];
  }
  if (!(before <= mark && mark < before + held(sh.sum[rank], tied, sh.count[rank]))) return;
  int owner = 0;
  for (; owner + 1 < kTopWarps; ++owner) {
    const uint64_t h = held(sh.warp_sum[owner], tied, sh.warp_count[owner]);
    if (mark < before + h) break;
    before += h;
    tied += sh.warp_count[owner];
  }
  // Every warp takes a part of that share, and the one whose part holds the mark finds the token.
  const int64_t o0 = ((int64_t)rank * kTopWarps + owner) * share;
  const Share<T, kAligned> o(logits, o0, min(share, p.vocab - o0));
  const int stripes = (p.stripes + kTopWarps - 1) / kTopWarps;
  uint64_t part = 0;
  uint32_t part_ties = 0;
#pragma unroll 1
  for (int pass = 0; pass < 2; ++pass) {
#pragma unroll 1
    for (int s = 0; s < stripes; ++s) {
      const int i = (warp * stripes + s) * 32 + lane;
      uint4 a = V::nothing();
      if (s + warp * stripes < p.stripes) {
        if (i < o.whole) a = o.get(i);
        else if (i == o.whole) a = o.rest(lane);
      }
      uint64_t own = 0;
      uint32_t n = 0;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float l = elem<T>(a, e);
        if (l >= above) own += whole_weight(side, l);
        else if (of_last && l >= last) ++n;
      }
      const uint64_t stripe = warp_sum(own);
      const uint32_t stripe_ties = __reduce_add_sync(0xffffffffu, n);
      if (pass == 0) {
        part += stripe;
        part_ties += stripe_ties;
        continue;
      }
      const uint64_t h = held(stripe, tied, stripe_ties);
      if (!(mark < before + h)) {
        before += h;
        tied += stripe_ties;
        continue;
      }
      uint32_t ties_upto = n;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const uint32_t x = __shfl_up_sync(0xffffffffu, ties_upto, d);
        if (lane >= d) ties_upto += x;
      }
      uint64_t rank_of = tied + ties_upto - n;  // ties before this lane's
      const uint64_t mine = held(own, rank_of, n);
      uint64_t upto = mine;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const uint64_t x = __shfl_up_sync(0xffffffffu, upto, d);
        if (lane >= d) upto += x;
      }
      uint64_t at = before + upto - mine;
      if (at <= mark && mark < at + mine) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float l = elem<T>(a, e);
          uint64_t w = 0;
          if (l >= above) w = whole_weight(side, l);
          else if (of_last && l >= last && rank_of++ < of_last) w = last_weight;
          if (at <= mark && mark < at + w) {
            p.token_out[row] = (int32_t)(o0 + (int64_t)i * E + e);
            if (p.prob_out) p.prob_out[row] = __fdiv_rn((float)(uint32_t)w, __ull2float_rn(total));
          }
          at += w;
        }
      }
      return;
    }
    if (pass == 1) return;
    if (lane == 0) {
      sh.part_sum[warp] = part;
      sh.part_count[warp] = part_ties;
    }
    __syncthreads();
    for (int w = 0; w < warp; ++w) {
      before += held(sh.part_sum[w], tied, sh.part_count[w]);
      tied += sh.part_count[w];
    }
    if (!(before <= mark && mark < before + held(part, tied, part_ties))) return;
  }
}

template <typename T, bool kAligned>
int launch_top(TopParams& p, cudaStream_t st) {
  static std::atomic<bool> wide[kMaxDevices];  // clusters of 16 are allowed
  auto k = sample_top_kernel<T, kAligned>;
  const int64_t nvec = ((int64_t)p.vocab * sizeof(T) + 15) / 16;
  auto stripes = [&](int c) { return (int)((nvec + (int64_t)c * kTopWarps * 32 - 1) / ((int64_t)c * kTopWarps * 32)); };
  // CTAs of a row: shares of up to 32 stripes (16 KB) a warp (and 65536 tokens a CTA at most: a bin's
  // sums stay below 2^32), shorter only to have a few CTAs for every SM.
  int c = 1;
  while (c < kTopCluster && (stripes(c) > 32 || (int64_t)stripes(c) * kTopWarps * 32 * (16 / (int)sizeof(T)) > 65536)) c *= 2;
  while (c < 8 && (int64_t)p.rows * c < 608 && stripes(2 * c) >= 4) c *= 2;
  // A row whose cut is searched for takes several times as long as the others, so that four CTAs pay where a call has
  // such rows, and cost where it has none (us, two and four; the usual filters, then filters of all kinds: 310 x 128256
  // bf16 25 and 31, 133 and 67; 512 x 128256 43 and 49, 145 and 89; 512 x 70001 41 and 54, 101 and 92; 512 x 50257 fp32
  // 39 and 50, 129 and 97).  Only the device knows the filters; up to 3.5 rounds of four (beyond, 560 x 128256: 45 and
  // 52, 143 and 102).
  if (c == 2 && p.rows <= 532 && stripes(4) >= 8) c = 4;
  while (c < kTopCluster && (int64_t)p.rows * c < 304 && stripes(c) > 4) c *= 2;
  if (c > 8) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return cuda_error(e, "cudaGetDevice");
    if (dev >= kMaxDevices || !wide[dev].load(std::memory_order_acquire)) {
      e = cudaFuncSetAttribute(k, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
      if (e != cudaSuccess) return cuda_error(e, "sampling attributes");
      if (dev < kMaxDevices) wide[dev].store(true, std::memory_order_release);
    }
  }
  p.stripes = stripes(c);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((int64_t)p.rows * c));
  cfg.blockDim = dim3(kTopThreads);
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
  return e == cudaSuccess ? RGD_OK : cuda_error(e, "sampling launch");
}

}  // namespace
}  // namespace rgd

using namespace rgd;

extern "C" int rgd_sample_top(int32_t rows, int32_t vocab, int32_t dtype, const void* logits, int64_t stride,
                              const uint8_t* is_probe, const float* temperature, const int32_t* top_k,
                              const float* top_p, const float* min_p, const float* draw_u, const uint8_t* row_active,
                              int32_t* token_out, int32_t* kept_count, float* prob_out, int32_t* dev_status,
                              rgd_stream_t stream) {
  clear_error();
  const char* fn = "rgd_sample_top";
  RGD_CHECK_ARG(rows >= 0, "%s: rows < 0", fn);
  RGD_CHECK_ARG(vocab >= 1, "%s: vocab < 1", fn);
  RGD_CHECK_ARG(dtype == RGD_F32 || dtype == RGD_BF16, "%s: dtype must be RGD_F32 or RGD_BF16", fn);
  RGD_CHECK_ARG(stride >= vocab, "%s: stride is below vocab", fn);
  if (rows == 0) return RGD_OK;
  RGD_CHECK_ARG(logits && temperature && draw_u && token_out, "%s: logits/temperature/draw_u/token_out must be non-NULL", fn);
  RGD_CHECK_ARG(aligned16(logits), "%s: logits must be 16-byte aligned", fn);
  // (sums of a row's weights stay below 2^52 then, and are exact in FP64)
  if (vocab > 1 << 20) return set_error(RGD_ERR_UNSUPPORTED, "%s: vocab %d too large (max %d)", fn, vocab, 1 << 20);
  if (rows > 0x7fffffff / kTopCluster) return set_error(RGD_ERR_UNSUPPORTED, "%s: too many rows", fn);
  const int es = dtype == RGD_F32 ? 4 : 2;
  TopParams p{};
  p.logits = static_cast<const uint8_t*>(logits);
  p.stride = stride * es;
  p.rows = rows;
  p.vocab = vocab;
  p.is_probe = is_probe;
  p.temperature = temperature;
  p.top_k = top_k;
  p.top_p = top_p;
  p.min_p = min_p;
  p.draw_u = draw_u;
  p.row_active = row_active;
  p.token_out = token_out;
  p.kept_count = kept_count;
  p.prob_out = prob_out;
  p.dev_status = dev_status;
  cudaStream_t st = (cudaStream_t)stream;
  const bool aligned = p.stride % 16 == 0;
  if (dtype == RGD_F32) return aligned ? launch_top<float, true>(p, st) : launch_top<float, false>(p, st);
  return aligned ? launch_top<__nv_bfloat16, true>(p, st) : launch_top<__nv_bfloat16, false>(p, st);
}
