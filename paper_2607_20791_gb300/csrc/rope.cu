// Rotary positions, with the norms of each head in the same pass.  A head x of D values is
// first scaled by w / sqrt(mean(x^2) + eps) (where norms are asked for), then each pair (a, b)
// of its first `rotary_dim` values becomes m (a cos t - b sin t, b cos t + a sin t), where t is
// the pair's frequency times the token's position.  Pairs lie side by side or half the
// rotated part apart.
//
// Angles.  A frequency is a fraction of a turn in 64 bits, so the position times it, modulo
// 2^64, is the angle modulo one turn without any loss, however far the position (an fp32 angle
// of 500000 radians is good to 0.016).  Its top 32 bits go to sincospif as an fp32, rounded by
// 2^-26 of a turn (1e-7 radians) at most.
//
// Bound by bytes: every value is read once and written once.  A lane holds two vectors of E
// values whose pairs it can turn by itself: side by side for adjacent pairs, half the rotated
// part apart for halves.  A head is D / 2E lanes, a warp works on as many heads at once as
// fit, and a lane keeps its cosines and sines for all the heads of the token.  Few tokens are
// spread over more warps, each with a share of the heads (and sines of its own).
//
// Measured: 16384 tokens of 32 + 8 heads of 128, normed, bf16: 62 us, 5.4 TB/s, 0.80 of what a
// copy reaches, fp32 103 us, 6.5 TB/s (0.96); 16384 tokens of 32 + 8 + 8 heads, half turned, keys and
// values into pages: 69 us, 4.8 TB/s (0.71).  Four loads a lane on their way are what that takes (three 63 us, two 62 to 65,
// one 78), and the registers that the compiler wants for them: held to 102 for a fifth CTA on an
// SM the prompt takes 62 us and the pages 76, held to 80 for a sixth 66 and 83.  Single steps are
// latency: 80 rows 3.7 us.
#include <cuda_bf16.h>

#include <algorithm>
#include <cmath>

#include "cache.h"
#include "common.h"
#include "ptx.cuh"

namespace rgd {
namespace {

constexpr int kRopeWarps = 4;
constexpr int kInFlight = 4;  // passes whose loads are on their way together

struct RopeParams {
  const uint8_t* in[3];  // queries, keys, values (values: into pages only)
  int64_t in_row[3], in_token[3];  // bytes from a row, and from a token of it, to the next
  uint8_t* out[3];
  int64_t out_token[3];  // bytes (queries, and keys that do not go into pages)
  const void* weight[2];
  int32_t heads[3];
  int32_t passes[3];  // of a warp over the heads of each kind
  int32_t each;       // passes of one warp
  int32_t chunks;     // warps of a token
  int32_t dim, rot, slots, group;  // group: lanes of a head, a power of two
  int32_t norm, weight_f32, pairs;
  float eps, magnitude, inv_dim;
  int32_t tokens, rows;  // of a row; rows
  const int32_t* positions;
  const uint64_t* turns;
  // into pages
  const int32_t* first;
  const int32_t* n_new;
  const int32_t* table;
  const int32_t* length;
  const uint8_t* row_active;
  int32_t cols, pages;
  int32_t* dev_status;
};

template <int kBytes>
struct Raw;
template <>
struct Raw<16> {
  using type = uint4;
};
template <>
struct Raw<8> {
  using type = uint2;
};
template <>
struct Raw<4> {
  using type = uint32_t;
};
template <>
struct Raw<2> {
  using type = uint16_t;
};

// E values of type T in one register vector.
template <typename T, int E>
struct Values {
  using R = typename Raw<E * (int)sizeof(T)>::type;
  R v;
  __device__ void get(float (&x)[E]) const {
    const T* t = reinterpret_cast<const T*>(&v);
#pragma unroll
    for (int i = 0; i < E; ++i) x[i] = (float)t[i];
  }
  __device__ void set(const float (&x)[E]) {
    T* t = reinterpret_cast<T*>(&v);
#pragma unroll
    for (int i = 0; i < E; ++i) t[i] = (T)x[i];
  }
};

// (of a token by itself)
__device__ __forceinline__ void turn(float& a, float& b, float c, float s) {
  const float x = a;
  a = fmaf(x, c, -b * s);
  b = fmaf(b, c, x * s);
}

// Where token i of row r goes: its position and its first byte in a page; false if nowhere.
__device__ __forceinline__ bool place(const RopeParams& p, int32_t r, int32_t i, bool tell, int64_t& pos, int64_t& at) {
  const int32_t n = p.n_new[r], len = p.length[r];
  if (p.row_active && !p.row_active[r]) return false;
  if (tell && i == 0 && (n < 0 || n > p.tokens) && p.dev_status) atomicOr(p.dev_status, RGD_DEV_BAD_PAGE);
  if (i >= n) return false;
  const int64_t t = (int64_t)len + i;
  const int32_t page = t >= 0 && t < (int64_t)p.cols * kPageSize ? p.table[(int64_t)r * p.cols + t / kPageSize] : -1;
  if (page < 0 || page >= p.pages) {
    if (tell && p.dev_status) atomicOr(p.dev_status, RGD_DEV_BAD_PAGE);
    return false;
  }
  pos = t + (p.first ? p.first[r] : 0);
  at = ((int64_t)page * p.heads[1] * kPageSize + t % kPageSize) * p.dim;
  return true;
}

__device__ __forceinline__ float weight_at(const RopeParams& p, const void* w, int i) {
  return p.weight_f32 ? static_cast<const float*>(w)[i] : (float)static_cast<const __nv_bfloat16*>(w)[i];
}

// Angle of a pair at a position, in half turns of [-1, 1).
__device__ __forceinline__ float half_turns(const RopeParams& p, int64_t pos, int pair) {
  const uint64_t t = (uint64_t)pos * p.turns[pair];
  return (float)(int32_t)(t >> 32) * 0x1p-31f;
}

__device__ __forceinline__ uint64_t both(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void each_of(uint64_t v, float& a, float& b) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v));
}
__device__ __forceinline__ uint64_t mul_both(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t fma_both(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}

// kAcross: pair j of a lane is (u[j], v[j]) of its two vectors u, v; else u's values are E / 2
// pairs, side by side, and v's as many more.
template <typename T, int E, bool kAcross>
__device__ __forceinline__ void pairs_of(const Values<T, E>& u, const Values<T, E>& v, float (&a)[E], float (&b)[E]) {
  float x[E], y[E];
  u.get(x);
  v.get(y);
#pragma unroll
  for (int j = 0; j < E; ++j) {
    a[j] = kAcross ? x[j] : j < E / 2 ? x[2 * j] : y[2 * j - E];
    b[j] = kAcross ? y[j] : j < E / 2 ? x[2 * j + 1] : y[2 * j - E + 1];
  }
}
template <typename T, int E, bool kAcross>
__device__ __forceinline__ void put_pairs(Values<T, E>& u, Values<T, E>& v, const float (&a)[E], const float (&b)[E]) {
  float x[E], y[E];
#pragma unroll
  for (int j = 0; j < E; ++j) {
    (kAcross ? x[j] : j < E / 2 ? x[2 * j] : y[2 * j - E]) = a[j];
    (kAcross ? y[j] : j < E / 2 ? x[2 * j + 1] : y[2 * j - E + 1]) = b[j];
  }
  u.set(x);
  v.set(y);
}

// A lane's pairs as coefficients: (a, b) becomes by (a ca - b sb, b cb + a sa), the norm's weights
// times the cosine and sine; `by` is the norm's factor.  Two pairs to an instruction.
template <int E>
struct Turns {
  static constexpr int N = E > 1 ? E / 2 : 1;
  uint64_t ca[N], sa[N], cb[N], sb[N];  // (sb negative)
};

template <typename T, int E, bool kAcross, bool kPages>
__global__ void __launch_bounds__(kRopeWarps * 32) rope_kernel(const RopeParams p) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");  // (a dependent waits for this kernel's end)
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int lane = threadIdx.x & 31, chunk = (int)blockIdx.y;
  const uint32_t t = blockIdx.x * kRopeWarps + (threadIdx.x >> 5);  // token
  const uint32_t r = kPages ? t / (uint32_t)p.tokens : t >= (uint32_t)p.tokens, i = kPages ? t - r * (uint32_t)p.tokens : t;
  if (r >= (uint32_t)p.rows) return;
  const int per = 32 / p.group, sub = lane / p.group, slot = lane & (p.group - 1);
  const bool on = slot < p.slots;
  const int half_slots = p.pairs ? 0 : p.rot / (2 * E);
  const int o0 = slot < half_slots ? slot * E : slot * 2 * E;  // the lane's two vectors
  const int o1 = slot < half_slots ? o0 + p.rot / 2 : o0 + E;
  const int turned = on ? p.rot / 2 - slot * E : 0;  // of the lane's pairs
  // Passes of one kind together, from `first` on: the first ones' loads are under way while the page is
  // looked up and the angles are worked out.
  const int last = min((chunk + 1) * p.each, p.passes[0] + p.passes[1] + p.passes[2]);
  int kind = 0, count = 0, h0 = 0;
  Values<T, E> u[kInFlight], v[kInFlight];
  auto load = [&](int first) {
    int q = first;
    for (kind = 0; q >= p.passes[kind];) q -= p.passes[kind++];
    count = min(min(last - first, p.passes[kind] - q), kInFlight);
    h0 = q * per + sub;
    const T* from = reinterpret_cast<const T*>(p.in[kind] + r * p.in_row[kind] + i * p.in_token[kind]) + h0 * p.dim;
#pragma unroll
    for (int k = 0; k < kInFlight; ++k) {
      if (k < count && on && h0 + k * per < p.heads[kind]) {
        u[k].v = *reinterpret_cast<const typename Values<T, E>::R*>(from + k * per * p.dim + o0);
        v[k].v = *reinterpret_cast<const typename Values<T, E>::R*>(from + k * per * p.dim + o1);
      }
    }
  };
  load(chunk * p.each);
  int64_t pos, page_at = 0;
  if (kPages) {
    if (!place(p, (int32_t)r, (int32_t)i, chunk == 0 && lane == 0, pos, page_at)) return;
  } else {
    pos = p.positions[t];
  }
  float c[E], s[E];
  if (E == 8 && p.group == 8 && p.rot == 128) {
    // Four heads of 128 at once: every pair's angle is wanted by four lanes, each works out two of its eight.
    float c2[2], s2[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) sincospif(half_turns(p, pos, slot * E + sub * 2 + j), &s2[j], &c2[j]);
#pragma unroll
    for (int j = 0; j < E; ++j) {
      c[j] = __shfl_sync(0xffffffffu, c2[j & 1], (j >> 1) * 8 + slot) * p.magnitude;
      s[j] = __shfl_sync(0xffffffffu, s2[j & 1], (j >> 1) * 8 + slot) * p.magnitude;
    }
  } else {
#pragma unroll
    for (int j = 0; j < E; ++j) {
      c[j] = 1.f;
      s[j] = 0.f;
      if (j < turned) {
        sincospif(half_turns(p, pos, slot * E + j), &s[j], &c[j]);
        c[j] *= p.magnitude;
        s[j] *= p.magnitude;
      }
    }
  }
  Turns<E> by_pair;
  int kind_of_weights = -1;
#pragma unroll 1
  for (int first = chunk * p.each; first < last;) {
    if (kind < 2 && kind != kind_of_weights) {
      kind_of_weights = kind;
      float wa[E], wb[E];
#pragma unroll
      for (int j = 0; j < E; ++j) {
        wa[j] = wb[j] = 1.f;
        if (p.norm && on && p.weight[kind]) {
          wa[j] = weight_at(p, p.weight[kind], kAcross ? o0 + j : o0 + 2 * j);
          wb[j] = weight_at(p, p.weight[kind], kAcross ? o1 + j : o0 + 2 * j + 1);
        }
      }
      if (E > 1) {
#pragma unroll
        for (int j = 0; j < E / 2; ++j) {
          const int x = 2 * j, y = E > 1 ? 2 * j + 1 : 0;
          by_pair.ca[j] = both(wa[x] * c[x], wa[y] * c[y]);
          by_pair.sa[j] = both(wa[x] * s[x], wa[y] * s[y]);
          by_pair.cb[j] = both(wb[x] * c[x], wb[y] * c[y]);
          by_pair.sb[j] = both(-wb[x] * s[x], -wb[y] * s[y]);
        }
      } else {
        by_pair.ca[0] = both(wa[0] * c[0], 0.f);
        by_pair.sa[0] = both(wa[0] * s[0], 0.f);
        by_pair.cb[0] = both(wb[0] * c[0], 0.f);
        by_pair.sb[0] = both(-wb[0] * s[0], 0.f);
      }
    }
    T* to = kPages && kind > 0 ? reinterpret_cast<T*>(p.out[kind]) + page_at + (int64_t)h0 * kPageSize * p.dim
                               : reinterpret_cast<T*>(p.out[kind] + t * p.out_token[kind]) + h0 * p.dim;
    const int64_t step = (int64_t)per * p.dim * (kPages && kind > 0 ? kPageSize : 1);
#pragma unroll
    for (int k = 0; k < kInFlight; ++k) {
      if (k >= count) break;
      const bool mine = on && h0 + k * per < p.heads[kind];
      if (kind < 2) {
        float a[E], b[E];
        pairs_of<T, E, kAcross>(u[k], v[k], a, b);
        uint64_t a2[Turns<E>::N], b2[Turns<E>::N];
#pragma unroll
        for (int j = 0; j < Turns<E>::N; ++j) {
          a2[j] = both(a[E > 1 ? 2 * j : 0], E > 1 ? a[E > 1 ? 2 * j + 1 : 0] : 0.f);
          b2[j] = both(b[E > 1 ? 2 * j : 0], E > 1 ? b[E > 1 ? 2 * j + 1 : 0] : 0.f);
        }
        float by = 1.f;
        if (p.norm) {
          uint64_t squares = 0;
#pragma unroll
          for (int j = 0; j < Turns<E>::N; ++j) squares = fma_both(a2[j], a2[j], fma_both(b2[j], b2[j], squares));
          float sum, high;
          each_of(squares, sum, high);
          sum = mine ? sum + high : 0.f;
          for (int o = p.group / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
          by = rsqrtf(fmaf(sum, p.inv_dim, p.eps));
        }
        const uint64_t by2 = both(by, by);
        if (turned >= E) {
#pragma unroll
          for (int j = 0; j < Turns<E>::N; ++j) {
            const uint64_t x = fma_both(a2[j], by_pair.ca[j], mul_both(b2[j], by_pair.sb[j]));
            const uint64_t y = fma_both(b2[j], by_pair.cb[j], mul_both(a2[j], by_pair.sa[j]));
            float lo, hi;
            each_of(mul_both(x, by2), lo, hi);
            a[E > 1 ? 2 * j : 0] = lo;
            if (E > 1) a[E > 1 ? 2 * j + 1 : 0] = hi;
            each_of(mul_both(y, by2), lo, hi);
            b[E > 1 ? 2 * j : 0] = lo;
            if (E > 1) b[E > 1 ? 2 * j + 1 : 0] = hi;
          }
          put_pairs<T, E, kAcross>(u[k], v[k], a, b);
        } else if (turned > 0 || p.norm) {
          // (values behind the rotated part are not turned by 0: an infinity's partner would be NaN)
#pragma unroll
          for (int j = 0; j < E; ++j) {
            float ca, sa, cb, sb, other;
            each_of(by_pair.ca[j / 2], E > 1 && (j & 1) ? other : ca, E > 1 && (j & 1) ? ca : other);
            each_of(by_pair.sa[j / 2], E > 1 && (j & 1) ? other : sa, E > 1 && (j & 1) ? sa : other);
            each_of(by_pair.cb[j / 2], E > 1 && (j & 1) ? other : cb, E > 1 && (j & 1) ? cb : other);
            each_of(by_pair.sb[j / 2], E > 1 && (j & 1) ? other : sb, E > 1 && (j & 1) ? sb : other);
            const float x = j < turned ? fmaf(a[j], ca, b[j] * sb) : a[j] * ca;
            const float y = j < turned ? fmaf(b[j], cb, a[j] * sa) : b[j] * cb;
            a[j] = x * by;
            b[j] = y * by;
          }
          put_pairs<T, E, kAcross>(u[k], v[k], a, b);
        }
      }
      if (!mine) continue;
      *reinterpret_cast<typename Values<T, E>::R*>(to + k * step + o0) = u[k].v;
      *reinterpret_cast<typename Values<T, E>::R*>(to + k * step + o1) = v[k].v;
    }
    first += count;
    if (first < last) load(first);
  }
}

// Any head, value by value: a warp for each head of a token.  (Odd sizes, rows off 4 bytes,
// heads too long for a lane to hold 1/32 of them in two vectors.)  A lane turns whole pairs,
// and reads them before it writes them, so that the output may be the input.
template <typename T, bool kPages>
__global__ void __launch_bounds__(kRopeWarps * 32) rope_any_kernel(const RopeParams p) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int lane = threadIdx.x & 31;
  const int64_t w = (int64_t)blockIdx.x * kRopeWarps + (threadIdx.x >> 5);
  const int heads = p.heads[0] + p.heads[1] + p.heads[2];
  const int64_t t = w / heads;
  int h = (int)(w - t * heads), kind = 0;
  const int32_t r = (int32_t)(t / p.tokens), i = (int32_t)(t - (int64_t)r * p.tokens);
  if (r >= p.rows) return;
  int64_t pos, page_at = 0;
  if (kPages) {
    if (!place(p, r, i, h == 0 && lane == 0, pos, page_at)) return;
  } else {
    pos = p.positions[t];
  }
  while (h >= p.heads[kind]) h -= p.heads[kind++];
  const T* x = reinterpret_cast<const T*>(p.in[kind] + r * p.in_row[kind] + i * p.in_token[kind]) + (int64_t)h * p.dim;
  T* to = kPages && kind > 0 ? reinterpret_cast<T*>(p.out[kind]) + page_at + (int64_t)h * kPageSize * p.dim
                             : reinterpret_cast<T*>(p.out[kind] + t * p.out_token[kind]) + (int64_t)h * p.dim;
  const void* weight = kind < 2 ? p.weight[kind] : nullptr;
  float by = 1.f;
  if (p.norm && kind < 2) {
    float sum = 0.f;
    for (int j = lane; j < p.dim; j += 32) sum = fmaf((float)x[j], (float)x[j], sum);
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    by = rsqrtf(fmaf(sum, p.inv_dim, p.eps));
  }
  auto value = [&](int j) {
    const float v = (float)x[j];
    return p.norm && kind < 2 ? v * (weight ? by * weight_at(p, weight, j) : by) : v;
  };
  const int half = kind < 2 ? p.rot / 2 : 0;
  for (int pair = lane; pair < half; pair += 32) {
    const int j = p.pairs ? 2 * pair : pair, k = p.pairs ? j + 1 : j + half;
    float a = value(j), b = value(k), c, s;
    sincospif(half_turns(p, pos, pair), &s, &c);
    turn(a, b, c * p.magnitude, s * p.magnitude);
    to[j] = (T)a;
    to[k] = (T)b;
  }
  for (int j = 2 * half + lane; j < p.dim; j += 32) to[j] = (T)value(j);
}

template <typename T, int E, bool kPages>
cudaError_t launch_vectors(RopeParams& p, cudaStream_t st) {
  p.slots = p.dim / (2 * E);
  p.group = 1;
  while (p.group < p.slots) p.group *= 2;
  const int per = 32 / p.group;
  int passes = 0;
  for (int k = 0; k < 3; ++k) passes += p.passes[k] = (p.heads[k] + per - 1) / per;
  // A warp takes all of a token's heads where that leaves enough warps for the SMs.
  const int64_t tokens = (int64_t)p.rows * p.tokens, wanted = 152 * 32;
  p.chunks = (int)std::min<int64_t>(passes, std::max<int64_t>(1, (wanted + tokens - 1) / tokens));
  p.each = (passes + p.chunks - 1) / p.chunks;
  p.chunks = (passes + p.each - 1) / p.each;
  const bool across = !p.pairs || E == 1;
  auto k = across ? rope_kernel<T, E, true, kPages> : rope_kernel<T, E, E == 1, kPages>;
  return launch_dependent(k, dim3((unsigned)((tokens + kRopeWarps - 1) / kRopeWarps), (unsigned)p.chunks), kRopeWarps * 32, 0, st, p);
}

template <typename T, bool kPages>
int launch_rope(const char* fn, RopeParams& p, cudaStream_t st) {
  // The widest vectors, up to 16 bytes, that the addresses, the strides and the layout allow.
  uint64_t bits = 0;
  for (int k = 0; k < 3; ++k) {
    if (!p.heads[k]) continue;
    bits |= reinterpret_cast<uintptr_t>(p.in[k]) | reinterpret_cast<uintptr_t>(p.out[k]) | (uint64_t)p.out_token[k] |
            (uint64_t)p.in_row[k] | (uint64_t)p.in_token[k];
  }
  bits |= (uint64_t)p.dim * sizeof(T);
  int e = 16 / (int)sizeof(T);
  while (e > 1 && (bits % (e * sizeof(T)) != 0 || p.dim % (2 * e) != 0 || (!p.pairs && (p.rot / 2) % e != 0))) e /= 2;
  const int64_t tokens = (int64_t)p.rows * p.tokens, heads = (int64_t)p.heads[0] + p.heads[1] + p.heads[2];
  if (tokens * heads > 0x7fffffffll * kRopeWarps) return set_error(RGD_ERR_UNSUPPORTED, "%s: too many tokens", fn);
  cudaError_t err;
  if (p.dim % 2 != 0 || p.dim / (2 * e) > 32) {
    const int64_t blocks = (tokens * heads + kRopeWarps - 1) / kRopeWarps;
    err = launch_dependent(rope_any_kernel<T, kPages>, (int)blocks, kRopeWarps * 32, 0, st, p);
  } else if (e == 8) {
    err = launch_vectors<T, sizeof(T) == 2 ? 8 : 4, kPages>(p, st);
  } else if (e == 4) {
    err = launch_vectors<T, 4, kPages>(p, st);
  } else if (e == 2) {
    err = launch_vectors<T, 2, kPages>(p, st);
  } else {
    err = launch_vectors<T, 1, kPages>(p, st);
  }
  return err == cudaSuccess ? RGD_OK : cuda_error(err, "rope launch");
}

constexpr int kMostHeads = 4096, kMostDim = 1024;

int check_rope(const char* fn, const rgd_rope_shape* s, const uint64_t* turns, int32_t weight_dtype, RopeParams& p) {
  RGD_CHECK_ARG(s, "%s: shape is NULL", fn);
  RGD_CHECK_ARG(s->num_q_heads >= 0 && s->num_k_heads >= 0, "%s: heads must not be negative", fn);
  RGD_CHECK_ARG(s->head_dim >= 1, "%s: head_dim < 1", fn);
  RGD_CHECK_ARG(s->rotary_dim >= 0 && s->rotary_dim <= s->head_dim && s->rotary_dim % 2 == 0,
                "%s: rotary_dim must be even and in [0, head_dim]", fn);
  RGD_CHECK_ARG(s->layout == RGD_ROPE_HALF || s->layout == RGD_ROPE_PAIRS, "%s: layout must be RGD_ROPE_HALF or RGD_ROPE_PAIRS", fn);
  RGD_CHECK_ARG(s->norm == 0 || s->norm == 1, "%s: norm must be 0 or 1", fn);
  RGD_CHECK_ARG(!s->norm || (s->eps >= 0.f && s->eps < INFINITY), "%s: eps must be finite and not negative", fn);
  RGD_CHECK_ARG(std::fabs(s->magnitude) < INFINITY, "%s: magnitude must be finite", fn);
  RGD_CHECK_ARG(!s->norm || weight_dtype == RGD_F32 || weight_dtype == RGD_BF16, "%s: weight_dtype must be RGD_F32 or RGD_BF16", fn);
  if (s->num_q_heads > kMostHeads || s->num_k_heads > kMostHeads || s->head_dim > kMostDim)
    return set_error(RGD_ERR_UNSUPPORTED, "%s: more than %d heads or a head_dim above %d", fn, kMostHeads, kMostDim);
  RGD_CHECK_ARG(s->rotary_dim == 0 || turns, "%s: turns must be non-NULL", fn);
  RGD_CHECK_ARG((reinterpret_cast<uintptr_t>(turns) & 7u) == 0, "%s: turns must be 8-byte aligned", fn);
  p.heads[0] = s->num_q_heads;
  p.heads[1] = s->num_k_heads;
  p.dim = s->head_dim;
  p.rot = s->rotary_dim;
  p.pairs = s->layout == RGD_ROPE_PAIRS;
  p.norm = s->norm;
  p.eps = s->eps;
  p.magnitude = s->magnitude;
  p.inv_dim = 1.f / (float)s->head_dim;
  p.weight_f32 = weight_dtype == RGD_F32;
  p.turns = turns;
  return RGD_OK;
}

}  // namespace
}  // namespace rgd

using namespace rgd;

extern "C" int rgd_rope_frequencies(int32_t rotary_dim, double base, int32_t scaling, double factor, double trained_length,
                                    double low, double high, uint64_t* turns, double* magnitude) {
  clear_error();
  const char* fn = "rgd_rope_frequencies";
  RGD_CHECK_ARG(rotary_dim >= 0 && rotary_dim % 2 == 0, "%s: rotary_dim must be even and not negative", fn);
  RGD_CHECK_ARG(base >= 1 && base < INFINITY, "%s: base must be finite and at least 1", fn);
  RGD_CHECK_ARG(scaling >= RGD_ROPE_PLAIN && scaling <= RGD_ROPE_RAMP, "%s: scaling is none of RGD_ROPE_*", fn);
  RGD_CHECK_ARG(scaling == RGD_ROPE_PLAIN || (factor >= 1 && factor < INFINITY), "%s: factor must be finite and at least 1", fn);
  const bool bands = scaling == RGD_ROPE_BANDS, ramp = scaling == RGD_ROPE_RAMP;
  RGD_CHECK_ARG(!(bands || ramp) || (trained_length > 0 && trained_length < INFINITY), "%s: trained_length must be positive", fn);
  RGD_CHECK_ARG(!(bands || ramp) || (low > 0 && high > low && high < INFINITY), "%s: low and high must be 0 < low < high", fn);
  RGD_CHECK_ARG(!ramp || base > 1, "%s: RGD_ROPE_RAMP needs a base above 1", fn);
  RGD_CHECK_ARG(rotary_dim == 0 || turns, "%s: turns must be non-NULL", fn);
  RGD_CHECK_ARG(magnitude, "%s: magnitude must be non-NULL", fn);
  constexpr double two_pi = 6.283185307179586;
  if (scaling == RGD_ROPE_BASE && rotary_dim > 2) base *= std::pow(factor, rotary_dim / (rotary_dim - 2.0));
  double from = 0, to = 0;
  if (ramp) {
    auto index = [&](double waves) { return rotary_dim * std::log(trained_length / (waves * two_pi)) / (2 * std::log(base)); };
    from = std::max(std::floor(index(high)), 0.0);
    to = std::min(std::ceil(index(low)), rotary_dim - 1.0);
  }
  for (int i = 0; i < rotary_dim / 2; ++i) {
    double f = std::pow(base, -2.0 * i / rotary_dim), keep = 1;
    if (scaling == RGD_ROPE_LINEAR) keep = 0;
    if (bands) keep = std::min(std::max((trained_length * f / two_pi - low) / (high - low), 0.0), 1.0);
    if (ramp) keep = 1 - std::min(std::max((i - from) / std::max(to - from, 0.001), 0.0), 1.0);
    if (scaling == RGD_ROPE_LINEAR || bands || ramp) f *= keep + (1 - keep) / factor;
    turns[i] = (uint64_t)(f / two_pi * 0x1p64);
  }
  *magnitude = ramp ? 0.1 * std::log(factor) + 1.0 : 1.0;
  return RGD_OK;
}

extern "C" int rgd_qk_rope(const rgd_rope_shape* shape, int32_t tokens, int32_t dtype, const void* q, int64_t q_stride,
                           const void* k, int64_t k_stride, const int32_t* positions, const uint64_t* turns,
                           int32_t weight_dtype, const void* q_weight, const void* k_weight, void* q_out,
                           int64_t q_out_stride, void* k_out, int64_t k_out_stride, int32_t* dev_status,
                           rgd_stream_t stream) {
  clear_error();
  const char* fn = "rgd_qk_rope";
  RopeParams p{};
  if (int rc = check_rope(fn, shape, turns, weight_dtype, p)) return rc;
  RGD_CHECK_ARG(tokens >= 0, "%s: tokens < 0", fn);
  RGD_CHECK_ARG(dtype == RGD_F32 || dtype == RGD_BF16, "%s: dtype must be RGD_F32 or RGD_BF16", fn);
  const int64_t qd = (int64_t)p.heads[0] * p.dim, kd = (int64_t)p.heads[1] * p.dim;
  RGD_CHECK_ARG(!p.heads[0] || (q_stride >= 0 && q_out_stride >= qd), "%s: q_stride is negative or q_out_stride below a token's queries", fn);
  RGD_CHECK_ARG(!p.heads[1] || (k_stride >= 0 && k_out_stride >= kd), "%s: k_stride is negative or k_out_stride below a token's keys", fn);
  if (tokens == 0 || p.heads[0] + p.heads[1] == 0) return RGD_OK;
  RGD_CHECK_ARG(positions && (!p.heads[0] || (q && q_out)) && (!p.heads[1] || (k && k_out)),
                "%s: positions/q/q_out/k/k_out must be non-NULL", fn);
  const int es = dtype == RGD_F32 ? 4 : 2;
  const void* base[4] = {q, k, q_out, k_out};
  for (int i = 0; i < 4; ++i)
    RGD_CHECK_ARG(!p.heads[i & 1] || reinterpret_cast<uintptr_t>(base[i]) % es == 0, "%s: tensors must be aligned to their elements", fn);
  const int64_t in[2] = {q_stride, k_stride}, out[2] = {q_out_stride, k_out_stride};
  const void* weight[2] = {q_weight, k_weight};
  for (int i = 0; i < 2; ++i) {
    p.in[i] = static_cast<const uint8_t*>(base[i]);
    p.out[i] = static_cast<uint8_t*>(const_cast<void*>(base[2 + i]));
    p.in_token[i] = in[i] * es;
    p.out_token[i] = out[i] * es;
    p.weight[i] = weight[i];
    RGD_CHECK_ARG(!p.norm || reinterpret_cast<uintptr_t>(weight[i]) % (p.weight_f32 ? 4 : 2) == 0, "%s: weights must be aligned to their elements", fn);
  }
  p.rows = 1;
  p.tokens = tokens;
  p.positions = positions;
  p.dev_status = dev_status;
  return dtype == RGD_F32 ? launch_rope<float, false>(fn, p, (cudaStream_t)stream)
                          : launch_rope<__nv_bfloat16, false>(fn, p, (cudaStream_t)stream);
}

extern "C" int rgd_qk_rope_cache(const rgd_rope_shape* shape, const rgd_cache_shape* cache, int32_t layer, int32_t rows,
                                 int32_t max_new, const rgd_bf16* q, const rgd_bf16* k, const rgd_bf16* v,
                                 int64_t row_stride, int64_t token_stride, const int32_t* first_position,
                                 const uint64_t* turns, int32_t weight_dtype, const void* q_weight,
                                 const void* k_weight, const int32_t* n_new, int32_t max_pages,
                                 const int32_t* block_table, const int32_t* length, const uint8_t* row_active,
                                 rgd_bf16* q_out, rgd_bf16* k_pages, rgd_bf16* v_pages, int32_t* dev_status,
                                 rgd_stream_t stream) {
  clear_error();
  const char* fn = "rgd_qk_rope_cache";
  CacheView c;
  if (int rc = check_cache_shape(fn, cache, c)) return rc;
  RopeParams p{};
  if (int rc = check_rope(fn, shape, turns, weight_dtype, p)) return rc;
  RGD_CHECK_ARG(p.heads[1] == c.heads && p.dim == c.dim, "%s: the two shapes differ in their key heads or head_dim", fn);
  RGD_CHECK_ARG(rows >= 0 && max_new >= 0 && max_pages >= 1, "%s: bad rows/max_new/max_pages", fn);
  RGD_CHECK_ARG(layer >= 0 && layer < c.layers, "%s: layer outside [0, num_layers)", fn);
  RGD_CHECK_ARG(row_stride >= 0 && token_stride >= 0, "%s: strides must not be negative", fn);
  if (rows == 0 || max_new == 0) return RGD_OK;
  RGD_CHECK_ARG((!p.heads[0] || (q && q_out)) && k && v && n_new && block_table && length && k_pages && v_pages,
                "%s: q/k/v/q_out/n_new/block_table/length/k_pages/v_pages must be non-NULL", fn);
  const void* weight[2] = {q_weight, k_weight};
  const rgd_bf16* in[3] = {q, k, v};
  rgd_bf16* out[3] = {q_out, k_pages + layer * c.layer_stride, v_pages + layer * c.layer_stride};
  p.heads[2] = c.heads;
  for (int i = 0; i < 3; ++i) {
    p.in[i] = reinterpret_cast<const uint8_t*>(in[i]);
    p.out[i] = reinterpret_cast<uint8_t*>(out[i]);
    p.in_row[i] = row_stride * 2;
    p.in_token[i] = token_stride * 2;
    RGD_CHECK_ARG(!p.heads[i] || ((reinterpret_cast<uintptr_t>(in[i]) | reinterpret_cast<uintptr_t>(out[i])) & 1u) == 0,
                  "%s: tensors must be aligned to their elements", fn);
    if (i == 2) break;
    p.weight[i] = weight[i];
    RGD_CHECK_ARG(!p.norm || reinterpret_cast<uintptr_t>(weight[i]) % (p.weight_f32 ? 4 : 2) == 0, "%s: weights must be aligned to their elements", fn);
  }
  RGD_CHECK_ARG(aligned16(k_pages) && aligned16(v_pages), "%s: the pools must be 16-byte aligned", fn);
  RGD_CHECK_ARG((int64_t)rows * max_new <= kMaxRows, "%s: too many tokens", fn);
  p.out_token[0] = (int64_t)p.heads[0] * p.dim * 2;
  p.rows = rows;
  p.tokens = max_new;
  p.first = first_position;
  p.n_new = n_new;
  p.table = block_table;
  p.length = length;
  p.row_active = row_active;
  p.cols = max_pages;
  p.pages = c.pages;
  p.dev_status = dev_status;
  return launch_rope<__nv_bfloat16, true>(fn, p, (cudaStream_t)stream);
}
