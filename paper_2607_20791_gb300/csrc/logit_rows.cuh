// Rows of logits as the kernels that draw from them read them: a warp's contiguous share of a
// row as 16-byte vectors, what a lane remembers of its part, and sums of token weights that
// are exact in any order.
#pragma once

#include <cuda_bf16.h>

#include <cstdint>

#include "ptx.cuh"

namespace rgd {

constexpr int kGroups = 16;  // groups of a lane's vectors whose maxima it keeps
// Loads in flight per lane: a vector of a row off 16 bytes is five.
template <bool kAligned>
constexpr int kFlight = kAligned ? 8 : 4;

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

// A lane's sum of whole(w), exact for up to 2^16 numbers.  They go in two halves, w = a 2^-15 +
// r with a the nearest whole number, and w 2^31 = a 2^16 + r 2^31, both read off the bits
// of a sum (2^23, and 1.5 2^23 for r's sign).  Conversions to integers would take the
// special function unit's time, which the exponentials need.
struct WholeSum {
  uint32_t a = 0, b = 0, pairs = 0;
  __device__ void add(uint64_t w2) {
    const uint64_t h = fma2(w2, pair(0x1p15f, 0x1p15f), pair(0x1p23f, 0x1p23f));
    const uint64_t n = add2(h, pair(-0x1p23f, -0x1p23f));
    const uint64_t r = fma2(n, pair(-0x1p-15f, -0x1p-15f), w2);
    const uint64_t l = fma2(r, pair(0x1p31f, 0x1p31f), pair(0x1.8p23f, 0x1.8p23f));
    a += (uint32_t)h + (uint32_t)(h >> 32);
    b += (uint32_t)l + (uint32_t)(l >> 32);
  }
  __device__ void count(int n) { pairs += n; }  // of the calls of add()
  __device__ uint64_t total() const {
    const uint32_t high = a - pairs * (2u * 0x4b000000u), low = b - pairs * (2u * 0x4b400000u);
    return ((uint64_t)high << 16) + (uint64_t)(int64_t)(int32_t)low;
  }
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
  __device__ static uint4 nothing() { return make_uint4(0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u); }
  __device__ static Max max_of(const uint4& w, Max m) {
    return fmaxf(fmaxf(fmaxf(fmaxf(m, __uint_as_float(w.x)), __uint_as_float(w.y)), __uint_as_float(w.z)), __uint_as_float(w.w));
  }
  __device__ static Max max_of(Max a, Max b, Max c) { return fmaxf(fmaxf(a, b), c); }
  __device__ static float value(Max m) { return m; }
  __device__ static __nv_bfloat162 up(Max a, Max b) { return {__float2bfloat16_ru(a), __float2bfloat16_ru(b)}; }
  __device__ static bool reaches(Max m, const Bound& b) { return m >= b.v; }
  __device__ static void get(const uint4& w, int i, float& a, float& b) {
    a = __uint_as_float(i ? w.z : w.x);
    b = __uint_as_float(i ? w.w : w.y);
  }
  // The same, those below a bound (and NaN) as -inf.
  __device__ static void get_from(const uint4& w, int i, const Bound& c, float& a, float& b) {
    get(w, i, a, b);
    a = a >= c.v ? a : -INFINITY;
    b = b >= c.v ? b : -INFINITY;
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
  __device__ static uint4 nothing() { return make_uint4(0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u); }
  __device__ static Max max_of(const uint4& w, Max m) {  // (NaN never wins, as with fmaxf)
    return __hmax2(__hmax2(__hmax2(b2(w.x), b2(w.y)), __hmax2(b2(w.z), b2(w.w))), m);
  }
  __device__ static Max max_of(Max a, Max b, Max c) { return __hmax2(__hmax2(a, b), c); }
  __device__ static __nv_bfloat162 up(Max a, Max b) {  // the larger half of each
    return __hmax2(__lows2bfloat162(a, b), __highs2bfloat162(a, b));
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
  __device__ static void get_from(const uint4& w, int i, const Bound& c, float& a, float& b) {
    uint32_t u = i == 0 ? w.x : i == 1 ? w.y : i == 2 ? w.z : w.w;
    const uint32_t m = __hge2_mask(b2(u), c.v);
    u = (u & m) | (0xff80ff80u & ~m);
    a = __uint_as_float(u << 16);
    b = __uint_as_float(u & 0xffff0000u);
  }
};

// Sum over the warp of numbers below 2^54, in two halves.
__device__ __forceinline__ uint64_t warp_sum(uint64_t v) {
  const uint32_t low = __reduce_add_sync(0xffffffffu, (uint32_t)v & 0x7ffffffu);
  return low + ((uint64_t)__reduce_add_sync(0xffffffffu, (uint32_t)(v >> 27)) << 27);
}
__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}

// A warp's share of a row in global memory, as vectors of E elements from its first on: those
// read whole, and the last one element by element where the row does not end with it (or
// does not start on 16 bytes: then every vector comes as the 4-byte words it lies in, and
// a whole one's last word may reach past the row).
template <typename T, bool kAligned>
struct Share {
  static constexpr int E = 16 / (int)sizeof(T);
  const uint8_t* at;
  int32_t n, whole;
  __device__ Share(const uint8_t* row, int64_t e0, int64_t count) {
    n = (int32_t)max(int64_t(0), count);
    at = n ? row + e0 * (int64_t)sizeof(T) : row;
    whole = kAligned ? n / E : n ? (n - 1) / E : 0;
  }
  __device__ uint4 get(int i) const {
    const uint8_t* p = at + (int64_t)i * 16;
    if (kAligned) return __ldg(reinterpret_cast<const uint4*>(p));
    uint32_t u[5];
    const uint32_t off = (uint32_t)(reinterpret_cast<uintptr_t>(p) & 3);
    const uint32_t* w = reinterpret_cast<const uint32_t*>(p - off);
#pragma unroll
    for (int k = 0; k < 4; ++k) u[k] = __ldg(w + k);
    u[4] = E == 8 && off ? __ldg(w + 4) : 0;  // (only where it holds an element of the vector)
    if (E == 4) return make_uint4(u[0], u[1], u[2], u[3]);
    return make_uint4(__funnelshift_r(u[0], u[1], 8 * off), __funnelshift_r(u[1], u[2], 8 * off),
                      __funnelshift_r(u[2], u[3], 8 * off), __funnelshift_r(u[3], u[4], 8 * off));
  }
  // The last vector, in the lane whose turn it is; elements past the row's end read as -inf.
  __device__ uint4 rest(int lane) const {
    uint4 w = Vec<T>::nothing();
    if (n == whole * E || (whole & 31) != lane) return w;
    uint32_t* u = &w.x;
#pragma unroll
    for (int k = 0; k < E; ++k) {
      if (whole * E + k >= n) continue;
      const uint8_t* p = at + (int64_t)(whole * E + k) * (int)sizeof(T);
      if (E == 4) u[k] = __ldg(reinterpret_cast<const uint32_t*>(p));
      else u[k >> 1] = __byte_perm(u[k >> 1], __ldg(reinterpret_cast<const uint16_t*>(p)), (k & 1) ? 0x5410 : 0x3254);
    }
    return w;
  }
};

// What a lane keeps of its part of a share: the maxima of its groups (group g: its vectors
// of stripes g, g + kGroups, ...) rounded up to bf16, two to a word, and the last vector.
struct Kept {
  uint32_t group[kGroups / 2];
  uint4 rest;
};

// The lane's own maximum; find_maxima: the warp's.
template <typename T, bool kAligned>
__device__ __forceinline__ float find_lane_maxima(const Share<T, kAligned>& v, Kept& kept, int stripes, int lane) {
  using V = Vec<T>;
  kept.rest = v.rest(lane);
  typename V::Max all = V::max_of(kept.rest, V::lowest());
#pragma unroll
  for (int g = 0; g < kGroups / 2; ++g) kept.group[g] = 0xff80ff80u;
#pragma unroll 1
  for (int s = 0; s < stripes; s += kGroups) {
#pragma unroll
    for (int g = 0; g < kGroups; g += kFlight<kAligned>) {
      if (s + g >= stripes) break;
      uint4 w[kFlight<kAligned>];
#pragma unroll
      for (int k = 0; k < kFlight<kAligned>; ++k) {
        const int i = (s + g + k) * 32 + lane;
        w[k] = V::nothing();
        if (i < v.whole) w[k] = v.get(i);
      }
#pragma unroll
      for (int k = 0; k < kFlight<kAligned>; k += 2) {
        const typename V::Max m0 = V::max_of(w[k], V::lowest()), m1 = V::max_of(w[k + 1], V::lowest());
        all = V::max_of(m0, m1, all);
        const __nv_bfloat162 m = __hmax2(V::up(m0, m1), *reinterpret_cast<const __nv_bfloat162*>(&kept.group[(g + k) / 2]));
        kept.group[(g + k) / 2] = *reinterpret_cast<const uint32_t*>(&m);
      }
    }
  }
  return V::value(all);
}
template <typename T, bool kAligned>
__device__ __forceinline__ float find_maxima(const Share<T, kAligned>& v, Kept& kept, int stripes, int lane) {
  return warp_max(find_lane_maxima(v, kept, stripes, lane));
}

// Walks a lane's vectors of the groups in `mask`; next() gives -1 after the last.
struct Walk {
  uint32_t mask;
  int stripes, whole, lane, s;
  __device__ Walk(uint32_t mask, int stripes, int whole, int lane)
      : mask(mask), stripes(stripes), whole(whole), lane(lane) {
    s = __ffs(mask) - 1;
  }
  __device__ int next() {
    while (mask) {
      const int i = s * 32 + lane;
      s += kGroups;
      if (s >= stripes) {
        mask &= mask - 1;
        s = mask ? __ffs(mask) - 1 : 0;
      }
      if (i < whole) return i;
    }
    return -1;
  }
};

// The groups whose maximum may reach a bound.
__device__ __forceinline__ uint32_t groups_reaching(const Kept& kept, float bound) {
  const __nv_bfloat162 b = __bfloat162bfloat162(__float2bfloat16_ru(bound));  // (bf16 maxima: see Vec's Bound)
  uint32_t mask = 0;
#pragma unroll
  for (int g = 0; g < kGroups; g += 2)
    mask |= (__hge2_mask(*reinterpret_cast<const __nv_bfloat162*>(&kept.group[g / 2]), b) & 0x00020001u) << g;
  return (mask | mask >> 16) & ((1u << kGroups) - 1);
}

// The kept weights of a vector, added to a sum (NaN and -inf have none).
template <typename T>
__device__ __forceinline__ void add_weights(const uint4& w, const Side& side, const typename Vec<T>::Bound& cut, WholeSum& sum) {
  using V = Vec<T>;
  const uint64_t top = pair(-side.top, -side.top), kexp = pair(side.kexp, side.kexp);
#pragma unroll
  for (int e = 0; e < V::kPairs; ++e) {
    float a, b;
    V::get_from(w, e, cut, a, b);
    unpair(mul2(add2(pair(a, b), top), kexp), a, b);
    sum.add(pair(ex2_approx(a), ex2_approx(b)));
  }
  sum.count(V::kPairs);
}

// The sum of a warp's weights, in whole multiples of 2^-31.
template <typename T, bool kAligned>
__device__ __forceinline__ uint64_t sum_weights(const Share<T, kAligned>& v, const Kept& kept, const Side& side, int stripes,
                                                int lane) {
  using V = Vec<T>;
  const typename V::Bound cut(side.cut);
  const uint32_t mask = groups_reaching(kept, side.cut);
  WholeSum sum;
  uint4 w = kept.rest;
  // (a step of the walk below costs about 1.7 vectors in order, and the warp takes as many as
  // its busiest lane)
  const int steps = (int)__reduce_max_sync(0xffffffffu, (uint32_t)__popc(mask)) * ((stripes + kGroups - 1) / kGroups);
  if (7 * steps > 4 * stripes) {  // all of the share, in order
#pragma unroll 1
    for (int i = lane; i < v.whole; i += 32 * kFlight<kAligned>) {
      uint4 x[kFlight<kAligned>];
#pragma unroll
      for (int k = 0; k < kFlight<kAligned>; ++k) {
        x[k] = V::nothing();
        if (i + 32 * k < v.whole) x[k] = v.get(i + 32 * k);
      }
#pragma unroll
      for (int k = 0; k < kFlight<kAligned>; ++k) add_weights<T>(x[k], side, cut, sum);
    }
    add_weights<T>(w, side, cut, sum);
  } else {  // the groups that reach the cutoff, two vectors on their way while one is worked on
    Walk walk(mask, stripes, v.whole, lane);
    uint4 w1 = V::nothing(), w2 = w1;
    int i1 = walk.next(), i2 = walk.next();
    if (i1 >= 0) w1 = v.get(i1);
    if (i2 >= 0) w2 = v.get(i2);
#pragma unroll 1
    for (;;) {
      const int i3 = walk.next();
      uint4 w3 = V::nothing();
      if (i3 >= 0) w3 = v.get(i3);
      add_weights<T>(w, side, cut, sum);
      if (i1 < 0) break;
      w = w1, w1 = w2, w2 = w3;
      i1 = i2, i2 = i3;
    }
  }
  return warp_sum(sum.total());
}

// The address of another CTA's shared memory in the cluster.
__device__ __forceinline__ uint32_t peer_addr(uint32_t addr, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
  return r;
}

}  // namespace rgd
