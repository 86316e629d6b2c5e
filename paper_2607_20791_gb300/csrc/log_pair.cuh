// The logarithm that a min-p cutoff needs, in pairs of floats.
#pragma once

#include <cmath>
#include <cstdint>

namespace rgd {
namespace {

// T ln p rounded once to fp32, p in [0, 1], T > 0: the same bits as (float)((double)T log((double)p)),
// which the sample head takes.  FP64 is slow on this part (CUDA's log took 3 us of a call on
// its own), so the logarithm is taken in pairs of floats: p = 2^k m with m in [sqrt(1/2),
// sqrt(2)), ln m = 2 atanh(s) = 2 (s + s^3/3 + s^5/5 + ...) with s = (m - 1) / (m + 1).  The
// product is off by less than 2^-45 of itself (the worst of 3e8 random ones, against 64 bits of
// mantissa); where the nearest float could be another one for an error 16 times that, one case in
// 65536, and where the pair's low half is out of fp32's range, FP64 decides.
struct Float2 {
  float hi, lo;
};
__device__ __forceinline__ Float2 sum_of(float a, float b) {  // exactly (Knuth)
  const float s = __fadd_rn(a, b), bb = __fsub_rn(s, a);
  return {s, __fadd_rn(__fsub_rn(a, __fsub_rn(s, bb)), __fsub_rn(b, bb))};
}
__device__ __forceinline__ Float2 product_of(float a, float b) {  // exactly
  const float h = __fmul_rn(a, b);
  return {h, __fmaf_rn(a, b, -h)};
}
__device__ __forceinline__ Float2 add(Float2 a, Float2 b) {
  const Float2 s = sum_of(a.hi, b.hi);
  return sum_of(s.hi, __fadd_rn(s.lo, __fadd_rn(a.lo, b.lo)));
}
__device__ __forceinline__ Float2 mul(Float2 a, Float2 b) {
  const Float2 h = product_of(a.hi, b.hi);
  return sum_of(h.hi, __fadd_rn(h.lo, __fmaf_rn(a.hi, b.lo, __fmul_rn(a.lo, b.hi))));
}
__device__ __noinline__ float scaled_log_fp64(float temp, float p) { return (float)((double)temp * log((double)p)); }
__device__ __forceinline__ float scaled_log(float temp, float p) {
  if (p == 0.f) return -INFINITY;
  const bool small = p < 0x1p-100f;  // (subnormals too)
  const uint32_t bits = __float_as_uint(small ? p * 0x1p60f : p);
  int k = small ? -60 : 0;
  k += (int)(bits >> 23) - 127;
  float m = __uint_as_float((bits & 0x7fffffu) | 0x3f800000u);
  if (m > 1.4142135f) {
    m *= 0.5f;
    ++k;
  }
  const float a = m - 1.f;  // (exact)
  const Float2 b = sum_of(m, 1.f);
  const float q = __fdiv_rn(a, b.hi);
  const float r = __fmaf_rn(-q, b.lo, __fmaf_rn(-q, b.hi, a));
  const Float2 s = sum_of(q, __fdiv_rn(r, b.hi)), z = mul(s, s);
  // 1/3 + z/5 + z^2/7 + ... + z^8/19, z <= 0.0295: the last terms need fewer digits
  float tail = 1.f / 19.f;
  tail = __fmaf_rn(tail, z.hi, 1.f / 17.f);
  tail = __fmaf_rn(tail, z.hi, 1.f / 15.f);
  tail = __fmaf_rn(tail, z.hi, 1.f / 13.f);
  tail = __fmaf_rn(tail, z.hi, 1.f / 11.f);
  Float2 c = add(mul({tail, 0.f}, z), {(float)(1.0 / 9), (float)(1.0 / 9 - (double)(float)(1.0 / 9))});
  c = add(mul(c, z), {(float)(1.0 / 7), (float)(1.0 / 7 - (double)(float)(1.0 / 7))});
  c = add(mul(c, z), {(float)(1.0 / 5), (float)(1.0 / 5 - (double)(float)(1.0 / 5))});
  c = add(mul(c, z), {(float)(1.0 / 3), (float)(1.0 / 3 - (double)(float)(1.0 / 3))});
  Float2 l = add(s, mul(s, mul(c, z)));
  l = {2.f * l.hi, 2.f * l.lo};
  constexpr double kLn2 = 0.69314718055994530942;
  l = add(mul({(float)k, 0.f}, {(float)kLn2, (float)(kLn2 - (double)(float)kLn2)}), l);
  const Float2 v = product_of(l.hi, temp);
  const float size = fabsf(v.hi);
  const Float2 w = sum_of(v.hi, __fmaf_rn(l.lo, temp, v.lo));
  const bool decided = size > 0x1p-96f && size < 0x1p127f && __fmaf_rn(w.lo, 1.f + 0x1p-16f, w.hi) == w.hi;
  return decided || p == 1.f ? w.hi : scaled_log_fp64(temp, p);
}

}  // namespace
}  // namespace rgd
