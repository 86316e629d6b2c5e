// Products of a few rows of activations with 4-bit weights: y = x W^T with
// W[n, k] = (q[n, k] - z[n, k / G]) s[n, k / G], q packed two to a byte along k.
//
// One warp per output column: each lane takes bytes of the column's row of W in turn, and
// the groups' scales with them.
#include <cuda_bf16.h>

#include <algorithm>

#include "common.h"
#include "ptx.cuh"

namespace rgd {
namespace {

constexpr int kW4Threads = 256;
constexpr int kW4Rows = 4;  // rows of x per pass over a warp's weights

struct W4Params {
  int32_t m, n, k, group, groups;
  const __nv_bfloat16* x;
  const uint8_t* w;
  const void* scales;
  const uint8_t* zeros;
  void* y;
  int64_t row_bytes, y_stride;
  int32_t scale_f32, out_f32;
};

__global__ void __launch_bounds__(kW4Threads) w4_kernel(const W4Params p) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");  // (a dependent waits for this kernel's end)
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int lane = threadIdx.x & 31;
  const int64_t n = (int64_t)blockIdx.x * (kW4Threads / 32) + (threadIdx.x >> 5);
  if (n >= p.n) return;
  const uint8_t* row = p.w + n * p.row_bytes;
  for (int m0 = 0; m0 < p.m; m0 += kW4Rows) {
    float acc[kW4Rows] = {};
    for (int b = lane; b < p.row_bytes; b += 32) {
      const uint8_t q = row[b];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int k = 2 * b + h;
        if (k >= p.k) break;
        const int64_t g = n * p.groups + k / p.group;
        const float s = p.scale_f32 ? static_cast<const float*>(p.scales)[g] : (float)static_cast<const __nv_bfloat16*>(p.scales)[g];
        const float w = (float)((h ? q >> 4 : q & 15) - (p.zeros ? p.zeros[g] : 8)) * s;
#pragma unroll
        for (int i = 0; i < kW4Rows; ++i)
          if (m0 + i < p.m) acc[i] = fmaf((float)p.x[(int64_t)(m0 + i) * p.k + k], w, acc[i]);
      }
    }
#pragma unroll
    for (int i = 0; i < kW4Rows; ++i) {
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) acc[i] += __shfl_xor_sync(0xffffffffu, acc[i], o);
      if (lane == 0 && m0 + i < p.m) {
        const int64_t at = (m0 + i) * p.y_stride + n;
        if (p.out_f32) static_cast<float*>(p.y)[at] = acc[i];
        else static_cast<__nv_bfloat16*>(p.y)[at] = __float2bfloat16(acc[i]);
      }
    }
  }
}

}  // namespace
}  // namespace rgd

using namespace rgd;

extern "C" int rgd_w4_matvec(int32_t m, int32_t n, int32_t k, int32_t group_size, const rgd_bf16* x,
                             const uint8_t* weights, int32_t scale_dtype, const void* scales, const uint8_t* zeros,
                             int32_t out_dtype, void* y, int64_t y_stride, rgd_stream_t stream) {
  clear_error();
  const char* fn = "rgd_w4_matvec";
  RGD_CHECK_ARG(m >= 0 && n >= 0 && k >= 1, "%s: bad m/n/k", fn);
  RGD_CHECK_ARG(group_size == 32 || group_size == 64 || group_size == 128, "%s: group_size must be 32, 64 or 128", fn);
  RGD_CHECK_ARG((scale_dtype == RGD_F32 || scale_dtype == RGD_BF16) && (out_dtype == RGD_F32 || out_dtype == RGD_BF16),
                "%s: scale_dtype and out_dtype must be RGD_F32 or RGD_BF16", fn);
  RGD_CHECK_ARG(y_stride >= n, "%s: y_stride < n", fn);
  if (m == 0 || n == 0) return RGD_OK;
  RGD_CHECK_ARG(x && weights && scales && y, "%s: x/weights/scales/y must be non-NULL", fn);
  RGD_CHECK_ARG(aligned16(x) && aligned16(weights) && aligned16(scales) && aligned16(zeros) && aligned16(y),
                "%s: tensors must be 16-byte aligned", fn);
  W4Params p{};
  p.m = m;
  p.n = n;
  p.k = k;
  p.group = group_size;
  p.groups = (k + group_size - 1) / group_size;
  p.x = reinterpret_cast<const __nv_bfloat16*>(x);
  p.w = weights;
  p.scales = scales;
  p.zeros = zeros;
  p.y = y;
  p.row_bytes = (k + 1) / 2;
  p.y_stride = y_stride;
  p.scale_f32 = scale_dtype == RGD_F32;
  p.out_f32 = out_dtype == RGD_F32;
  const int grid = (int)(((int64_t)n + kW4Threads / 32 - 1) / (kW4Threads / 32));
  const cudaError_t e = launch_dependent(w4_kernel, grid, kW4Threads, 0, (cudaStream_t)stream, p);
  return e == cudaSuccess ? RGD_OK : cuda_error(e, "w4 launch");
}
