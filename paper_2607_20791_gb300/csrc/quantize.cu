// 8-bit floating point (e4m3) with a scale for every block of 128 columns, of one row
// (activations) or of 128 rows (weights).  The block's largest magnitude becomes 448, the
// largest number of the type: up = 448 / most, q = e4m3(x up), scale = most / 448.
//
// Bound by bytes: values are read once and stay in registers while their block's largest is
// found.  Eight lanes hold a row's 128 columns, 16 each: whole 16-byte stores, three shuffles
// a block.  16384 x 14336 bf16: 115 us, 6.1 TB/s, 0.91 of what a copy reaches; fp32: 166 us, 7.1 TB/s;
// 80 x 4096: 1.5 us.  Blocks of 128 rows, 14336 x 4096: bf16 54 us, 3.3 TB/s, fp32 46 us, 6.3 TB/s.  Rows
// off 16 bytes go value by value: 16384 x 14333 bf16 434 us.
#include <cuda_bf16.h>

#include "common.h"
#include "ptx.cuh"

namespace rgd {
namespace {

constexpr int kBlockCols = 128;
constexpr float kMostE4m3 = 448.f;
// A block whose largest magnitude is below this is scaled as if it were this: 448 / most stays
// finite and most / 448 normal.
constexpr float kLeast = 0x1p-100f;

struct QuantizeParams {
  const uint8_t* x;
  int64_t x_stride;  // bytes
  uint8_t* q;
  int64_t q_stride;
  float* scales;
  int32_t rows, cols, blocks;  // blocks of columns
  int32_t* dev_status;
};

// 16 values from column c0 on; 0 from the row's end on.
template <typename T, bool kVectors>
__device__ __forceinline__ void load16(const QuantizeParams& p, int64_t row, int64_t c0, float (&x)[16]) {
  const uint8_t* at = p.x + row * p.x_stride + c0 * (int64_t)sizeof(T);
  if (kVectors && c0 + 16 <= p.cols) {
#pragma unroll
    for (int v = 0; v < (int)sizeof(T); ++v) {
      const uint4 w = __ldcs(reinterpret_cast<const uint4*>(at) + v);
      const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (sizeof(T) == 4) {
          x[4 * v + i] = __uint_as_float(u[i]);
        } else {
          x[8 * (v & 1) + 2 * i] = __uint_as_float(u[i] << 16);
          x[8 * (v & 1) + 2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
        }
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = c0 + i < p.cols ? (float)reinterpret_cast<const T*>(at)[i] : 0.f;
  }
}

// The largest magnitude; NaN if any value is (so that a scale says so).
__device__ __forceinline__ float larger(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float most16(const float (&x)[16]) {
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) m = larger(m, fabsf(x[i]));
  return m;
}

__device__ __forceinline__ uint32_t e4m3x2(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}

template <bool kVectors>
__device__ __forceinline__ void store16(const QuantizeParams& p, int64_t row, int64_t c0, const float (&x)[16], float up) {
  uint32_t u[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    u[i] = e4m3x2(x[4 * i] * up, x[4 * i + 1] * up) | e4m3x2(x[4 * i + 2] * up, x[4 * i + 3] * up) << 16;
  uint8_t* at = p.q + row * p.q_stride + c0;
  if (kVectors && c0 + 16 <= p.cols) {
    *reinterpret_cast<uint4*>(at) = make_uint4(u[0], u[1], u[2], u[3]);
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (c0 + i < p.cols) at[i] = (uint8_t)(u[i >> 2] >> (8 * (i & 3)));
  }
}

// 448 / most for a block (0 for one of zeros), and its scale where `tell`.
__device__ __forceinline__ float scale_of(const QuantizeParams& p, float most, bool tell, int64_t at) {
  const float m = most > 0.f ? fmaxf(most, kLeast) : most;
  if (tell) {
    p.scales[at] = __fdiv_rn(m, kMostE4m3);
    if (!(most < INFINITY) && p.dev_status) atomicOr(p.dev_status, RGD_DEV_BAD_PARAM);
  }
  return most == 0.f ? 0.f : __fdiv_rn(kMostE4m3, m);
}

constexpr int kQuantizeThreads = 256;
constexpr int kGroupsEach = kQuantizeThreads / 8;  // blocks of columns that a CTA works on at once

// Eight lanes to a block of one row.
template <typename T, bool kVectors>
__global__ void __launch_bounds__(kQuantizeThreads) quantize_rows_kernel(const QuantizeParams p) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");  // (a dependent waits for this kernel's end)
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int64_t unit = (int64_t)blockIdx.x * kGroupsEach + (threadIdx.x >> 3);
  const int64_t row = unit / p.blocks;
  const int block = (int)(unit - row * p.blocks), part = threadIdx.x & 7;
  const bool on = row < p.rows;
  const int64_t c0 = (int64_t)block * kBlockCols + part * 16;
  float x[16];
  if (on) load16<T, kVectors>(p, row, c0, x);
  float most = on ? most16(x) : 0.f;
#pragma unroll
  for (int o = 4; o > 0; o >>= 1) most = larger(most, __shfl_xor_sync(0xffffffffu, most, o));
  if (!on) return;
  const float up = scale_of(p, most, part == 0, unit);
  store16<kVectors>(p, row, c0, x, up);
}

// A CTA to a block of 128 rows: every eight lanes hold 128 columns of four of them.
template <typename T, bool kVectors>
__global__ void __launch_bounds__(kQuantizeThreads) quantize_blocks_kernel(const QuantizeParams p) {
  __shared__ float part_most[kQuantizeThreads / 32];
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  constexpr int kEach = kBlockCols / kGroupsEach;
  const int64_t r0 = (int64_t)(blockIdx.x / (uint32_t)p.blocks) * kBlockCols;
  const int block = (int)(blockIdx.x % (uint32_t)p.blocks);
  const int64_t c0 = (int64_t)block * kBlockCols + (threadIdx.x & 7) * 16;
  float x[kEach][16], most = 0.f;
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int64_t row = r0 + i * kGroupsEach + (threadIdx.x >> 3);
    if (row < p.rows) load16<T, kVectors>(p, row, c0, x[i]);
  }
#pragma unroll
  for (int i = 0; i < kEach; ++i)
    if (r0 + i * kGroupsEach + (threadIdx.x >> 3) < p.rows) most = larger(most, most16(x[i]));
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) most = larger(most, __shfl_xor_sync(0xffffffffu, most, o));
  if ((threadIdx.x & 31) == 0) part_most[threadIdx.x >> 5] = most;
  __syncthreads();
  most = part_most[threadIdx.x & 7];
#pragma unroll
  for (int o = 4; o > 0; o >>= 1) most = larger(most, __shfl_xor_sync(0xffffffffu, most, o));
  const float up = scale_of(p, most, threadIdx.x == 0, blockIdx.x);
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int64_t row = r0 + i * kGroupsEach + (threadIdx.x >> 3);
    if (row < p.rows) store16<kVectors>(p, row, c0, x[i], up);
  }
}

template <typename T>
cudaError_t launch_quantize(const QuantizeParams& p, int32_t block_rows, bool vectors, cudaStream_t st) {
  if (block_rows == 1) {
    const int64_t units = (int64_t)p.rows * p.blocks;
    const int grid = (int)((units + kGroupsEach - 1) / kGroupsEach);
    return vectors ? launch_dependent(quantize_rows_kernel<T, true>, grid, kQuantizeThreads, 0, st, p)
                   : launch_dependent(quantize_rows_kernel<T, false>, grid, kQuantizeThreads, 0, st, p);
  }
  const int grid = (int)(((int64_t)p.rows + kBlockCols - 1) / kBlockCols * p.blocks);
  return vectors ? launch_dependent(quantize_blocks_kernel<T, true>, grid, kQuantizeThreads, 0, st, p)
                 : launch_dependent(quantize_blocks_kernel<T, false>, grid, kQuantizeThreads, 0, st, p);
}

}  // namespace
}  // namespace rgd

using namespace rgd;

extern "C" int rgd_fp8_quantize(int32_t rows, int32_t cols, int32_t dtype, const void* x, int64_t x_stride,
                                int32_t block_rows, uint8_t* q, int64_t q_stride, float* scales, int32_t* dev_status,
                                rgd_stream_t stream) {
  clear_error();
  const char* fn = "rgd_fp8_quantize";
  RGD_CHECK_ARG(rows >= 0 && cols >= 0, "%s: rows and cols must not be negative", fn);
  RGD_CHECK_ARG(dtype == RGD_F32 || dtype == RGD_BF16, "%s: dtype must be RGD_F32 or RGD_BF16", fn);
  RGD_CHECK_ARG(block_rows == 1 || block_rows == kBlockCols, "%s: block_rows must be 1 or 128", fn);
  RGD_CHECK_ARG(x_stride >= cols && q_stride >= cols, "%s: a stride is below cols", fn);
  if (rows == 0 || cols == 0) return RGD_OK;
  RGD_CHECK_ARG(x && q && scales, "%s: x/q/scales must be non-NULL", fn);
  const int es = dtype == RGD_F32 ? 4 : 2;
  RGD_CHECK_ARG(reinterpret_cast<uintptr_t>(x) % es == 0 && reinterpret_cast<uintptr_t>(scales) % 4 == 0,
                "%s: x and scales must be aligned to their elements", fn);
  QuantizeParams p{};
  p.x = static_cast<const uint8_t*>(x);
  p.x_stride = x_stride * es;
  p.q = q;
  p.q_stride = q_stride;
  p.scales = scales;
  p.rows = rows;
  p.cols = cols;
  p.blocks = (int32_t)(((int64_t)cols + kBlockCols - 1) / kBlockCols);
  p.dev_status = dev_status;
  const int64_t units = block_rows == 1 ? ((int64_t)rows * p.blocks + kGroupsEach - 1) / kGroupsEach
                                        : ((int64_t)rows + kBlockCols - 1) / kBlockCols * p.blocks;
  if (units > 0x7fffffff) return set_error(RGD_ERR_UNSUPPORTED, "%s: too many blocks", fn);
  const bool vectors = aligned16(x) && aligned16(q) && p.x_stride % 16 == 0 && q_stride % 16 == 0;
  const cudaError_t e = dtype == RGD_F32 ? launch_quantize<float>(p, block_rows, vectors, (cudaStream_t)stream)
                                         : launch_quantize<__nv_bfloat16>(p, block_rows, vectors, (cudaStream_t)stream);
  return e == cudaSuccess ? RGD_OK : cuda_error(e, "quantize launch");
}
