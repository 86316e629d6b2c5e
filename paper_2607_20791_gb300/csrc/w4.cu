// Products with 4-bit weights: the entry point (the kernel is in w4_kernel.cuh).
#include "w4.h"

using namespace rgd;

extern "C" int rgd_w4_matvec(int32_t m, int32_t n, int32_t k, int32_t group_size, const rgd_bf16* x,
                             const uint8_t* weights, int32_t scale_dtype, const void* scales, const uint8_t* zeros,
                             int32_t out_dtype, void* y, int64_t y_stride, int32_t* dev_status,
                             rgd_stream_t stream) {
  clear_error();
  const char* fn = "rgd_w4_matvec";
  RGD_CHECK_ARG(m >= 0 && n >= 0 && k >= 1, "%s: bad m/n/k", fn);
  RGD_CHECK_ARG(k <= kW4MaxK, "%s: k too large", fn);
  RGD_CHECK_ARG(group_size == 32 || group_size == 64 || group_size == 128, "%s: group_size must be 32, 64 or 128", fn);
  RGD_CHECK_ARG((scale_dtype == RGD_F32 || scale_dtype == RGD_BF16) && (out_dtype == RGD_F32 || out_dtype == RGD_BF16),
                "%s: scale_dtype and out_dtype must be RGD_F32 or RGD_BF16", fn);
  RGD_CHECK_ARG(y_stride >= n, "%s: y_stride < n", fn);
  if (m == 0 || n == 0) return RGD_OK;
  RGD_CHECK_ARG(x && weights && scales && y, "%s: x/weights/scales/y must be non-NULL", fn);
  RGD_CHECK_ARG(aligned16(x) && aligned16(weights) && aligned16(scales) && aligned16(zeros) && aligned16(y),
                "%s: tensors must be 16-byte aligned", fn);
  RGD_CHECK_ARG(n <= 0x7fffffff - 1024, "%s: n too large", fn);
  W4Params p{};
  p.m = m;
  p.n = n;
  p.k = k;
  p.group_shift = group_size == 32 ? 5 : group_size == 64 ? 6 : 7;
  p.groups = (int32_t)(((int64_t)k + group_size - 1) / group_size);
  p.x = x;
  p.w = weights;
  p.scales = static_cast<const uint8_t*>(scales);
  p.zeros = zeros;
  p.y = y;
  p.row_bytes = ((int64_t)k + 1) / 2;
  p.total_bytes = p.row_bytes * n;
  p.y_stride = y_stride;
  p.scale_bytes = scale_dtype == RGD_F32 ? 4 : 2;
  p.out_f32 = out_dtype == RGD_F32;
  p.x_vec = k % 8 == 0 ? 2 : k % 2 == 0 ? 1 : 0;
  p.dev_status = dev_status;
  cudaStream_t st = (cudaStream_t)stream;
  return m <= 8 ? launch_w4_n8(p, st) : launch_w4_n16(p, st);
}
