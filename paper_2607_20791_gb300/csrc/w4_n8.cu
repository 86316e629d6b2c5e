// The 4-bit products' kernel for up to 8 rows of x (a translation unit each, compiled in parallel).
#include "w4_kernel.cuh"

namespace rgd {

int launch_w4_n8(W4Params& p, cudaStream_t st) { return launch_w4<1>(p, st); }

}  // namespace rgd
