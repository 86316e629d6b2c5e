// The 4-bit products' kernel for more than 8 rows of x (a translation unit each, compiled in parallel).
#include "w4_kernel.cuh"

namespace rgd {

int launch_w4_n16(W4Params& p, cudaStream_t st) { return launch_w4<2>(p, st); }

}  // namespace rgd
