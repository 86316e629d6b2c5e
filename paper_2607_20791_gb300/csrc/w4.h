// Shared between the 4-bit products' host side and their kernel's instantiations.
#pragma once

#include "common.h"

namespace rgd {

constexpr int kW4MaxK = 1 << 24;

struct W4Params {
  int32_t m, n, k, groups;
  int32_t group_shift;   // log2 of the group size
  int32_t block_chunks;  // chunks of a block of k
  int32_t blocks;        // blocks of k
  int32_t ksplit;        // blocks of a cluster that share a tile, each with rank_chunks chunks
  int32_t rank_chunks;
  int32_t batch;         // tiles of a block (or cluster) between which k may go in blocks
  const uint16_t* x;
  const uint8_t* w;
  const uint8_t* scales;
  const uint8_t* zeros;
  void* y;
  int64_t row_bytes, y_stride, total_bytes;
  int32_t scale_bytes, out_f32;
  int32_t x_vec;      // 2: rows of x lie on 16 bytes, 1: on 4
  int32_t scale_vec;  // a chunk's scales of a row are whole, aligned vectors
  int32_t x_shift;  // log2 of the rows of x that lie in shared memory of every 8
  int32_t* dev_status;
};

// Launches the kernel for 8 and for 16 rows of x at a time.
int launch_w4_n8(W4Params& p, cudaStream_t st);
int launch_w4_n16(W4Params& p, cudaStream_t st);

}  // namespace rgd
