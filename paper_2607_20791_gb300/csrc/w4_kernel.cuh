// Products of a few rows of activations with 4-bit weights: y = x W^T with
// W[n, k] = (q[n, k] - z[n, k / G]) s[n, k / G], q packed two to a byte along k.
//
// The weights are read once; everything else is small.  A tile is 32 rows of W, its k goes in
// chunks of 256 weights (for up to 8 rows of x and groups of 64 or 128, else 128), and each
// warp of a block takes an equal stretch of all its tiles' chunks, one tile after another.
// A chunk comes by TMA boxes of 64 bytes by the tile's rows into the warp's own ring in
// shared memory, 4 to 8 KB ahead of its use.  Every 128 weights are 8 mma.m16n8k16 with the
// weights as A for every 16 rows of W and 8 rows of x: one row of x costs the same as
// eight, and the tensor pipe does the sums over k in fp32.  (With 17 to 32 rows of x the
// weights are read twice, 16 rows at a time: 156 us for 32 x 4096 x 128256 where one pass
// of 32 took 198, x coming from shared memory in blocks of k.)
//
// Which k a lane's A elements stand for is free as long as B agrees, so a lane feeds the
// 8 nibbles of a 32-bit word as they lie: nibbles p and p + 4 are the two halves of
// (word >> 4p) & 0x000f000f, and with 0x4300 over each (bf16 128) they are the bf16
// numbers 128 + q.  128 + z taken from them leaves q - z exactly.  x lies in shared memory
// in that order, one 16-byte load a lane for two MMAs.  With groups of 128 a lane of a quad
// has 16 bytes of a row in one load.  With smaller ones an MMA's k must stay within 32
// weights: its quad reads a word each of the same 16 bytes, from boxes swizzled by 64 bytes
// so that the warp's 32 words lie in 32 banks.  A group's sum is scaled in fp32 after its
// last MMA.
//
// Rows off 16 bytes have no box: 16-byte asynchronous copies bring the whole vectors that
// hold a row's part of a chunk, and a lane's word is cut from the two it lies in.  (A bulk
// copy a row took 14 cycles each, half of the kernel's time.)
//
// One block of 16 warps fills an SM, so that x lies there once.  A warp writes the sums of the
// tiles it has whole; a tile that several warps have parts of is joined in shared memory at
// the end, so that nothing waits in between (groups of 4 warps that shared each tile, with
// two barriers a tile, took 61 us where this takes 57 for 5 x 4096 x 128256, and 33 where
// this takes 28 for 13 x 2730 x 20011).  Where x does not fit, k goes in blocks, with the
// sums of the block's tiles kept in shared memory between them.  Few tiles of long rows are
// shared by the blocks of a cluster, each with a stretch of k, whose sums the first one joins.
//
// What bounds it: 5 x 4096 x 128256 in groups of 128 takes 57 us, 0.71 of the copy rate, with
// 0.6 of the issue slots and of the integer pipe's cycles taken (7 integer operations and 4
// subtractions for every 8 weights of 32 rows), the tensor pipe a quarter busy.
#pragma once

#include <cuda_bf16.h>

#include <algorithm>

#include "ptx.cuh"
#include "w4.h"

namespace rgd {
namespace {

constexpr int kPart = 128;           // weights of a row that a lane's quad works on together
constexpr int kW4Smem = 226 * 1024;  // (of 227; the barriers take the rest)
constexpr int kWarps = 16;           // of a block

constexpr int kSub = 2;              // groups of 16 rows of W in a tile
constexpr int kRows = 16 * kSub;     // of a tile
constexpr int kAhead = 2;            // chunks in flight
constexpr int kMaxSplit = 8;         // blocks that share a tile's k

// Parts of a chunk (GS: steps of 32 weights in a group): two halve what a chunk costs besides its
// products, but the scales of small groups would take more registers than there are.
template <int NT, int GS>
constexpr int kParts = NT == 1 && GS > 1 ? 2 : 1;
template <int NT, int GS>
constexpr int kChunk = kPart * kParts<NT, GS>;

// Shared memory: the warps' rings, every warp's sums of a tile, the sums kept between blocks of
// k, the warps' scales (where groups are small), x.
template <int NT, int GS, bool kAligned, bool kZeros>
struct Layout {
  static constexpr int kSums = kRows * 8 * NT;
  static constexpr int kJoin = kWarps * kSums * 4;
  static constexpr int kPitch = kAligned ? 64 : kParts<NT, GS> * 64 + 16;            // from a row to the next
  static constexpr int kSlot = kRows * (kAligned ? kParts<NT, GS> * 64 : kPitch);    // of a chunk
  static constexpr int kRing = kWarps * kAhead * kSlot;
  static constexpr int kGroups = 4 / GS;                                         // of a part
  static constexpr int kScales = GS == 4 ? 0 : kParts<NT, GS> * kRows * kGroups * 4;  // bytes of a warp
  static constexpr int kZeroBytes = GS == 4 || !kZeros ? 0 : kParts<NT, GS> * kRows * kGroups;
  static constexpr int kFixed = kRing + kJoin + kWarps * (kScales + kZeroBytes);
};

__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// The same from zero.
__device__ __forceinline__ void mma16816_first(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                               uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}

// Nibbles p and p + 4 of a word as bf16 q - z (bias: 128 + z twice).  `magic` is 0x43004300 in a
// register, so that mask and exponent go in by one instruction.
__device__ __forceinline__ uint32_t weights2(uint32_t word, int p, uint32_t magic, uint32_t bias) {
  uint32_t u;
  asm("lop3.b32 %0, %1, 0x000f000f, %2, 0xea;" : "=r"(u) : "r"(word >> (4 * p)), "r"(magic));
  const __nv_bfloat162 v = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&u), *reinterpret_cast<const __nv_bfloat162*>(&bias));
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ uint32_t exponent_bits() {
  uint32_t m;
  asm volatile("mov.b32 %0, 0x43004300;" : "=r"(m));
  return m;
}

__device__ __forceinline__ void copy_box(uint32_t dst, const CUtensorMap* map, int32_t x, int32_t y, uint64_t* bar) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
               "l"(map), "r"(x), "r"(y), "r"(smem_u32(bar))
               : "memory");
}

// A chunk's scales and zeros (NL a row) as they lie in memory; a load must not be waited for
// before its use.  Where the rows' counts allow (scale_vec) lane i has those of row i of the
// tile, by one or two vector loads, bf16 scales two and zeros four to a word.  Else load i
// brings those of rows 32 / NL i .. by one each: lane j that of row j / NL, group j % NL.  (A
// load of one scale from each of 32 rows looks up 32 lines: with groups of 32 that was the
// kernel's time twice over.)
template <int NL, bool kZeros>
struct Scales {
  uint32_t s[NL], z[kZeros ? NL : 1];
};

template <int kBytes>
__device__ __forceinline__ void load_bytes(const uint8_t* p, uint32_t* into) {
  if (kBytes == 1) into[0] = __ldg(p);
  if (kBytes == 2) into[0] = __ldg(reinterpret_cast<const uint16_t*>(p));
  if (kBytes == 4) into[0] = __ldg(reinterpret_cast<const uint32_t*>(p));
  if (kBytes == 8) {
    const uint2 v = __ldg(reinterpret_cast<const uint2*>(p));
    into[0] = v.x, into[1] = v.y;
  }
#pragma unroll
  for (int i = 0; i < kBytes / 16; ++i) {
    const uint4 v = __ldg(reinterpret_cast<const uint4*>(p) + i);
    into[4 * i] = v.x, into[4 * i + 1] = v.y, into[4 * i + 2] = v.z, into[4 * i + 3] = v.w;
  }
}

// Where a tile's scales and zeros begin, and its last row that W has.
struct TileScales {
  const uint8_t *s, *z;
  int last;
  __device__ TileScales(const W4Params& p, int tile) {
    const int64_t at = (int64_t)tile * kRows * p.groups;
    s = p.scales + at * p.scale_bytes;
    z = p.zeros + at;
    last = (int)min(int64_t(kRows - 1), p.n - 1 - (int64_t)tile * kRows);
  }
};
template <int NL, bool kZeros>
__device__ __forceinline__ void load_scales(const W4Params& p, Scales<NL, kZeros>& c, const TileScales& tile, int part, int lane) {
  const int g = (part * kPart) >> p.group_shift;
  if (p.scale_vec) {
    const int at = min(lane, tile.last) * p.groups + g;
    if (p.scale_bytes == 2) load_bytes<2 * NL>(tile.s + 2 * (int64_t)at, c.s);
    else load_bytes<4 * NL>(tile.s + 4 * (int64_t)at, c.s);
    if (kZeros) load_bytes<NL>(tile.z + at, c.z);
    return;
  }
  const int mine = min(g + lane % NL, p.groups - 1);  // (past the row's end x is zero)
#pragma unroll
  for (int i = 0; i < NL; ++i) {
    const int at = min(i * (32 / NL) + lane / NL, tile.last) * p.groups + mine;
    if (p.scale_bytes == 2) c.s[i] = __ldg(reinterpret_cast<const uint16_t*>(tile.s) + at);
    else c.s[i] = __ldg(reinterpret_cast<const uint32_t*>(tile.s) + at);
    if (kZeros) c.z[i] = __ldg(tile.z + at);
  }
}
// Scale i as a number.
template <int NL, bool kZeros>
__device__ __forceinline__ float scale_of(const W4Params& p, const Scales<NL, kZeros>& c, int i) {
  if (p.scale_bytes == 4) return __uint_as_float(c.s[i]);
  if (!p.scale_vec) return __uint_as_float(c.s[i] << 16);
  return __uint_as_float((i & 1) ? c.s[i / 2] & 0xffff0000u : c.s[i / 2] << 16);
}

// Small groups' scales and zeros into the warp's place in shared memory, as [part][row][group].
template <int kEach, int NL, bool kZeros>
__device__ __forceinline__ void spread_scales(const W4Params& p, const Scales<NL, kZeros>& c, float* scales, uint8_t* zeros, int lane) {
  if (p.scale_vec) {
#pragma unroll
    for (int i = 0; i < NL; ++i) scales[(i / kEach * kRows + lane) * kEach + i % kEach] = scale_of(p, c, i);
    if constexpr (kZeros) {
#pragma unroll
      for (int c2 = 0; c2 < NL / kEach; ++c2) {
        uint8_t* to = zeros + (c2 * kRows + lane) * kEach;
        if (kEach == 4) *reinterpret_cast<uint32_t*>(to) = c.z[c2];
        else *reinterpret_cast<uint16_t*>(to) = (uint16_t)(c.z[0] >> (16 * c2));
      }
    }
  } else {
    const int row = lane / NL, i0 = lane % NL;
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int at = (i0 / kEach * kRows + i * (32 / NL) + row) * kEach + i0 % kEach;
      scales[at] = scale_of(p, c, i);
      if constexpr (kZeros) zeros[at] = (uint8_t)c.z[i];
    }
  }
}

// Adds the products of a part of the tile's rows (q: a lane's words of rows g + 8 h by step) to
// their sums.  s: the groups' scales of those rows; z: their zeros, a byte each.
template <int NT, int GS, bool kZeros>
__device__ __forceinline__ void multiply_part(const uint32_t (&q)[2 * kSub][4], const float (&s)[2 * kSub][4 / GS],
                                              const uint32_t (&z)[2 * kSub], const uint8_t* xs, int unit,
                                              float (&acc)[kSub][NT][4], uint32_t magic) {
#pragma unroll
  for (int g = 0; g < 4 / GS; ++g) {
    uint32_t bias[2 * kSub];
#pragma unroll
    for (int h = 0; h < 2 * kSub; ++h) bias[h] = kZeros ? __byte_perm(z[h], 0x43, 0x4040 + 0x101 * g) : 0x43084308u;
    float sum[kSub][NT][4];
#pragma unroll
    for (int i = 0; i < GS; ++i) {
      const int j = g * GS + i;
      uint4 x[NT];
#pragma unroll
      for (int n = 0; n < NT; ++n) x[n] = *reinterpret_cast<const uint4*>(xs + (j * NT + n) * unit);
#pragma unroll
      for (int b = 0; b < kSub; ++b) {
        uint32_t lo[4], hi[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          lo[e] = weights2(q[2 * b][j], e, magic, bias[2 * b]);
          hi[e] = weights2(q[2 * b + 1][j], e, magic, bias[2 * b + 1]);
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          if (i == 0) mma16816_first(sum[b][n], lo[0], hi[0], lo[1], hi[1], x[n].x, x[n].y);
          else mma16816(sum[b][n], lo[0], hi[0], lo[1], hi[1], x[n].x, x[n].y);
          mma16816(sum[b][n], lo[2], hi[2], lo[3], hi[3], x[n].z, x[n].w);
        }
      }
    }
#pragma unroll
    for (int b = 0; b < kSub; ++b)
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[b][n][e] = fmaf(s[2 * b + (e >> 1)][g], sum[b][n][e], acc[b][n][e]);
  }
}

// Eight numbers of x from a place of any alignment: from the two aligned vectors they lie in, or
// one by one where those reach past the end of x; `left` of them (or more) are the row's.
struct Eight {
  uint4 v[2];
  __device__ __forceinline__ void load(const W4Params& p, const uint16_t* src, int left) {
    const uint16_t* end = p.x + (int64_t)p.m * p.k;
    const uint16_t* at = reinterpret_cast<const uint16_t*>(reinterpret_cast<uintptr_t>(src) & ~uintptr_t(15));
    if (at + 16 <= end) {
      v[0] = __ldg(reinterpret_cast<const uint4*>(at));
      v[1] = __ldg(reinterpret_cast<const uint4*>(at) + 1);
    } else {  // (as if they lay where `src` does in its vector)
      uint16_t e[16];
      const int off = (int)(src - at);
#pragma unroll
      for (int b = 0; b < 16; ++b) e[b] = b >= off && b < off + left && at + b < end ? __ldg(at + b) : 0;
#pragma unroll
      for (int h = 0; h < 2; ++h)
        v[h] = make_uint4(e[8 * h] | (uint32_t)e[8 * h + 1] << 16, e[8 * h + 2] | (uint32_t)e[8 * h + 3] << 16,
                          e[8 * h + 4] | (uint32_t)e[8 * h + 5] << 16, e[8 * h + 6] | (uint32_t)e[8 * h + 7] << 16);
    }
  }
  __device__ __forceinline__ uint4 get(const uint16_t* src, int left) const {
    const uint32_t by = (uint32_t)reinterpret_cast<uintptr_t>(src);
    uint32_t w[8] = {v[0].x, v[0].y, v[0].z, v[0].w, v[1].x, v[1].y, v[1].z, v[1].w};
#pragma unroll
    for (int i = 0; i < 6; ++i) w[i] = (by & 8) ? w[i + 2] : w[i];
#pragma unroll
    for (int i = 0; i < 5; ++i) w[i] = (by & 4) ? w[i + 1] : w[i];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      w[i] = __funnelshift_r(w[i], w[i + 1], (by & 2) * 8);
      if (left < 2 * i + 2) w[i] = left > 2 * i ? w[i] & 0xffffu : 0;
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
};

// A block of x into shared memory: for every part and step the 8 numbers of each row and lane
// of a quad, in the order of the nibbles; a power of two up to 8 rows of every 8.
template <int NT, bool kTurned>
__device__ __forceinline__ void stage_x(const W4Params& p, uint8_t* xs, int part0, int parts, int m0) {
  constexpr int kThreads = kWarps * 32;
  const int lanes = 2 + p.x_shift;  // log2 of the lanes that have x
  const int units = (parts * 4 * NT) << lanes;
  auto place = [&](int u, int& m, int& k) {
    const int v = u >> lanes, i = v % NT, j = v / NT & 3, c = v / (NT * 4), t = u & 3;
    m = m0 + i * 8 + (u >> 2 & ((1 << p.x_shift) - 1));
    k = (part0 + c) * kPart + (kTurned ? j * 32 + t * 8 : t * 32 + j * 8);
  };
  auto store = [&](int u, const uint4& r) {
    if (u < units)
      *reinterpret_cast<uint4*>(xs + (int64_t)u * 16) =
          make_uint4(__byte_perm(r.x, r.z, 0x5410), __byte_perm(r.x, r.z, 0x7632), __byte_perm(r.y, r.w, 0x5410),
                     __byte_perm(r.y, r.w, 0x7632));
  };
  if (p.x_vec) {
    constexpr int kBatch = 8;  // loads in flight
    for (int u0 = threadIdx.x; u0 < units; u0 += kThreads * kBatch) {
      uint4 r[kBatch];
#pragma unroll
      for (int f = 0; f < kBatch; ++f) {
        int m, k;
        place(u0 + f * kThreads, m, k);
        r[f] = make_uint4(0, 0, 0, 0);
        if (u0 + f * kThreads >= units || m >= p.m || k >= p.k) continue;
        const uint16_t* src = p.x + (int64_t)m * p.k + k;
        if (p.x_vec == 2) {  // (p.k is a multiple of 8)
          r[f] = __ldg(reinterpret_cast<const uint4*>(src));
        } else {  // (... of 2)
          const uint32_t* q = reinterpret_cast<const uint32_t*>(src);
          r[f].x = __ldg(q);
          if (k + 2 < p.k) r[f].y = __ldg(q + 1);
          if (k + 4 < p.k) r[f].z = __ldg(q + 2);
          if (k + 6 < p.k) r[f].w = __ldg(q + 3);
        }
      }
#pragma unroll
      for (int f = 0; f < kBatch; ++f) store(u0 + f * kThreads, r[f]);
    }
    return;
  }
  // Odd p.k.  (Eight 2-byte loads took 36 us where this takes 32 for 16 x 4095 x 20011; 4-byte
  // loads above are the faster where they will do, 28 us for 31 of 13 x 2730 x 20011.)
  constexpr int kBatch = 4;
#pragma unroll 1
  for (int u0 = threadIdx.x; u0 < units; u0 += kThreads * kBatch) {
    Eight r[kBatch];
#pragma unroll
    for (int f = 0; f < kBatch; ++f) {
      int m, k;
      place(u0 + f * kThreads, m, k);
      r[f].v[0] = r[f].v[1] = make_uint4(0, 0, 0, 0);
      if (u0 + f * kThreads < units && m < p.m && k < p.k) r[f].load(p, p.x + (int64_t)m * p.k + k, p.k - k);
    }
#pragma unroll
    for (int f = 0; f < kBatch; ++f) {
      int m, k;
      place(u0 + f * kThreads, m, k);
      store(u0 + f * kThreads, r[f].get(p.x + (int64_t)m * p.k + k, p.k - k));
    }
  }
}

// Rows off 16 bytes: starts the copies of the vectors that hold the tile's part (or two).
// Nothing is read past the weights' end or for rows past the last: zeros fill its place.
template <int P>
__device__ __forceinline__ void copy_vectors(const W4Params& p, uint32_t to, int tile, int part, int lane) {
  constexpr int kEach = P * 4 + 1;  // vectors of a row
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int u = i * 32 + lane, row = u / kEach, v = u % kEach;
    const int64_t n = (int64_t)tile * kRows + row;
    const int64_t at = ((n * p.row_bytes + (int64_t)part * (kPart / 2)) & ~int64_t(15)) + 16 * v;
    const int bytes = n < p.n ? (int)max(int64_t(0), min(int64_t(16), p.total_bytes - at)) : 0;
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to + u * 16), "l"(p.w + (bytes ? at : 0)), "r"(bytes) : "memory");
  }
}

__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
}
__device__ __forceinline__ void push_sum(float* slot, float v) {
  uint32_t at;
  asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(at) : "r"(smem_u32(slot)));
  asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(at), "f"(v) : "memory");
}
__device__ __forceinline__ void write_sum(const W4Params& p, int m, int64_t n, float v) {
  if (m >= p.m || n >= p.n) return;
  if (p.out_f32) static_cast<float*>(p.y)[m * p.y_stride + n] = v;
  else static_cast<__nv_bfloat16*>(p.y)[m * p.y_stride + n] = __float2bfloat16(v);
}

template <int NT, int GS, bool kAligned, bool kZeros>
__global__ void __launch_bounds__(kWarps * 32, 1) w4_kernel(const W4Params p, const __grid_constant__ CUtensorMap map) {
  using L = Layout<NT, GS, kAligned, kZeros>;
  constexpr bool kTurned = GS < 4 || !kAligned;  // a quad's words are of the same 16 bytes
  constexpr int kSums = L::kSums, R = kRows / 8, A = kAhead, P = kParts<NT, GS>;
  constexpr int H = GS == 4 ? 2 : 1;  // chunks whose scales are on their way (2 for groups of 32: 31.8 us for 28.8 in 13 x 2730 x 20011)
  constexpr int kEach = L::kGroups, NL = P * kEach;  // scales of a lane and part, and chunk
  extern __shared__ __align__(1024) uint8_t dyn[];
  __shared__ uint64_t landed[kWarps][A];
  __shared__ int begun[kWarps];  // the tile that a warp has the first of several parts of (as ~tile: in its ring), or -1
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, t = lane & 3;
  const uint8_t* ring = dyn + warp * A * L::kSlot;
  float* join = reinterpret_cast<float*>(dyn + L::kRing);                       // [kWarps][kSums]
  float* scales = reinterpret_cast<float*>(dyn + L::kRing + L::kJoin + warp * L::kScales);  // [P][kRows][kGroups]
  uint8_t* zeros = dyn + L::kRing + L::kJoin + kWarps * L::kScales + warp * L::kZeroBytes;  // [P][kRows][kGroups]
  float* others = reinterpret_cast<float*>(dyn + L::kFixed);                                // [ksplit][kSums]
  float* kept = others + (p.ksplit > 1 ? p.ksplit * kSums : 0);                             // [batch][kSums]
  uint8_t* xs = dyn + L::kFixed + ((p.ksplit > 1 ? p.ksplit : 0) + (p.blocks > 1 ? p.batch : 0)) * kSums * 4;
  if (lane == 0) {
#pragma unroll
    for (int s = 0; s < A; ++s) mbar_init(&landed[warp][s], 1);
    fence_mbar_init();
    fence_proxy_async_smem();
  }
  __syncwarp();
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");  // (a dependent waits for this kernel's end)
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int tiles = (p.n + kRows - 1) / kRows;
  // block (or cluster) b of B takes tiles b, b + B, ...
  const int block = (int)blockIdx.x / p.ksplit, rank = (int)blockIdx.x % p.ksplit, blocks = (int)gridDim.x / p.ksplit;
  const int mine = (tiles - block + blocks - 1) / blocks;
  const int my_chunks = min((p.k + kChunk<NT, GS> - 1) / kChunk<NT, GS>, (rank + 1) * p.rank_chunks);  // up to which this block goes
  const uint32_t ring_at = smem_u32(ring), magic = exponent_bits();
  const int unit = 64 << p.x_shift;                                            // bytes of x of a step and 8 rows
  const uint8_t* my_x = xs + (lane & ((4 << p.x_shift) - 1)) * 16;             // (rows that are not there repeat others; their sums are dropped)
  // where a lane's words of a part lie: of row g, by step
  uint32_t word_at[4], cut[R];
  {
    const int g = lane >> 2;
#pragma unroll
    for (int j = 0; j < 4; ++j) word_at[j] = kAligned ? g * 64 + ((j ^ (g >> 1 & 3)) << 4) + t * 4 : g * L::kPitch + j * 16 + t * 4;
#pragma unroll
    for (int h = 0; h < R; ++h)  // (rows off 16 bytes: where their first byte lies in its vector; tiles start on one)
      cut[h] = kAligned ? 0 : (uint32_t)(((int64_t)(g + 8 * h) * p.row_bytes) & 15);
  }
  if (p.ksplit > 1) cluster_sync();  // (every block has started)
  uint32_t parity = 0;       // of each slot's barrier
  int flying = 0, lost = 0;  // copies on their way, and the slot of the oldest once a wait has given up
  bool alive = true;         // no wait has given up
  for (int m0 = 0; m0 < p.m; m0 += 8 * NT) {
    for (int first = 0; first < mine; first += p.batch) {
      const int batch = min(p.batch, mine - first);
      for (int kb = 0; kb < p.blocks; ++kb) {
        // The chunks of the tiles, in order: each warp takes a stretch of them.
        const int chunk0 = rank * p.rank_chunks + kb * p.block_chunks;
        const int chunks = max(0, min(p.block_chunks, my_chunks - chunk0));
        const int items = batch * chunks, per = (items + kWarps - 1) / kWarps;
        const int begin = min(warp * per, items), end = min(begin + per, items);
        int tile = batch == 1 ? 0 : begin / max(chunks, 1), at = begin - tile * chunks;
        int li = begin, lc = at, load_tile = block + (first + tile) * blocks;  // the next chunk to load, and its tile
        auto load = [&](int s) {
          if (li < end) {
            const int part = (chunk0 + lc) * P;
            if (!kAligned) {
              copy_vectors<P>(p, ring_at + s * L::kSlot, load_tile, part, lane);
            } else if (alive) {
              ++flying;
              if (lane == 0) {
                mbar_arrive_expect_tx(&landed[warp][s], L::kSlot);
#pragma unroll
                for (int c2 = 0; c2 < P; ++c2)  // (what lies past a row's end or the last row is filled with zeros)
                  copy_box(ring_at + s * L::kSlot + c2 * kRows * 64, &map, (part + c2) * (kPart / 2), load_tile * kRows,
                           &landed[warp][s]);
              }
            }
          }
          if (!kAligned) asm volatile("cp.async.commit_group;" ::: "memory");
          ++li;
          if (++lc < chunks) return;
          lc = 0;
          load_tile += blocks;
        };
        // Scales are loaded ahead too: of the next chunk, or two where they take few registers.
        Scales<NL, kZeros> ahead[H] = {};
        int si = begin, sat = at, scale_tile = load_tile;
        TileScales tile_scales(p, scale_tile);
        auto load_next = [&](Scales<NL, kZeros>& into) {
          if (si < end) load_scales(p, into, tile_scales, (chunk0 + sat) * P, lane);
          ++si;
          if (++sat < chunks) return;
          sat = 0;
          scale_tile += blocks;
          tile_scales = TileScales(p, scale_tile);
        };
#pragma unroll
        for (int s = 0; s < A; ++s) load(s);
#pragma unroll
        for (int u = 0; u < H; ++u) load_next(ahead[u]);
        if (p.blocks > 1 || first == 0) {
          __syncthreads();  // (the x of the block before is no longer read)
          stage_x<NT, kTurned>(p, xs, chunk0 * P, chunks * P, m0);
          __syncthreads();
        }
        // A sum of a tile over this block of k: kept for the next, or a result.
        auto emit = [&](int of, int o, float v) {
          if (kb > 0) v += kept[of * kSums + o];
          if (kb + 1 < p.blocks) kept[of * kSums + o] = v;
          else if (p.ksplit > 1) push_sum(others + rank * kSums + o, v);  // (into the cluster's first block)
          else write_sum(p, m0 + o / kRows, (int64_t)(block + (first + of) * blocks) * kRows + o % kRows, v);
        };
        float acc[kSub][NT][4] = {};
        int from = at;        // where in the tile this warp's part begins
        bool earlier = false;  // a part of another tile went before
        if (lane == 0) begun[warp] = -1;
        int s = 0;  // the ring's slot of the chunk
#pragma unroll 1
        for (int it = begin; it < end; it += H) {
#pragma unroll
          for (int u = 0; u < H; ++u) {
            if (it + u >= end) break;
            if (!kAligned) {
              asm volatile("cp.async.wait_group %0;" ::"n"(A - 1) : "memory");  // this lane's copies of the chunk have landed
              __syncwarp();
            } else {
              if (alive && !mbar_wait(&landed[warp][s], (parity >> s) & 1u)) {
                if (p.dev_status) atomicOr(p.dev_status, RGD_DEV_WAIT_TIMEOUT);
                alive = false;  // (no more copies; those on their way are waited for at the end)
                lost = s;
              }
              if (alive) {
                parity ^= 1u << s;
                --flying;
              }
            }
            const Scales<NL, kZeros> now = ahead[u];
            const bool apart = P == 2 && !p.scale_vec;  // (groups of 128: a lane has one of two parts of rows 16 i .. in load i)
            float own[NL];
            if constexpr (GS == 4) {
#pragma unroll
              for (int i = 0; i < NL; ++i) own[i] = scale_of(p, now, i);
            }
            if constexpr (GS < 4) {
              spread_scales<kEach>(p, now, scales, zeros, lane);
              __syncwarp();
            }
            load_next(ahead[u]);
            const uint8_t* slot = ring + s * L::kSlot;
#pragma unroll
            for (int c2 = 0; c2 < P; ++c2) {
              uint32_t q[R][4];
#pragma unroll
              for (int h = 0; h < R; ++h) {
                if (!kTurned) {
                  const uint4 v = *reinterpret_cast<const uint4*>(slot + c2 * kRows * 64 + h * 512 + lane * 16);
                  q[h][0] = v.x, q[h][1] = v.y, q[h][2] = v.z, q[h][3] = v.w;
                } else if (kAligned) {
#pragma unroll
                  for (int j = 0; j < 4; ++j)
                    q[h][j] = *reinterpret_cast<const uint32_t*>(slot + c2 * kRows * 64 + h * 512 + word_at[j]);
                } else {
#pragma unroll
                  for (int j = 0; j < 4; ++j) {
                    const uint32_t* w = reinterpret_cast<const uint32_t*>(slot + c2 * 64 + h * 8 * L::kPitch + word_at[j] + (cut[h] & ~3u));
                    q[h][j] = __funnelshift_r(w[0], w[1], 8 * (cut[h] & 3));
                  }
                }
              }
              if (c2 + 1 == P) {
                if (kAligned) fence_proxy_async_smem();  // (without it a read was put off until the copy had overwritten its place)
                __syncwarp();
                load(s);  // (over what the warp has just read)
              }
              float sc[R][L::kGroups];
              uint32_t z[R] = {};
#pragma unroll
              for (int h = 0; h < R; ++h) {
                const int row = 8 * h + (lane >> 2);
                if constexpr (GS == 4) {
                  const int from = apart ? row % 16 * 2 + c2 : row;
                  sc[h][0] = __shfl_sync(0xffffffffu, apart ? own[h / 2 % NL] : own[c2], from);
                  if constexpr (kZeros)
                    z[h] = __shfl_sync(0xffffffffu, apart ? now.z[h / 2 % NL] : p.scale_vec ? now.z[0] >> (8 * c2) : now.z[c2], from) & 15u;
                } else {
#pragma unroll
                  for (int g = 0; g < L::kGroups; ++g) sc[h][g] = scales[(c2 * kRows + row) * L::kGroups + g];
                  if constexpr (kZeros) {
                    const uint8_t* at = zeros + (c2 * kRows + row) * L::kGroups;
                    z[h] = (L::kGroups == 4 ? *reinterpret_cast<const uint32_t*>(at) : *reinterpret_cast<const uint16_t*>(at)) & 0x0f0f0f0fu;
                  }
                }
              }
              multiply_part<NT, GS, kZeros>(q, sc, z, my_x + (at * P + c2) * 4 * NT * unit, unit, acc, magic);
            }
            if (GS < 4) __syncwarp();  // (the scales have been read)
            s = s + 1 == A ? 0 : s + 1;
            if (++at < chunks && it + u + 1 < end) continue;
            // The end of the tile, or of what this warp has of it: then its first part goes into its
            // place for joins and its last one into its ring, which it no longer needs.
            const bool all = from == 0 && at == chunks && p.ksplit == 1;
            const int o0 = t * 2 * kRows + (lane >> 2);  // a lane's first sum
            float* to = all ? kept + tile * kSums : earlier ? reinterpret_cast<float*>(dyn + warp * A * L::kSlot) : join + warp * kSums;
            if (all && kb + 1 == p.blocks && p.ksplit == 1) {
              const int64_t n0 = (int64_t)(block + (first + tile) * blocks) * kRows + (lane >> 2);
#pragma unroll
              for (int i = 0; i < NT; ++i)
#pragma unroll
                for (int h = 0; h < 2 * kSub; ++h)
#pragma unroll
                  for (int e = 0; e < 2; ++e) {
                    float v = acc[h / 2][i][(h & 1) * 2 + e];
                    if (kb > 0) v += to[o0 + (i * 8 + e) * kRows + 8 * h];
                    write_sum(p, m0 + i * 8 + t * 2 + e, n0 + 8 * h, v);
                  }
            } else {
#pragma unroll
              for (int i = 0; i < NT; ++i)
#pragma unroll
                for (int h = 0; h < 2 * kSub; ++h)
#pragma unroll
                  for (int e = 0; e < 2; ++e) {
                    float& v = to[o0 + (i * 8 + e) * kRows + 8 * h];
                    v = (all && kb > 0 ? v : 0.f) + acc[h / 2][i][(h & 1) * 2 + e];
                  }
              if (!all && from == 0 && lane == 0) begun[warp] = earlier ? ~tile : tile;
            }
#pragma unroll
            for (int b = 0; b < kSub; ++b)
#pragma unroll
              for (int i = 0; i < NT; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[b][i][e] = 0.f;
            earlier = true;
            at = from = 0;
            ++tile;
          }
        }
        // The tiles that several warps had parts of, by the first of these warps.
        __syncthreads();
        constexpr int kAtOnce = kWarps * 32 / kSums;
        uint32_t owners = __ballot_sync(0xffffffffu, begun[lane % kWarps] != -1) & ((1u << kWarps) - 1);
        for (int i = 0; owners; ++i, owners &= owners - 1) {
          if (i % kAtOnce != (int)threadIdx.x / kSums) continue;
          const int w = __ffs(owners) - 1, o = threadIdx.x % kSums;
          int of = begun[w];
          const float* mp = of < 0 ? reinterpret_cast<const float*>(dyn + w * A * L::kSlot) : join + w * kSums;
          of = of < 0 ? ~of : of;
          float v = mp[o];
          const int stop = (of + 1) * chunks;
#pragma unroll
          for (int i = 1; i < kWarps; ++i) v += w + i < kWarps && (w + i) * per < stop ? join[(w + i) * kSums + o] : 0.f;
          emit(of, o, v);
        }
        if (chunks == 0)  // (a cluster's last block may have none in the last block of k)
          for (int o = threadIdx.x; o < batch * kSums; o += kWarps * 32) emit(o / kSums, o % kSums, 0.f);
        if (p.ksplit > 1 && kb + 1 == p.blocks) {  // (one tile)
          cluster_sync();
          if (rank == 0) {
            for (int o = threadIdx.x; o < kSums; o += kWarps * 32) {
              float v = 0.f;
              for (int r = 0; r < p.ksplit; ++r) v += others[r * kSums + o];
              write_sum(p, m0 + o / kRows, (int64_t)block * kRows + o % kRows, v);
            }
          }
          cluster_sync();
        }
        if (kb + 1 < p.blocks || first + batch < mine || m0 + 8 * NT < p.m) {
          if (kAligned) fence_proxy_async_smem();
          __syncthreads();  // (rings, sums kept and parts have been read)
        }
      }
    }
  }
  if (!kAligned) asm volatile("cp.async.wait_all;" ::: "memory");
  if (!alive)
    for (int i = 0; i < flying; ++i) mbar_wait(&landed[warp][(lost + i) % A], (parity >> (lost + i) % A) & 1u);
}

template <int NT, int GS, bool kAligned, bool kZeros>
int launch_w4_as(W4Params& p, cudaStream_t st) {
  static std::atomic<bool> done[kMaxDevices];
  using L = Layout<NT, GS, kAligned, kZeros>;
  auto k = w4_kernel<NT, GS, kAligned, kZeros>;
  if (int rc = ensure_smem(k, kW4Smem, done)) return rc;
  constexpr int W = kWarps, sms = 152;
  constexpr int sums = L::kSums * 4;  // bytes
  constexpr int room = kW4Smem - L::kFixed;
  static_assert(room - kMaxSplit * sums >= 4 * sums && room - room / 4 - kMaxSplit * sums >= 4 * kParts<NT, GS> * NT * 512, "a tile's sums and a block of k must fit");
  static_assert(kAhead * L::kSlot >= sums, "a part's sums must fit a warp's ring");
  p.scale_vec = p.groups % (kParts<NT, GS> * (GS == 4 ? 1 : L::kGroups)) == 0;
  // rows of x that are kept of every 8: a power of two
  p.x_shift = NT > 1 || p.m > 4 ? 3 : p.m > 2 ? 2 : p.m > 1 ? 1 : 0;
  const int x_bytes = 4 * kParts<NT, GS> * NT * (64 << p.x_shift);  // of a chunk
  const int tiles = (p.n + kRows - 1) / kRows;
  const int chunks = (p.k + kChunk<NT, GS> - 1) / kChunk<NT, GS>;
  // Few tiles of long rows: as many blocks to a tile as leave each warp a chunk.
  int split = 1;
  while (split < kMaxSplit && tiles * split * 2 <= sms && chunks >= split * 2 * W) split *= 2;
  p.ksplit = split;
  p.rank_chunks = (chunks + split - 1) / split;
  const int others = split > 1 ? split * sums : 0, left = room - others;
  const int grid = split > 1 ? tiles * split : std::min(tiles, sms);
  p.blocks = 1;
  p.block_chunks = p.rank_chunks;
  p.batch = 0x3fffffff;
  int smem = L::kFixed + others + p.rank_chunks * x_bytes;
  if (p.rank_chunks > left / x_bytes) {  // blocks of k, as even as they come: up to a quarter of the room keeps sums
    p.batch = split > 1 ? 1 : std::min(left / 4 / sums, (tiles + grid - 1) / grid);
    const int fits = (left - p.batch * sums) / x_bytes;
    p.blocks = (p.rank_chunks + fits - 1) / fits;
    p.block_chunks = (p.rank_chunks + p.blocks - 1) / p.blocks;
    p.blocks = (p.rank_chunks + p.block_chunks - 1) / p.block_chunks;
    smem = L::kFixed + others + p.batch * sums + p.block_chunks * x_bytes;
  }
  CUtensorMap map = {};
  if (kAligned) {
    const auto encode = tensor_map_encoder();
    if (!encode) return set_error(RGD_ERR_CUDA, "cuTensorMapEncodeTiled is unavailable");
    const cuuint64_t dims[2] = {(cuuint64_t)p.row_bytes, (cuuint64_t)p.n}, strides[1] = {(cuuint64_t)p.row_bytes};
    const cuuint32_t box[2] = {kPart / 2, kRows}, ones[2] = {1, 1};
    const CUresult r = encode(&map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<uint8_t*>(p.w), dims, strides, box, ones,
                              CU_TENSOR_MAP_INTERLEAVE_NONE, GS == 4 ? CU_TENSOR_MAP_SWIZZLE_NONE : CU_TENSOR_MAP_SWIZZLE_64B,
                              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) return set_error(RGD_ERR_CUDA, "cuTensorMapEncodeTiled failed (%d)", (int)r);
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)grid);
  cfg.blockDim = dim3(W * 32);
  cfg.dynamicSmemBytes = (size_t)smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim = {(unsigned)split, 1, 1};
  cfg.attrs = attr;
  cfg.numAttrs = split > 1 ? 2 : 1;
  cudaError_t e = cudaLaunchKernelEx(&cfg, k, p, map);
  if (e == cudaSuccess) e = cudaGetLastError();
  return e == cudaSuccess ? RGD_OK : cuda_error(e, "w4 launch");
}

template <int NT, int GS>
int launch_w4_steps(W4Params& p, cudaStream_t st) {
  if (p.row_bytes % 16 == 0) return p.zeros ? launch_w4_as<NT, GS, true, true>(p, st) : launch_w4_as<NT, GS, true, false>(p, st);
  return p.zeros ? launch_w4_as<NT, GS, false, true>(p, st) : launch_w4_as<NT, GS, false, false>(p, st);
}
template <int NT>
int launch_w4(W4Params& p, cudaStream_t st) {
  return p.group_shift == 5 ? launch_w4_steps<NT, 1>(p, st)
                            : p.group_shift == 6 ? launch_w4_steps<NT, 2>(p, st) : launch_w4_steps<NT, 4>(p, st);
}

}  // namespace
}  // namespace rgd
