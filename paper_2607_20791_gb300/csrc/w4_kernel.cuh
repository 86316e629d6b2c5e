// Products of a few rows of activations with 4-bit weights: y = x W^T with
// W[n, k] = (q[n, k] - z[n, k / G]) s[n, k / G], q packed two to a byte along k.
//
// The weights are read once; everything else is small.  A tile is 32 rows of W (16 above
// 16 rows of x); the warps of its group take the 128-weight chunks of those rows in turn,
// so that together they read contiguous bytes of a row.  A chunk is one
// TMA box of 64 bytes by the tile's rows into the warp's own ring in shared memory, 4 KB
// ahead of its use, read 16 bytes a lane (lane 4g + t: rows g, g + 8, ..., bytes 16t ..), and
// 8 mma.m16n8k16 with the weights as A for every 16 of its rows and 8 rows of x: one row
// costs the same as eight, and the tensor pipe does the sums over k in fp32.  (Rows off
// 16 bytes come by 4-byte asynchronous copies.)
//
// Which k a lane's A elements stand for is free as long as B agrees, so a lane feeds the
// 8 nibbles of a 32-bit word as they lie: nibbles p and p + 4 are the two halves of
// (word >> 4p) & 0x000f000f, and with 0x4300 over each (bf16 128) they are the bf16
// numbers 128 + q.  128 + z taken from them leaves q - z exactly.  x lies in shared memory
// in that order, one 16-byte load a lane for two MMAs.  With groups of 128 the four words
// of a 16-byte copy share a scale and go in as they are; with smaller groups an MMA's k
// must stay within 32 weights, so the quad's 4 x 4 words are transposed first.  A group's
// sum is scaled in fp32 after its last MMA.
//
// One block of 24 warps (16 above 8 rows of x) fills an SM, so that x lies there once.  Its
// warps form groups of S that share a tile and whose sums meet in shared memory: few tiles
// want a wide group, many a narrow one, whose joins cost less.  Where x does not fit, k goes
// in blocks, with the sums of a group's tiles kept in shared memory between them.
#pragma once

#include <cuda_bf16.h>

#include <algorithm>

#include "ptx.cuh"
#include "w4.h"

namespace rgd {
namespace {

constexpr int kPart = 128;   // weights of a row that a lane's quad holds at a time
constexpr int kUnit = 512;   // bytes of x per MMA step: 8 rows, 32 weights
constexpr int kW4Smem = 226 * 1024;  // (of 227; the barriers take the rest)

constexpr int kWarps = 16;   // of a block
// For 8 NT rows of x: groups of 16 rows of W in a tile, 128-weight parts of a chunk, chunks in flight.
template <int NT>
constexpr int kSub = NT == 4 ? 1 : 2;
template <int NT>
constexpr int kParts = NT == 1 ? 2 : 1;
template <int NT>
constexpr int kAhead = NT == 4 ? 4 : 2;
template <int NT>
constexpr int kChunk = kPart * kParts<NT>;
// Bytes of 8 rows of a chunk in a warp's ring; rows off 16 bytes come as the five words that hold a lane's 16 bytes.
template <bool kAligned>
constexpr int kPiece = kAligned ? 512 : 640;

__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
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

__device__ __forceinline__ void copy4(uint32_t dst, const void* src, int bytes) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy_box(uint32_t dst, const CUtensorMap* map, int32_t x, int32_t y, uint64_t* bar) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
               "l"(map), "r"(x), "r"(y), "r"(smem_u32(bar))
               : "memory");
}

// A chunk's scales and zeros as they lie in memory (a load must not be waited for before its
// use).  Lane i has those of row i of the tile (of row i - 16 for the second half of k in a
// tile of 16 rows): one of every 128 weights, or of every 32 where groups are smaller.
template <int NL, bool kZeros>
struct Scales {
  uint32_t s[NL], z[kZeros ? NL : 1];
};

template <int kRows, int kParts, int NL, bool kSmallGroups, bool kZeros>
__device__ __forceinline__ void load_scales(const W4Params& p, Scales<NL, kZeros>& c, const uint8_t* row_scales,
                                            const uint8_t* row_zeros, int chunk, int lane) {
  constexpr int kEach = NL / kParts;
#pragma unroll
  for (int i = 0; i < NL; ++i) {
    const int k = (chunk * kParts + i / kEach) * kPart + (kSmallGroups ? (lane / kRows * kEach + i % kEach) * 32 : 0);
    const int g = min(k >> p.group_shift, p.groups - 1);  // (weights past the row's end meet zeros of x)
    if (p.scale_bytes == 2) c.s[i] = __ldg(reinterpret_cast<const uint16_t*>(row_scales) + g);
    else c.s[i] = __ldg(reinterpret_cast<const uint32_t*>(row_scales) + g);
    if (kZeros) c.z[i] = __ldg(row_zeros + g);
  }
}

// Rows off 16 bytes: starts the copies of the words that hold the lane's 16 bytes of rows
// g, g + 8, ... of a part.  Nothing is read past the weights' end or for rows past the
// last: those bytes are filled with zeros.
template <int R>
__device__ __forceinline__ void copy_words(const W4Params& p, uint32_t to, int tile, int part, int lane) {
  const int64_t n = (int64_t)tile * (8 * R) + (lane >> 2);
  const int off = part * (kPart / 2) + (lane & 3) * 16;
#pragma unroll
  for (int h = 0; h < R; ++h) {
    const bool has = n + 8 * h < p.n && off < (int)p.row_bytes;
    const int64_t at = (has ? (n + 8 * h) * p.row_bytes + off : 0) & ~int64_t(3);
#pragma unroll
    for (int i = 0; i < 5; ++i) {
      const int64_t left = p.total_bytes - (at + 4 * i);
      const int bytes = !has || left <= 0 ? 0 : left < 4 ? (int)left : 4;
      copy4(to + h * 640 + i * 128 + lane * 4, p.w + (bytes ? at + 4 * i : 0), bytes);
    }
  }
}

// A lane's 32 weights of row h out of the ring.  `shift`: bits that the row's bytes lie past a word's start.
template <bool kAligned>
__device__ __forceinline__ uint4 chunk_row(const uint8_t* slot, int h, uint32_t shift, int lane) {
  if (kAligned) return *reinterpret_cast<const uint4*>(slot + h * 512 + lane * 16);
  uint32_t u[5];
#pragma unroll
  for (int i = 0; i < 5; ++i) u[i] = *reinterpret_cast<const uint32_t*>(slot + h * 640 + i * 128 + lane * 4);
  return make_uint4(__funnelshift_r(u[0], u[1], shift), __funnelshift_r(u[1], u[2], shift),
                    __funnelshift_r(u[2], u[3], shift), __funnelshift_r(u[3], u[4], shift));
}

// The quad's 4 x 4 words transposed: lane t gets word t of each of its lanes.
__device__ __forceinline__ void transpose_quad(uint4& v, int t) {
  uint32_t w[4] = {v.x, v.y, v.z, v.w};
  const bool odd = t & 1, high = t & 2;
#pragma unroll
  for (int i = 0; i < 4; i += 2) {  // words i and i + 1 with lane ^ 1
    const uint32_t other = __shfl_xor_sync(0xffffffffu, odd ? w[i] : w[i + 1], 1);
    (odd ? w[i] : w[i + 1]) = other;
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {  // words i and i + 2 with lane ^ 2
    const uint32_t other = __shfl_xor_sync(0xffffffffu, high ? w[i] : w[i + 2], 2);
    (high ? w[i] : w[i + 2]) = other;
  }
  v = make_uint4(w[0], w[1], w[2], w[3]);
}

// Adds the products of 16 rows' chunk (a lane's weights of rows g and g + 8, rows `sub` ..
// of the tile) to their sums.  s and z: the tile's scales and biases by lane, the chunk's part's
// from `first` on.
template <int NT, int kRows, int NL, bool kSmallGroups, bool kZeros>
__device__ __forceinline__ void multiply_rows(uint4 q0, uint4 q1, const float (&s)[NL], const uint32_t (&z)[kZeros ? NL : 1],
                                              int first, int sub, const uint8_t* xs, float (&acc)[NT][4], uint32_t magic, int lane) {
  if (kSmallGroups) {
    transpose_quad(q0, lane & 3);
    transpose_quad(q1, lane & 3);
  }
  float sum[NT][4], t0 = 0.f, t1 = 0.f;
  uint32_t b0 = 0x43084308u, b1 = 0x43084308u;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t lo = j == 0 ? q0.x : j == 1 ? q0.y : j == 2 ? q0.z : q0.w;
    const uint32_t hi = j == 0 ? q1.x : j == 1 ? q1.y : j == 2 ? q1.z : q1.w;
    if (kSmallGroups || j == 0) {
      constexpr int kEach = NL / kParts<NT>;
      const int from = sub + (lane >> 2) + (kSmallGroups ? j / kEach * kRows : 0), i = first + (kSmallGroups ? j % kEach : 0);
      t0 = __shfl_sync(0xffffffffu, s[i], from);
      t1 = __shfl_sync(0xffffffffu, s[i], from + 8);
      if (kZeros) {
        b0 = __shfl_sync(0xffffffffu, z[kZeros ? i : 0], from);
        b1 = __shfl_sync(0xffffffffu, z[kZeros ? i : 0], from + 8);
      }
    }
    uint32_t a[4], b[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      a[q] = weights2(lo, q, magic, b0);
      b[q] = weights2(hi, q, magic, b1);
    }
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      if (kSmallGroups || j == 0)
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[i][e] = 0.f;
      const uint4 x = *reinterpret_cast<const uint4*>(xs + (j * NT + i) * kUnit + lane * 16);
      mma16816(sum[i], a[0], b[0], a[1], b[1], x.x, x.y);
      mma16816(sum[i], a[2], b[2], a[3], b[3], x.z, x.w);
      if (kSmallGroups || j == 3) {
        acc[i][0] = fmaf(t0, sum[i][0], acc[i][0]);
        acc[i][1] = fmaf(t0, sum[i][1], acc[i][1]);
        acc[i][2] = fmaf(t1, sum[i][2], acc[i][2]);
        acc[i][3] = fmaf(t1, sum[i][3], acc[i][3]);
      }
    }
  }
}

// A block of x into shared memory, 8 numbers a lane and step, in the order of the nibbles.
template <int NT, bool kSmallGroups>
__device__ __forceinline__ void stage_x(const W4Params& p, uint8_t* xs, int part0, int parts, int m0) {
  constexpr int kThreads = kWarps * 32, kBatch = 8;  // (loads in flight)
  const int units = parts * 4 * NT * 32;
  for (int u0 = threadIdx.x; u0 < units; u0 += kThreads * kBatch) {
    uint4 r[kBatch];
#pragma unroll
    for (int f = 0; f < kBatch; ++f) {
      const int u = u0 + f * kThreads;
      const int lane = u & 31, i = (u >> 5) % NT, j = (u >> 5) / NT & 3, c = (u >> 5) / (NT * 4);
      const int t = lane & 3, m = m0 + i * 8 + (lane >> 2);
      const int k = (part0 + c) * kPart + (kSmallGroups ? j * 32 + t * 8 : t * 32 + j * 8);
      r[f] = make_uint4(0, 0, 0, 0);
      if (u < units && m < p.m && k < p.k) {
        const uint16_t* src = p.x + (int64_t)m * p.k + k;
        if (p.x_vec) {  // (k is then a multiple of 8)
          r[f] = __ldg(reinterpret_cast<const uint4*>(src));
        } else {
          uint16_t e[8];
#pragma unroll
          for (int b = 0; b < 8; ++b) e[b] = k + b < p.k ? __ldg(src + b) : 0;
          r[f] = make_uint4(e[0] | (uint32_t)e[1] << 16, e[2] | (uint32_t)e[3] << 16, e[4] | (uint32_t)e[5] << 16,
                            e[6] | (uint32_t)e[7] << 16);
        }
      }
    }
#pragma unroll
    for (int f = 0; f < kBatch; ++f) {
      const int u = u0 + f * kThreads;
      if (u < units)
        *reinterpret_cast<uint4*>(xs + (int64_t)u * 16) =
            make_uint4(__byte_perm(r[f].x, r[f].z, 0x5410), __byte_perm(r[f].x, r[f].z, 0x7632),
                       __byte_perm(r[f].y, r[f].w, 0x5410), __byte_perm(r[f].y, r[f].w, 0x7632));
    }
  }
}

// The threads of a group of warps wait for one another.
__device__ __forceinline__ void group_barrier(int group, int warps) {
  asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(warps * 32) : "memory");
}

// Shared memory: the warps' rings, every warp's sums of a tile, the sums kept between blocks of k, x.
template <int NT, bool kAligned>
struct Layout {
  static constexpr int kRows = 16 * kSub<NT>;   // of a tile
  static constexpr int kSums = kRows * 8 * NT;
  static constexpr int kJoin = kWarps * kSums * 4;
  static constexpr int kPartBytes = 2 * kSub<NT> * kPiece<kAligned>;
  static constexpr int kSlot = kParts<NT> * kPartBytes;
  static constexpr int kRing = kWarps * kAhead<NT> * kSlot;
};

template <int NT, bool kSmallGroups, bool kAligned, bool kZeros>
__global__ void __launch_bounds__(kWarps * 32, 1) w4_kernel(const W4Params p, const __grid_constant__ CUtensorMap map) {
  using L = Layout<NT, kAligned>;
  constexpr int kSums = L::kSums, kRows = L::kRows, R = kRows / 8, A = kAhead<NT>, P = kParts<NT>;
  constexpr int NL = P * (kSmallGroups ? kRows / 8 : 1);
  extern __shared__ __align__(128) uint8_t dyn[];
  __shared__ uint64_t landed[kWarps][A];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int S = p.split, groups = kWarps / S, group = warp / S, member = warp % S;
  const uint8_t* ring = dyn + warp * A * L::kSlot;
  float* part = reinterpret_cast<float*>(dyn + L::kRing) + group * S * kSums;                   // [S][kSums]
  float* kept = reinterpret_cast<float*>(dyn + L::kRing + L::kJoin) + group * p.batch * kSums;  // [batch][kSums]
  uint8_t* xs = dyn + L::kRing + L::kJoin + (p.blocks > 1 ? groups * p.batch * kSums * 4 : 0);
  if (kAligned && lane == 0) {
#pragma unroll
    for (int s = 0; s < A; ++s) mbar_init(&landed[warp][s], 1);
    fence_mbar_init();
    fence_proxy_async_smem();
  }
  __syncwarp();
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");  // (a dependent waits for this kernel's end)
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int tiles = (p.n + kRows - 1) / kRows;
  // group g of block b takes tiles b + gridDim g, then every (gridDim groups)-th
  const int tile0 = (int)blockIdx.x + group * (int)gridDim.x, stride = (int)gridDim.x * groups;
  const int mine = tile0 < tiles ? (tiles - tile0 + stride - 1) / stride : 0;
  const int most = (int)blockIdx.x < tiles ? (tiles - (int)blockIdx.x + stride - 1) / stride : 0;  // of any group here
  const int scale_shift = p.scale_bytes == 2 ? 16 : 0;
  const uint32_t ring_at = smem_u32(ring), magic = exponent_bits();
  uint32_t parity = 0;  // of each slot's barrier
  int flying = 0, lost = 0;  // copies on their way, and the slot of the oldest once a wait has given up
  bool alive = true;    // no wait has given up
  for (int m0 = 0; m0 < p.m; m0 += 8 * NT) {
    for (int first = 0; first < most; first += p.batch) {
      const int batch = max(0, min(p.batch, mine - first));
      for (int kb = 0; kb < p.blocks; ++kb) {
        const int chunk0 = kb * p.block_chunks;
        const int chunks = min(p.block_chunks, (p.k + kChunk<NT> - 1) / kChunk<NT> - chunk0);
        const int per = (chunks - member + S - 1) / S;  // chunks of this warp and a tile (none: the group's others have them)
        const int items = batch * max(per, 1);
        Scales<NL, kZeros> c[A];
        // the next chunk to load, its tile, and the scales and zeros of the lane's row (of the last row for those past it)
        int lt = 0, lc = member, load_tile = tile0 + first * stride;
        const uint8_t *row_scales, *row_zeros;
        auto at_row = [&] {
          const int64_t g = min((int64_t)load_tile * kRows + lane % kRows, (int64_t)p.n - 1) * p.groups;
          row_scales = p.scales + g * p.scale_bytes;
          row_zeros = p.zeros + g;
        };
        at_row();
        auto load = [&](Scales<NL, kZeros>& into, int s) {
          if (lt < batch && lc < chunks) {
            if (!kAligned) {
              for (int c2 = 0; c2 < P; ++c2)
                copy_words<R>(p, ring_at + s * L::kSlot + c2 * L::kPartBytes, load_tile, (chunk0 + lc) * P + c2, lane);
            } else if (lane == 0 && alive) {
              mbar_arrive_expect_tx(&landed[warp][s], L::kSlot);
#pragma unroll
              for (int c2 = 0; c2 < P; ++c2)  // (a part past the row's end is filled with zeros)
                copy_box(ring_at + s * L::kSlot + c2 * L::kPartBytes, &map, ((chunk0 + lc) * P + c2) * (kPart / 2),
                         load_tile * kRows, &landed[warp][s]);
            }
            if (kAligned && alive) ++flying;
            load_scales<kRows, P, NL, kSmallGroups, kZeros>(p, into, row_scales, row_zeros, chunk0 + lc, lane);
          }
          if (!kAligned) asm volatile("cp.async.commit_group;" ::: "memory");
          lc += S;
          if (lc < chunks) return;
          lc = member;
          ++lt;
          load_tile += stride;
          at_row();
        };
#pragma unroll
        for (int s = 0; s < A; ++s) load(c[s], s);
        if (p.blocks > 1 || first == 0) {
          __syncthreads();  // (the x of the block before is no longer read)
          stage_x<NT, kSmallGroups>(p, xs, chunk0 * P, chunks * P, m0);
          __syncthreads();
        }
        float acc[kSub<NT>][NT][4] = {};
        int tile = 0, at = member;
        for (int it = 0; it < items; it += A) {
#pragma unroll
          for (int s = 0; s < A; ++s) {
            if (it + s >= items) break;
            if (at < chunks) {
              uint32_t shift = 0;  // (the same for all of a lane's rows, which are 8 apart)
              if (kAligned) {
                if (alive && !mbar_wait(&landed[warp][s], (parity >> s) & 1u)) {
                  if (p.dev_status) atomicOr(p.dev_status, RGD_DEV_WAIT_TIMEOUT);
                  alive = false;  // (no more copies; those on their way are waited for at the end)
                  lost = s;
                }
                if (alive) {
                  parity ^= 1u << s;
                  --flying;
                }
              } else {
                asm volatile("cp.async.wait_group %0;" ::"n"(A - 1) : "memory");  // this lane's copies of the chunk have landed
                shift = (uint32_t)(((int64_t)(tile0 + (first + tile) * stride) * kRows + (lane >> 2)) * p.row_bytes & 3) * 8;
              }
              uint4 q[P][R];
#pragma unroll
              for (int c2 = 0; c2 < P; ++c2)
#pragma unroll
                for (int h = 0; h < R; ++h)
                  q[c2][h] = chunk_row<kAligned>(ring + s * L::kSlot + c2 * L::kPartBytes, h, shift, lane);
              float sc[NL];
              uint32_t z[kZeros ? NL : 1];
#pragma unroll
              for (int i = 0; i < NL; ++i) {
                sc[i] = __uint_as_float(c[s].s[i] << scale_shift);
                if (kZeros) z[i] = 0x43004300u + 0x00010001u * (c[s].z[i] & 15u);
              }
              __syncwarp();
              load(c[s], s);  // (over what the warp has just read)
#pragma unroll
              for (int c2 = 0; c2 < P; ++c2)
#pragma unroll
                for (int b = 0; b < kSub<NT>; ++b)
                  multiply_rows<NT, kRows, NL, kSmallGroups, kZeros>(q[c2][2 * b], q[c2][2 * b + 1], sc, z, c2 * (NL / P), 16 * b,
                                                                     xs + (int64_t)(at * P + c2) * 4 * NT * kUnit, acc[b],
                                                                     magic, lane);
            } else {
              load(c[s], s);
            }
            at += S;
            if (at < chunks) continue;
            // the tile's sums: this warp's, once the group has read those of the tile before, then all of them
            group_barrier(group, S);
            float* mp = part + member * kSums + (lane & 3) * 2 * kRows + (lane >> 2);
#pragma unroll
            for (int b = 0; b < kSub<NT>; ++b)
#pragma unroll
              for (int i = 0; i < NT; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  mp[(i * 8 + (e & 1)) * kRows + b * 16 + (e >> 1) * 8] = acc[b][i][e];
                  acc[b][i][e] = 0.f;
                }
            group_barrier(group, S);
            for (int o = member * 32 + lane; o < kSums; o += S * 32) {
              float v = kb > 0 ? kept[tile * kSums + o] : 0.f;
#pragma unroll 4
              for (int w = 0; w < S; ++w) v += part[w * kSums + o];
              if (kb + 1 < p.blocks) {
                kept[tile * kSums + o] = v;
                continue;
              }
              const int m = m0 + o / kRows;
              const int64_t n = (int64_t)(tile0 + (first + tile) * stride) * kRows + o % kRows;
              if (m >= p.m || n >= p.n) continue;
              if (p.out_f32) static_cast<float*>(p.y)[m * p.y_stride + n] = v;
              else static_cast<__nv_bfloat16*>(p.y)[m * p.y_stride + n] = __float2bfloat16(v);
            }
            at = member;
            ++tile;
          }
        }
      }
    }
  }
  if (!kAligned) asm volatile("cp.async.wait_all;" ::: "memory");
  if (!alive)
    for (int i = 0; i < flying; ++i) mbar_wait(&landed[warp][(lost + i) % A], (parity >> (lost + i) % A) & 1u);
}

template <int NT, bool kSmallGroups, bool kAligned, bool kZeros>
int launch_w4_as(W4Params& p, cudaStream_t st) {
  static std::atomic<bool> done[kMaxDevices];
  using L = Layout<NT, kAligned>;
  auto k = w4_kernel<NT, kSmallGroups, kAligned, kZeros>;
  if (int rc = ensure_smem(k, kW4Smem, done)) return rc;
  constexpr int W = kWarps, sms = 152;
  constexpr int sums = L::kSums * 4;        // bytes
  constexpr int x_bytes = 4 * kParts<NT> * NT * kUnit;  // of a chunk
  constexpr int room = kW4Smem - L::kJoin - L::kRing;
  const int tiles = (p.n + L::kRows - 1) / L::kRows;
  const int chunks = (p.k + kChunk<NT> - 1) / kChunk<NT>;
  static_assert(room / 4 >= W / 4 * sums, "a tile of each group must be kept");
  static_assert(room - room / 4 >= x_bytes * 4, "a block of k must fit");
  // (a block of a group's width of k has to fit)
  int S = tiles <= sms ? W : tiles <= 4 * sms ? 8 : 4;
  while (S * x_bytes > room - room / 4) S /= 2;
  p.split = S;
  const int groups = W / S;
  const int whole = (chunks + S - 1) / S * S;
  p.blocks = 1;
  p.block_chunks = whole;
  p.batch = 0x3fffffff;
  int smem = L::kJoin + L::kRing + whole * x_bytes;
  if (whole > room / x_bytes) {  // blocks of k, as even as they come: a quarter of the room keeps sums
    p.batch = std::max(1, room / 4 / (groups * sums));
    const int fits = (room - p.batch * groups * sums) / (x_bytes * S) * S;
    p.blocks = (chunks + fits - 1) / fits;
    p.block_chunks = ((chunks + p.blocks - 1) / p.blocks + S - 1) / S * S;
    p.blocks = (chunks + p.block_chunks - 1) / p.block_chunks;
    smem = L::kJoin + L::kRing + p.batch * groups * sums + p.block_chunks * x_bytes;
  }
  CUtensorMap map = {};
  if (kAligned) {
    const auto encode = tensor_map_encoder();
    if (!encode) return set_error(RGD_ERR_CUDA, "cuTensorMapEncodeTiled is unavailable");
    const cuuint64_t dims[2] = {(cuuint64_t)p.row_bytes, (cuuint64_t)p.n}, strides[1] = {(cuuint64_t)p.row_bytes};
    const cuuint32_t box[2] = {kPart / 2, L::kRows}, ones[2] = {1, 1};
    const CUresult r = encode(&map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<uint8_t*>(p.w), dims, strides, box, ones,
                              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) return set_error(RGD_ERR_CUDA, "cuTensorMapEncodeTiled failed (%d)", (int)r);
  }
  const cudaError_t e = launch_dependent(k, std::min(tiles, sms), W * 32, smem, st, p, map);
  return e == cudaSuccess ? RGD_OK : cuda_error(e, "w4 launch");
}

template <int NT, bool kSmallGroups, bool kAligned>
int launch_w4_zeros(W4Params& p, cudaStream_t st) {
  return p.zeros ? launch_w4_as<NT, kSmallGroups, kAligned, true>(p, st)
                 : launch_w4_as<NT, kSmallGroups, kAligned, false>(p, st);
}
template <int NT>
int launch_w4(W4Params& p, cudaStream_t st) {
  const bool small = p.group_shift < 7, aligned = p.row_bytes % 16 == 0;
  if (small) return aligned ? launch_w4_zeros<NT, true, true>(p, st) : launch_w4_zeros<NT, true, false>(p, st);
  return aligned ? launch_w4_zeros<NT, false, true>(p, st) : launch_w4_zeros<NT, false, false>(p, st);
}

}  // namespace
}  // namespace rgd
