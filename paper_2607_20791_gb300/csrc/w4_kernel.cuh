// Products of a few rows of activations with 4-bit weights: y = x W^T with
// W[n, k] = (q[n, k] - z[n, k / G]) s[n, k / G], q packed two to a byte along k.
//
// The weights are read once; everything else is small.  A tile is 32 rows of W (16 above
// 16 rows of x); the warps of its group take the 128-weight chunks of those rows in turn,
// so that together they read contiguous bytes of a row.  A chunk is one 16-byte
// asynchronous copy a lane and 8 rows (lane 4g + t: rows g, g + 8, ..., bytes 16t ..) into the
// lane's own place in shared memory, 4 KB a warp ahead of their use, and 8
// mma.m16n8k16 with the weights as A for every 16 of its rows and 8 rows of x: one row
// costs the same as eight, and the tensor pipe does the sums over k in fp32.
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

constexpr int kChunk = 128;  // weights of a row per chunk
constexpr int kNoChunk = kW4MaxK / kChunk;  // past every row's end
constexpr int kUnit = 512;   // bytes of x per MMA step: 8 rows, 32 weights
constexpr int kW4Smem = 226 * 1024;

// For 8 NT rows of x: warps of a block, groups of 16 rows of W in a tile, chunks in flight.
template <int NT>
constexpr int kWarps = NT == 1 ? 24 : 16;
template <int NT>
constexpr int kSub = NT == 4 ? 1 : 2;
template <int NT>
constexpr int kAhead = NT == 4 ? 4 : 2;
// Bytes of 8 rows of a chunk in a warp's ring; rows off 16 bytes come as the five words that hold a lane's 16 bytes.
template <bool kAligned>
constexpr int kPiece = kAligned ? 512 : 640;

__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Nibbles p and p + 4 of a word as bf16 q - z (bias: 128 + z twice).
__device__ __forceinline__ uint32_t weights2(uint32_t word, int p, uint32_t bias) {
  const uint32_t u = ((word >> (4 * p)) & 0x000f000fu) | 0x43004300u;
  const __nv_bfloat162 v = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&u), *reinterpret_cast<const __nv_bfloat162*>(&bias));
  return *reinterpret_cast<const uint32_t*>(&v);
}

__device__ __forceinline__ void copy16(uint32_t dst, const void* src, int bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy4(uint32_t dst, const void* src, int bytes) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}

// A chunk's scales and zeros, of one group of each of a lane's rows, as they lie in memory (a
// load must not be waited for before its use).
template <int R, bool kZeros>
struct Scales {
  uint32_t s[R], z[kZeros ? R : 1];
};

// Where a lane's rows of a tile lie: row g of the tile, and how many of its rows g, g + 8, ... there are.
struct Rows {
  const uint8_t* w;  // the lane's first 16 bytes of chunk 0
  int64_t group;     // the row's first group
  int32_t count;
};
template <int R>
__device__ __forceinline__ Rows rows_of(const W4Params& p, int tile, int lane) {
  const int64_t n = (int64_t)tile * (8 * R) + (lane >> 2);
  Rows r;
  r.count = n < p.n ? (int)min((p.n - n + 7) / 8, (int64_t)R) : 0;
  r.w = p.w + n * p.row_bytes + (lane & 3) * 16;
  r.group = n * p.groups;
  return r;
}

// Starts the copy of a lane's part of a chunk into the ring slot at `to`.  Nothing is
// read past the weights' end: a copy's bytes there are filled with zeros.
template <int R, bool kSmallGroups, bool kAligned, bool kZeros>
__device__ __forceinline__ void load_chunk(const W4Params& p, Scales<R, kZeros>& c, uint32_t to, const Rows& r, int chunk,
                                           int lane) {
  const int off = chunk * (kChunk / 2);
  // (a group of the whole chunk is every lane's, also of those past the row's end)
  const int k = chunk * kChunk + (kSmallGroups ? (lane & 3) * 32 : 0);
  const int some = k < p.k ? r.count : 0, all = off + (lane & 3) * 16 < (int)p.row_bytes ? r.count : 0;
  const uint8_t* w = r.w + off;
  const int64_t g = r.group + (k >> p.group_shift);
  const uint8_t* s = p.scales + g * p.scale_bytes;
  const int64_t row_step = 8 * p.row_bytes;
  const int group_step = 8 * p.groups, scale_step = group_step * p.scale_bytes;
#pragma unroll
  for (int h = 0; h < R; ++h) {
    const uint8_t* src = w + h * row_step;
    if (kAligned) {
      copy16(to + h * 512 + lane * 16, h < all ? src : p.w, h < all ? 16 : 0);
    } else {
      const int64_t at = (h < all ? src - p.w : 0) & ~int64_t(3);
#pragma unroll
      for (int i = 0; i < 5; ++i) {
        const int64_t left = p.total_bytes - (at + 4 * i);
        const int bytes = h >= all || left <= 0 ? 0 : left < 4 ? (int)left : 4;
        copy4(to + h * 640 + i * 128 + lane * 4, p.w + (bytes ? at + 4 * i : 0), bytes);
      }
    }
    c.s[h] = 0;
    if (kZeros) c.z[h] = 0;
    if (h < some) {
      if (p.scale_bytes == 2) c.s[h] = __ldg(reinterpret_cast<const uint16_t*>(s + (int64_t)h * scale_step));
      else c.s[h] = __ldg(reinterpret_cast<const uint32_t*>(s + (int64_t)h * scale_step));
      if (kZeros) c.z[h] = __ldg(p.zeros + g + (int64_t)h * group_step);
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

// Adds the products of 16 rows' chunk (a lane's weights of rows g and g + 8) to their sums.
template <int NT, bool kSmallGroups>
__device__ __forceinline__ void multiply_rows(uint4 q0, uint4 q1, float s0, float s1, uint32_t z0, uint32_t z1,
                                              const uint8_t* xs, float (&acc)[NT][4], int lane) {
  if (kSmallGroups) {
    transpose_quad(q0, lane & 3);
    transpose_quad(q1, lane & 3);
  }
  float sum[NT][4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t lo = j == 0 ? q0.x : j == 1 ? q0.y : j == 2 ? q0.z : q0.w;
    const uint32_t hi = j == 0 ? q1.x : j == 1 ? q1.y : j == 2 ? q1.z : q1.w;
    float t0 = s0, t1 = s1;
    uint32_t b0 = z0, b1 = z1;
    if (kSmallGroups) {  // (the group of these 32 weights is lane j's of the quad)
      const int from = (lane & ~3) | j;
      t0 = __shfl_sync(0xffffffffu, s0, from);
      t1 = __shfl_sync(0xffffffffu, s1, from);
      b0 = __shfl_sync(0xffffffffu, z0, from);
      b1 = __shfl_sync(0xffffffffu, z1, from);
    }
    uint32_t a[4], b[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      a[q] = weights2(lo, q, b0);
      b[q] = weights2(hi, q, b1);
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
__device__ __forceinline__ void stage_x(const W4Params& p, uint8_t* xs, int chunk0, int chunks, int m0) {
  for (int u = threadIdx.x; u < chunks * 4 * NT * 32; u += kWarps<NT> * 32) {
    const int lane = u & 31, i = (u >> 5) % NT, j = (u >> 5) / NT & 3, c = (u >> 5) / (NT * 4);
    const int t = lane & 3, m = m0 + i * 8 + (lane >> 2);
    const int64_t k = (int64_t)(chunk0 + c) * kChunk + (kSmallGroups ? j * 32 + t * 8 : t * 32 + j * 8);
    uint4 v = make_uint4(0, 0, 0, 0);
    if (m < p.m && k < p.k) {
      const uint16_t* src = p.x + (int64_t)m * p.k + k;
      uint16_t e[8];
      if (p.x_vec) {  // (k is then a multiple of 8)
        const uint4 r = __ldg(reinterpret_cast<const uint4*>(src));
        const uint32_t q[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int b = 0; b < 8; ++b) e[b] = (uint16_t)(b & 1 ? q[b / 2] >> 16 : q[b / 2] & 0xffffu);
      } else {
#pragma unroll
        for (int b = 0; b < 8; ++b) e[b] = k + b < p.k ? __ldg(src + b) : 0;
      }
      v = make_uint4(e[0] | (uint32_t)e[4] << 16, e[1] | (uint32_t)e[5] << 16, e[2] | (uint32_t)e[6] << 16,
                     e[3] | (uint32_t)e[7] << 16);
    }
    *reinterpret_cast<uint4*>(xs + (int64_t)u * 16) = v;
  }
}

// The threads of a group of warps wait for one another.
__device__ __forceinline__ void group_barrier(int group, int warps) {
  asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(warps * 32) : "memory");
}

// Shared memory: every warp's sums of a tile, the sums kept between blocks of k, the warps' rings, x.
template <int NT, bool kAligned>
struct Layout {
  static constexpr int kRows = 16 * kSub<NT>;   // of a tile
  static constexpr int kSums = kRows * 8 * NT;
  static constexpr int kPart = kWarps<NT> * kSums * 4;
  static constexpr int kSlot = 2 * kSub<NT> * kPiece<kAligned>;
  static constexpr int kRing = kWarps<NT> * kAhead<NT> * kSlot;
};

template <int NT, bool kSmallGroups, bool kAligned, bool kZeros>
__global__ void __launch_bounds__(kWarps<NT> * 32, 1) w4_kernel(const W4Params p) {
  using L = Layout<NT, kAligned>;
  constexpr int kSums = L::kSums, kRows = L::kRows, R = kRows / 8, A = kAhead<NT>;
  extern __shared__ __align__(16) uint8_t dyn[];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int S = p.split, groups = kWarps<NT> / S, group = warp / S, member = warp % S;
  float* part = reinterpret_cast<float*>(dyn) + group * S * kSums;  // [S][kSums]
  const uint8_t* ring = dyn + L::kPart + warp * A * L::kSlot;
  float* kept = reinterpret_cast<float*>(dyn + L::kPart + L::kRing) + group * p.batch * kSums;  // [batch][kSums]
  uint8_t* xs = dyn + L::kPart + L::kRing + (p.blocks > 1 ? groups * p.batch * kSums * 4 : 0);
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");  // (a dependent waits for this kernel's end)
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int tiles = (p.n + kRows - 1) / kRows;
  // group g of block b takes tiles b + gridDim g, then every (gridDim groups)-th
  const int tile0 = (int)blockIdx.x + group * (int)gridDim.x, stride = (int)gridDim.x * groups;
  const int mine = tile0 < tiles ? (tiles - tile0 + stride - 1) / stride : 0;
  const int most = (int)blockIdx.x < tiles ? (tiles - (int)blockIdx.x + stride - 1) / stride : 0;  // of any group here
  const int scale_shift = p.scale_bytes == 2 ? 16 : 0;
  const uint32_t ring_at = smem_u32(ring);
  for (int m0 = 0; m0 < p.m; m0 += 8 * NT) {
    for (int first = 0; first < most; first += p.batch) {
      const int batch = max(0, min(p.batch, mine - first));
      for (int kb = 0; kb < p.blocks; ++kb) {
        const int chunk0 = kb * p.block_chunks;
        const int chunks = min(p.block_chunks, (p.k + kChunk - 1) / kChunk - chunk0);
        const int per = (chunks + S - 1) / S;  // chunks of a warp and tile
        const int items = batch * per;
        Scales<R, kZeros> c[A];
        int lt = 0, lc = member;  // the next chunk to load: tile of the batch, chunk of the tile
        Rows rows = rows_of<R>(p, tile0 + first * stride, lane);
        auto load = [&](Scales<R, kZeros>& into, int s) {
          load_chunk<R, kSmallGroups, kAligned, kZeros>(p, into, ring_at + s * L::kSlot, rows,
                                                        lt < batch && lc < chunks ? chunk0 + lc : kNoChunk, lane);
          asm volatile("cp.async.commit_group;" ::: "memory");
          lc += S;
          if (lc < per * S) return;
          lc = member;
          ++lt;
          rows = rows_of<R>(p, tile0 + (first + lt) * stride, lane);
        };
#pragma unroll
        for (int s = 0; s < A; ++s) load(c[s], s);
        if (p.blocks > 1 || first == 0) {
          __syncthreads();  // (the x of the block before is no longer read)
          stage_x<NT, kSmallGroups>(p, xs, chunk0, per * S, m0);
          __syncthreads();
        }
        float acc[kSub<NT>][NT][4] = {};
        int tile = 0, at = member;
        for (int it = 0; it < items; it += A) {
#pragma unroll
          for (int s = 0; s < A; ++s) {
            if (it + s >= items) break;
            uint32_t shift = 0;  // (the same for all of a lane's rows, which are 8 apart)
            if (!kAligned)
              shift = (uint32_t)(((int64_t)(tile0 + (first + tile) * stride) * kRows + (lane >> 2)) * p.row_bytes & 3) * 8;
            asm volatile("cp.async.wait_group %0;" ::"n"(A - 1) : "memory");  // this lane's copy of the chunk has landed
            uint4 q[R];
#pragma unroll
            for (int h = 0; h < R; ++h) q[h] = chunk_row<kAligned>(ring + s * L::kSlot, h, shift, lane);
            const Scales<R, kZeros> now = c[s];
            load(c[s], s);  // (over what this lane has just read)
#pragma unroll
            for (int b = 0; b < kSub<NT>; ++b) {
              const int h = 2 * b;
              multiply_rows<NT, kSmallGroups>(
                  q[h], q[h + 1], __uint_as_float(now.s[h] << scale_shift), __uint_as_float(now.s[h + 1] << scale_shift),
                  kZeros ? 0x43004300u + 0x00010001u * (now.z[kZeros ? h : 0] & 15u) : 0x43084308u,
                  kZeros ? 0x43004300u + 0x00010001u * (now.z[kZeros ? h + 1 : 0] & 15u) : 0x43084308u,
                  xs + (int64_t)at * 4 * NT * kUnit, acc[b], lane);
            }
            at += S;
            if (at < per * S) continue;
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
  asm volatile("cp.async.wait_all;" ::: "memory");
}

template <int NT, bool kSmallGroups, bool kAligned, bool kZeros>
int launch_w4_as(W4Params& p, cudaStream_t st) {
  static std::atomic<bool> done[kMaxDevices];
  using L = Layout<NT, kAligned>;
  auto k = w4_kernel<NT, kSmallGroups, kAligned, kZeros>;
  if (int rc = ensure_smem(k, kW4Smem, done)) return rc;
  constexpr int W = kWarps<NT>, sms = 152;
  constexpr int sums = L::kSums * 4;        // bytes
  constexpr int x_bytes = 4 * NT * kUnit;   // of a chunk
  constexpr int room = kW4Smem - L::kPart - L::kRing;
  const int tiles = (p.n + L::kRows - 1) / L::kRows;
  const int chunks = (p.k + kChunk - 1) / kChunk;
  static_assert(room / 4 >= W / 4 * sums, "a tile of each group must be kept");
  static_assert(room - room / 4 >= x_bytes * 4, "a block of k must fit");
  // a block of a group's width of k has to fit; 24 and 16 are whole blocks, 12, 8 and 4 divide them
  int S = tiles <= sms ? W : tiles <= 4 * sms ? 8 : 4;
  while (S * x_bytes > room - room / 4) S = S > 12 ? (W == 24 ? 12 : 8) : S > 8 ? 8 : 4;
  p.split = S;
  const int groups = W / S;
  const int whole = (chunks + S - 1) / S * S;
  p.blocks = 1;
  p.block_chunks = whole;
  p.batch = 0x3fffffff;
  int smem = L::kPart + L::kRing + whole * x_bytes;
  if (whole > room / x_bytes) {  // blocks of k, as even as they come: a quarter of the room keeps sums
    p.batch = std::max(1, room / 4 / (groups * sums));
    const int fits = (room - p.batch * groups * sums) / (x_bytes * S) * S;
    p.blocks = (chunks + fits - 1) / fits;
    p.block_chunks = ((chunks + p.blocks - 1) / p.blocks + S - 1) / S * S;
    p.blocks = (chunks + p.block_chunks - 1) / p.block_chunks;
    smem = L::kPart + L::kRing + p.batch * groups * sums + p.block_chunks * x_bytes;
  }
  const cudaError_t e = launch_dependent(k, std::min(tiles, sms), W * 32, smem, st, p);
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
