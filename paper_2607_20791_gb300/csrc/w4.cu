// Products of a few rows of activations with 4-bit weights: y = x W^T with
// W[n, k] = (q[n, k] - z[n, k / G]) s[n, k / G], q packed two to a byte along k.
//
// The weights are read once; everything else is small.  A tile is 16 rows of W; its CTA's
// eight warps take the 128-weight chunks of those rows in turn, so that together they
// read 512 contiguous bytes of a row at a time.  A chunk is two 16-byte loads a lane
// (lane 4g + t: rows g and g + 8, bytes 16t ..), four chunks ahead of their use, and
// eight or sixteen mma.m16n8k16 with the weights as A: up to 8 rows of x are its N, so one
// row costs the same as eight, and the tensor pipe does the sums over k in fp32.
//
// Which k a lane's A elements stand for is free as long as B agrees, so a lane feeds the
// 8 nibbles of a 32-bit word as they lie: nibbles p and p + 4 are the two halves of
// (word >> 4p) & 0x000f000f, and with 0x4300 over each (bf16 128) they are the bf16
// numbers 128 + q.  128 + z taken from them leaves q - z exactly.  x lies in shared memory
// in that order, one 16-byte load a lane for two MMAs.  With groups of 128 the four words
// of a 16-byte load share a scale and go in as they are; with smaller groups an MMA's k
// must stay within 32 weights, so the quad's 4 x 4 words are transposed first.  A group's
// sum is scaled in fp32 after its last MMA.
//
// The eight warps' sums of a tile meet in shared memory.  Where x does not fit, k goes in
// blocks, with the sums of the CTA's tiles kept in shared memory between them.
#include <cuda_bf16.h>

#include <algorithm>

#include "common.h"
#include "ptx.cuh"

namespace rgd {
namespace {

constexpr int kW4Warps = 8;
constexpr int kW4Threads = kW4Warps * 32;
constexpr int kChunk = 128;      // weights of a row per chunk
constexpr int kAhead = 4;        // chunks in flight per warp
constexpr int kTileRows = 16;
constexpr int kMaxK = 1 << 24;
constexpr int kNoChunk = kMaxK / kChunk;  // past every row's end
constexpr int kUnit = 512;       // bytes of x per MMA step: 8 rows, 32 weights
constexpr int kW4Smem = 112 * 1024;  // of a CTA at most: two to an SM
// Tiles whose sums are kept while k goes in blocks, for 8 NT rows of x.
constexpr int kBatchSums = 32;  // in units of 8 rows: 32 / NT tiles

struct W4Params {
  int32_t m, n, k, groups;
  int32_t group_shift;  // log2 of the group size
  int32_t block_chunks;  // chunks of a block of k (a multiple of kW4Warps)
  int32_t blocks;        // blocks of k
  const uint16_t* x;
  const uint8_t* w;
  const void* scales;
  const uint8_t* zeros;
  void* y;
  int64_t row_bytes, y_stride, total_bytes;
  int32_t scale_f32, out_f32, x_vec;
};

__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Nibbles p and p + 4 of a word as bf16 q - z (bias: 128 + z twice).
__device__ __forceinline__ uint32_t weights2(uint32_t word, int p, uint32_t bias) {
  const uint32_t u = ((word >> (4 * p)) & 0x000f000fu) | 0x43004300u;
  const __nv_bfloat162 v = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&u), *reinterpret_cast<const __nv_bfloat162*>(&bias));
  return *reinterpret_cast<const uint32_t*>(&v);
}

// What a lane holds of a chunk: 32 weights of rows g and g + 8, and one group's scale and
// zero of each, as they lie in memory (a load must not be waited for before its use).
struct Chunk {
  uint4 q[2];
  uint32_t s[2], z[2];
};

// 16 bytes that no other block reads.
__device__ __forceinline__ uint4 load_once(const uint8_t* p) {
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}

// 16 bytes from any address: the five words they lie in, shifted.  A word that ends past
// the buffer is put together from its bytes.
__device__ __forceinline__ uint4 load_unaligned(const uint8_t* w, int64_t at, int64_t total) {
  const int64_t a = at & ~int64_t(3);
  const uint32_t sh = (uint32_t)(at & 3) * 8;
  uint32_t u[5];
#pragma unroll
  for (int i = 0; i < 5; ++i) {
    const int64_t o = a + 4 * i;
    u[i] = 0;
    if (o + 4 <= total) u[i] = __ldg(reinterpret_cast<const uint32_t*>(w + o));
    else
      for (int b = 0; b < 4; ++b)
        if (o + b < total) u[i] |= (uint32_t)w[o + b] << (8 * b);
  }
  return make_uint4(__funnelshift_r(u[0], u[1], sh), __funnelshift_r(u[1], u[2], sh), __funnelshift_r(u[2], u[3], sh),
                    __funnelshift_r(u[3], u[4], sh));
}

// Where a lane's rows of a tile lie.
struct Rows {
  int64_t w[2];  // byte of the lane's first 16 of chunk 0
  int64_t g[2];  // first group
};
__device__ __forceinline__ void at_tile(const W4Params& p, Rows& r, int tile, int lane) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int n = min(tile * kTileRows + (lane >> 2) + 8 * h, p.n - 1);  // (rows past the last are not written)
    r.w[h] = n * p.row_bytes + (lane & 3) * 16;
    r.g[h] = (int64_t)n * p.groups;
  }
}

template <bool kSmallGroups, bool kAligned>
__device__ __forceinline__ void load_chunk(const W4Params& p, Chunk& c, const Rows& r, int chunk, int lane) {
  const int off = chunk * (kChunk / 2);
  // (a group of the whole chunk is every lane's, also of those past the row's end)
  const int k = chunk * kChunk + (kSmallGroups ? (lane & 3) * 32 : 0);
  const bool some = k < p.k, all = off + (lane & 3) * 16 < (int)p.row_bytes;
  const int group = k >> p.group_shift;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    c.q[h] = make_uint4(0, 0, 0, 0);
    c.s[h] = 0;
    c.z[h] = 8;
    if (all) c.q[h] = kAligned ? load_once(p.w + r.w[h] + off) : load_unaligned(p.w, r.w[h] + off, p.total_bytes);
    if (some) {
      if (p.scale_f32) c.s[h] = __ldg(static_cast<const uint32_t*>(p.scales) + r.g[h] + group);
      else c.s[h] = __ldg(static_cast<const uint16_t*>(p.scales) + r.g[h] + group);
      if (p.zeros) c.z[h] = __ldg(p.zeros + r.g[h] + group);
    }
  }
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

// Adds a chunk's products to the sums of its tile.
template <int NT, bool kSmallGroups>
__device__ __forceinline__ void multiply_chunk(Chunk& c, const uint8_t* xs, float (&acc)[NT][4], int scale_shift, int lane) {
  if (kSmallGroups) {
    transpose_quad(c.q[0], lane & 3);
    transpose_quad(c.q[1], lane & 3);
  }
  const float sc[2] = {__uint_as_float(c.s[0] << scale_shift), __uint_as_float(c.s[1] << scale_shift)};
  const uint32_t zc[2] = {0x43004300u + 0x00010001u * (c.z[0] & 15u), 0x43004300u + 0x00010001u * (c.z[1] & 15u)};
  float sum[NT][4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t lo = j == 0 ? c.q[0].x : j == 1 ? c.q[0].y : j == 2 ? c.q[0].z : c.q[0].w;
    const uint32_t hi = j == 0 ? c.q[1].x : j == 1 ? c.q[1].y : j == 2 ? c.q[1].z : c.q[1].w;
    float s0 = sc[0], s1 = sc[1];
    uint32_t z0 = zc[0], z1 = zc[1];
    if (kSmallGroups) {  // (the group of these 32 weights is lane j's of the quad)
      const int from = (lane & ~3) | j;
      s0 = __shfl_sync(0xffffffffu, s0, from);
      s1 = __shfl_sync(0xffffffffu, s1, from);
      z0 = __shfl_sync(0xffffffffu, z0, from);
      z1 = __shfl_sync(0xffffffffu, z1, from);
    }
    uint32_t a[4], b[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      a[q] = weights2(lo, q, z0);
      b[q] = weights2(hi, q, z1);
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
        acc[i][0] = fmaf(s0, sum[i][0], acc[i][0]);
        acc[i][1] = fmaf(s0, sum[i][1], acc[i][1]);
        acc[i][2] = fmaf(s1, sum[i][2], acc[i][2]);
        acc[i][3] = fmaf(s1, sum[i][3], acc[i][3]);
      }
    }
  }
}

// A block of x into shared memory, 8 numbers a lane and step, in the order of the nibbles.
template <int NT, bool kSmallGroups>
__device__ __forceinline__ void stage_x(const W4Params& p, uint8_t* xs, int chunk0, int chunks, int m0) {
  for (int u = threadIdx.x; u < chunks * 4 * NT * 32; u += kW4Threads) {
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

// NT: groups of 8 rows of x.
template <int NT, bool kSmallGroups, bool kAligned>
__global__ void __launch_bounds__(kW4Threads, 2) w4_kernel(const W4Params p) {
  constexpr int kSums = kTileRows * 8 * NT, kBatch = kBatchSums / NT;
  extern __shared__ __align__(16) uint8_t dyn[];
  float* part = reinterpret_cast<float*>(dyn);             // [2][warps][kSums]
  float* kept = part + 2 * kW4Warps * kSums;               // [kBatch][kSums], where k goes in blocks
  uint8_t* xs = reinterpret_cast<uint8_t*>(kept + (p.blocks > 1 ? kBatch * kSums : 0));
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");  // (a dependent waits for this kernel's end)
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int tiles = (p.n + kTileRows - 1) / kTileRows;
  const int mine = (tiles - (int)blockIdx.x + (int)gridDim.x - 1) / (int)gridDim.x;  // this CTA's tiles, gridDim apart
  const int scale_shift = p.scale_f32 ? 0 : 16;
  int flip = 0;
  for (int m0 = 0; m0 < p.m; m0 += 8 * NT) {
    for (int first = 0; first < mine; first += kBatch) {
      const int batch = min(kBatch, mine - first);
      for (int kb = 0; kb < p.blocks; ++kb) {
        const int chunk0 = kb * p.block_chunks;
        const int chunks = min(p.block_chunks, (p.k + kChunk - 1) / kChunk - chunk0);
        const int per = (chunks + kW4Warps - 1) / kW4Warps;  // chunks of a warp and tile
        const int items = batch * per;
        Chunk c[kAhead];
        int lt = 0, lc = 0;  // the next chunk to load: tile of the batch, chunk of the tile
        Rows rows;
        at_tile(p, rows, (int)blockIdx.x + first * (int)gridDim.x, lane);
        auto load = [&](Chunk& into) {
          const int chunk = lc * kW4Warps + warp;
          load_chunk<kSmallGroups, kAligned>(p, into, rows, lt < batch && chunk < chunks ? chunk0 + chunk : kNoChunk, lane);
          if (++lc < per) return;
          lc = 0;
          ++lt;
          at_tile(p, rows, (int)blockIdx.x + (first + lt) * (int)gridDim.x, lane);
        };
#pragma unroll
        for (int s = 0; s < kAhead; ++s) load(c[s]);
        if (p.blocks > 1 || first == 0) {
          __syncthreads();  // (the x of the block before is no longer read)
          stage_x<NT, kSmallGroups>(p, xs, chunk0, per * kW4Warps, m0);
          __syncthreads();
        }
        float acc[NT][4] = {};
        int tile = 0, at = 0;
        for (int it = 0; it < items; it += kAhead) {
#pragma unroll
          for (int s = 0; s < kAhead; ++s) {
            if (it + s >= items) break;
            multiply_chunk<NT, kSmallGroups>(c[s], xs + (int64_t)(at * kW4Warps + warp) * 4 * NT * kUnit, acc, scale_shift, lane);
            load(c[s]);
            if (++at < per) continue;
            // the tile's sums: this warp's, then all of them
            float* mp = part + (flip * kW4Warps + warp) * kSums;
#pragma unroll
            for (int i = 0; i < NT; ++i)
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                mp[(i * 8 + (lane & 3) * 2 + (e & 1)) * kTileRows + (lane >> 2) + (e >> 1) * 8] = acc[i][e];
                acc[i][e] = 0.f;
              }
            __syncthreads();
            for (int o = threadIdx.x; o < kSums; o += kW4Threads) {
              float v = p.blocks > 1 && kb > 0 ? kept[tile * kSums + o] : 0.f;
#pragma unroll
              for (int w = 0; w < kW4Warps; ++w) v += part[(flip * kW4Warps + w) * kSums + o];
              if (kb + 1 < p.blocks) {
                kept[tile * kSums + o] = v;
                continue;
              }
              const int m = m0 + o / kTileRows;
              const int64_t n = (int64_t)((int)blockIdx.x + (first + tile) * (int)gridDim.x) * kTileRows + o % kTileRows;
              if (m >= p.m || n >= p.n) continue;
              if (p.out_f32) static_cast<float*>(p.y)[m * p.y_stride + n] = v;
              else static_cast<__nv_bfloat16*>(p.y)[m * p.y_stride + n] = __float2bfloat16(v);
            }
            flip ^= 1;  // (the other half is free: every thread has passed the barrier after its sums were read)
            at = 0;
            ++tile;
          }
        }
      }
    }
  }
}

template <int NT, bool kSmallGroups, bool kAligned>
int launch_w4(W4Params& p, cudaStream_t st) {
  static std::atomic<bool> done[kMaxDevices];
  auto k = w4_kernel<NT, kSmallGroups, kAligned>;
  if (int rc = ensure_smem(k, kW4Smem, done)) return rc;
  const int chunks = (p.k + kChunk - 1) / kChunk;
  constexpr int sums = kTileRows * 8 * NT * 4;  // bytes
  constexpr int x_bytes = 4 * NT * kUnit;       // of a chunk
  constexpr int fixed = 2 * kW4Warps * sums, kept = kBatchSums / NT * sums;
  static_assert(fixed + kept + x_bytes * kW4Warps <= kW4Smem, "a block of k must fit");
  const int whole = (chunks + kW4Warps - 1) / kW4Warps * kW4Warps;
  p.blocks = 1;
  p.block_chunks = whole;
  int smem = fixed + whole * x_bytes;
  if (smem > kW4Smem) {  // blocks of k, as even as they come
    const int most = (kW4Smem - fixed - kept) / (x_bytes * kW4Warps) * kW4Warps;
    p.blocks = (chunks + most - 1) / most;
    p.block_chunks = ((chunks + p.blocks - 1) / p.blocks + kW4Warps - 1) / kW4Warps * kW4Warps;
    p.blocks = (chunks + p.block_chunks - 1) / p.block_chunks;
    smem = fixed + kept + p.block_chunks * x_bytes;
  }
  const int tiles = (p.n + kTileRows - 1) / kTileRows;
  const int grid = std::min(tiles, 304);
  const cudaError_t e = launch_dependent(k, grid, kW4Threads, smem, st, p);
  return e == cudaSuccess ? RGD_OK : cuda_error(e, "w4 launch");
}

template <int NT>
int launch_w4_kind(W4Params& p, cudaStream_t st) {
  const bool small = p.group_shift < 7, aligned = p.row_bytes % 16 == 0;
  if (small) return aligned ? launch_w4<NT, true, true>(p, st) : launch_w4<NT, true, false>(p, st);
  return aligned ? launch_w4<NT, false, true>(p, st) : launch_w4<NT, false, false>(p, st);
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
  RGD_CHECK_ARG(k <= kMaxK, "%s: k too large", fn);
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
  p.scales = scales;
  p.zeros = zeros;
  p.y = y;
  p.row_bytes = ((int64_t)k + 1) / 2;
  p.total_bytes = p.row_bytes * n;
  p.y_stride = y_stride;
  p.scale_f32 = scale_dtype == RGD_F32;
  p.out_f32 = out_dtype == RGD_F32;
  p.x_vec = k % 8 == 0;
  cudaStream_t st = (cudaStream_t)stream;
  return m <= 8 ? launch_w4_kind<1>(p, st) : m <= 16 ? launch_w4_kind<2>(p, st) : launch_w4_kind<4>(p, st);
}
