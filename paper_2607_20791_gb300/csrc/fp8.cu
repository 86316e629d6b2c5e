// Products of 8-bit floating-point activations and weights, each with a scale for every 128
// values of k:
//   y[i, j] = sum_b sx[i, b] sw[j / 128, b] sum_{k in block b} x[i, k] w[j, k].
//
// One block of k is four tensor core instructions (K = 32 each) into one of two to eight TMEM
// accumulators; while the next blocks' run into others, warps read the sums of the last one and
// add them, scaled, to what they hold in registers in fp32.  So a scale is applied once to 128
// products' sum, whatever its value.
//
// The tensor core takes 128 rows (TMEM lanes) by up to 256 columns.  Many rows of x: x's are
// the lanes and w's the columns (a lane's scale is one number), 128 of them to a CTA or 256
// to a pair of CTAs with 256 rows.  Few (up to 128): w's are the lanes and all of x's rows the
// columns, so that the weights are read once; bound by them.  Where there are too few tiles
// for the SMs a cluster of CTAs shares one, each with a part of k, and they add their parts
// up in order: the same sums in every call.
//
// Warps: the first 4, 8 or 16 add sums up, one copies tiles in by TMA, one issues the tensor
// core's instructions, one fetches scales.
//
// Measured back to back, with inputs that change (a copy runs at 6.75 TB/s, bf16 products at 1.93 PFLOP/s):
//   x rows  n x k          time     rate                  bound by
//   8192    14336 x 4096   387 us   2.49 PFLOP/s          reading sums: a pair's step of 256 x 256 x 128 takes
//                                                         960 clocks, 640 if its sums are not read; at length
//                                                         power (353 us for a short run over one set of inputs)
//   4096    4096 x 4096    62 us    2.22 PFLOP/s          the same
//   200     128256 x 4096  118 us   4.4 TB/s of weights   the steps of 128 x 128 tiles
//   80      128256 x 4096  102 us   5.1 TB/s              adding sums, with factors of their own
//   64      128256 x 4096  88 us    6.0 TB/s              weights
//   16      128256 x 4096  88 us    6.0 TB/s              weights
//   80      6144 x 4096    13.0 us  1.9 TB/s              16 steps one after another on 96 SMs, start and join
#include <cuda_bf16.h>

#include <algorithm>

#include "common.h"
#include "ptx.cuh"

namespace rgd {
namespace {

constexpr int kLanes = 128;              // rows of A a CTA's tile
constexpr int kStep = 128;               // values of k that share a scale: one step
constexpr int kABytes = kLanes * kStep;  // of a stage
constexpr int kMostStages = 12;
constexpr int kScaleSteps = 4;  // steps whose scales are fetched together: a slot
constexpr int kScaleSlots = 4;  // on their way or in use
constexpr int kScaleAhead = 2;  // on their way
constexpr int kMostSums = 8;    // accumulators at most
constexpr int kRoom = 227 * 1024 - 1024;

struct Fp8Params {
  int32_t m, n, steps;  // steps of k
  const float* sx;
  const float* sw;
  uint8_t* y;
  int64_t y_stride;  // elements
  int32_t out_f32, vectors;
  int32_t a_tiles, b_tiles, tiles, band, split;
  int32_t cols;                   // columns of a tile: the instructions' N
  int32_t stages;
  int32_t* dev_status;
};

struct Fp8Shared {
  uint64_t full[kMostStages], empty[kMostStages], sum_full[kMostSums], sum_empty[kMostSums];
  uint64_t scale_full[kScaleSlots], scale_empty[kScaleSlots], drained;
  uint32_t tmem;
  int dead;
};

__device__ __forceinline__ uint64_t pair2(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void unpair2(uint64_t v, float& a, float& b) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v));
}
__device__ __forceinline__ uint64_t fma_pair(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}

// Tile t: `band` of A's tiles by all of B's, then the next band: what the SMs work on at a time
// are few of either.
__device__ __forceinline__ void tile_at(const Fp8Params& p, int t, int& ta, int& tb) {
  const int first = t / (p.band * p.b_tiles) * p.band, high = min(p.band, p.a_tiles - first), r = t - first * p.b_tiles;
  ta = first + r % high;
  tb = r / high;
}

__device__ __forceinline__ void put(uint8_t* to, int f32, float v) {
  if (f32) *reinterpret_cast<float*>(to) = v;
  else *reinterpret_cast<__nv_bfloat16*>(to) = __float2bfloat16_rn(v);
}
__device__ __forceinline__ void write_one(const Fp8Params& p, int64_t row, int64_t col, float v) {
  if (row >= p.m || col >= p.n) return;
  put(p.y + (row * p.y_stride + col) * (p.out_f32 ? 4 : 2), p.out_f32, v);
}

// A store of its own instruction: 128 of them in a row must not be converted ahead of time.
__device__ __forceinline__ void put_if(bool on, uint8_t* to, int f32, float v) {
  if (f32)
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %0, 0;\n\t@p st.global.f32 [%1], %2;\n\t}" ::"r"((int)on), "l"(to), "f"(v) : "memory");
  else
    asm volatile("{\n\t.reg .pred p;\n\t.reg .b16 h;\n\tsetp.ne.b32 p, %0, 0;\n\tcvt.rn.bf16.f32 h, %2;\n\t@p st.global.b16 [%1], h;\n\t}" ::"r"((int)on), "l"(to), "f"(v) : "memory");
}

constexpr int kStageWords = 17;  // of a row: 16 and one that spreads rows over the banks

// The whole warp: 16 words each of 32 rows that lie in shared memory go to y; `rows` of them and
// `count` elements of kSize bytes are y's.
template <int kSize>
__device__ __forceinline__ void write_rows(const Fp8Params& p, const uint32_t* words, uint8_t* to, int rows, int count, int lane) {
  __syncwarp();
  if (p.vectors) {  // rows of y on 16 bytes
    const int part = lane & 3;
    const bool whole = (part + 1) * (16 / kSize) <= count;
#pragma unroll 1
    for (int r = lane >> 2; r < rows; r += 8) {
      const uint32_t* w = words + r * kStageWords + part * 4;
      uint8_t* at = to + r * p.y_stride * kSize + part * 16;
      if (whole) {
        *reinterpret_cast<uint4*>(at) = make_uint4(w[0], w[1], w[2], w[3]);
      } else {
#pragma unroll 1
        for (int i = 0; i < 16 / kSize && part * (16 / kSize) + i < count; ++i) {
          if (kSize == 4) reinterpret_cast<uint32_t*>(at)[i] = w[i];
          else reinterpret_cast<uint16_t*>(at)[i] = (uint16_t)(w[i / 2] >> (16 * (i & 1)));
        }
      }
    }
  } else if (p.y_stride * kSize % 4 == 0) {  // on 4: words, lanes side by side (6860 x 7494 x 144, fp32: 73 us, 174 as above)
    const int i = lane & 15, n = (i + 1) * (4 / kSize) - count;  // (elements of the word that are not y's)
    uint8_t* at = to + (lane >> 4) * p.y_stride * kSize + i * 4;
    const uint32_t* w = words + (lane >> 4) * kStageWords + i;
#pragma unroll 4
    for (int r = lane >> 4; r < rows; r += 2, at += 2 * p.y_stride * kSize, w += 2 * kStageWords) {
      if (n <= 0) *reinterpret_cast<uint32_t*>(at) = *w;
      else if (kSize == 2 && n == 1) *reinterpret_cast<uint16_t*>(at) = (uint16_t)*w;
    }
  } else {
    uint8_t* at = to + lane * 2;
#pragma unroll 4
    for (int r = 0; r < rows; ++r, at += p.y_stride * 2)
      if (lane < count) *reinterpret_cast<uint16_t*>(at) = (uint16_t)(words[r * kStageWords + lane / 2] >> (16 * (lane & 1)));
  }
  __syncwarp();
}

constexpr int kMostSplit = 8;  // CTAs that share a tile
template <int NT>
constexpr int kPartRow = NT + 4;  // floats of a lane's part (lanes on different banks)
constexpr int kBox = 4096;  // 32 rows of 128 bytes
// The whole warp: a box that it has filled goes to y at column x and row y0, as far as y has them.
__device__ __forceinline__ void send_box(const Fp8Params& p, const CUtensorMap& map, const uint8_t* box, int x, int y0, int lane) {
  fence_proxy_async_smem();
  __syncwarp();
  if (lane == 0) {
    if (y0 < p.m && x < p.n) tma_store_2d(&map, box, x, y0);
    bulk_commit();
  }
}

// Threads that add up: a warp to 32 lanes, two from 33 columns on, and four where every sum has a factor of its own
// (80 x 6144 x 4096: 13.0 us with four, 14.2 with two; 256 rows of x, whose sums have one: 17.8 and 16.6).
template <int NT, bool kTurned>
constexpr int kAdders = NT == 128 && kTurned ? 512 : NT > 32 ? 256 : 128;
template <int NT, bool kTurned>
constexpr int kFp8Threads = kAdders<NT, kTurned> + 128;

__device__ __forceinline__ uint64_t mul_pair(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
// Waits for all loads; those into r and s are not read before.
template <int N>
__device__ __forceinline__ void tmem_load_wait(uint32_t (&r)[N], uint32_t (&s)[N]) {
  if constexpr (N == 32) {
    tmem_ld_wait32(r);
    tmem_after_wait32(s);
  } else {
    tmem_ld_wait16(r);
    tmem_after_wait16(s);
  }
}
// 4 bytes to shared memory, without a wait; zeros if not `on`.
__device__ __forceinline__ void copy_async4(float* dst, const float* src, bool on) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(smem_u32(dst)), "l"(src), "r"(on ? 4 : 0) : "memory");
}

// NT: columns of a tile at most.  kTurned: w's rows are the lanes, x's the columns.  kPair: two
// CTAs take 256 rows of x by 256 columns; each copies its own rows and half of the columns, so
// that a value that is copied takes part in half as many copies again (48 KB a step by one CTA,
// 32 by each of two), and the tensor cores read it from both CTAs' memory.
template <int NT, bool kTurned, bool kPair>
__global__ void __launch_bounds__(kFp8Threads<NT, kTurned>, 1)
    fp8_kernel(const Fp8Params p, const __grid_constant__ CUtensorMap amap, const __grid_constant__ CUtensorMap bmap,
               const __grid_constant__ CUtensorMap ymap) {
  static_assert(!kPair || (NT == 256 && !kTurned), "");
  constexpr int kOwn = NT / (kAdders<NT, kTurned> / 128);  // columns of a thread
  constexpr int kProducer = kAdders<NT, kTurned> / 32, kIssuer = kProducer + 1, kScaler = kProducer + 2;
  constexpr int kSums = 512 / NT < kMostSums ? 512 / NT : kMostSums;  // accumulators
  constexpr uint32_t kTmemCols = kSums * NT;
  constexpr int kRows = kTurned ? NT : kLanes;  // x's rows of a tile
  extern __shared__ uint8_t raw[];
  __shared__ Fp8Shared sh;
  __shared__ __align__(16) float x_scale[kScaleSlots * kScaleSteps][kRows];
  __shared__ float w_scale[kScaleSlots * kScaleSteps][2];
  __shared__ uint32_t stage[kTurned || kPair ? 1 : kAdders<NT, kTurned> * kStageWords];
  uint8_t* ring = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~uintptr_t(1023));
  uint8_t* out = ring + (kPair ? p.stages * (kABytes + 128 * kStep) : 0);  // boxes on their way to y
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int b_rows = kPair ? p.cols / 2 : p.cols;  // of B that this CTA copies
  const int stage_bytes = kABytes + b_rows * kStep;
  uint32_t rank = 0, tile0 = blockIdx.x, tile_step = gridDim.x;
  if (kPair || p.split > 1) {
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    asm volatile("mov.u32 %0, %%clusterid.x;" : "=r"(tile0));
    tile_step = kPair ? gridDim.x / 2 : (uint32_t)p.tiles;
  }
  const int parts = kPair ? 1 : p.split, part_rank = kPair ? 0 : (int)rank;
  const int step0 = (int)((int64_t)p.steps * part_rank / parts), steps = (int)((int64_t)p.steps * (part_rank + 1) / parts) - step0;
  const int total = ((p.tiles - 1 - (int)tile0) / (int)tile_step + 1) * steps;

  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");  // (a dependent waits for this kernel's end)
  if (warp == kIssuer) {
    if (kPair) {
      tmem_alloc_pair(&sh.tmem, kTmemCols);
      tmem_relinquish_pair();
    } else {
      tmem_alloc(&sh.tmem, kTmemCols);
      tmem_relinquish();
    }
  }
  if (threadIdx.x == 0) {
    sh.dead = 0;
    for (int i = 0; i < p.stages; ++i) {
      mbar_init(&sh.full[i], 1);
      mbar_init(&sh.empty[i], 1);
    }
    for (int i = 0; i < kSums; ++i) {
      mbar_init(&sh.sum_full[i], 1);
      mbar_init(&sh.sum_empty[i], kAdders<NT, kTurned> / 32 * (kPair ? 2 : 1));
    }
    for (int i = 0; i < kScaleSlots; ++i) {
      mbar_init(&sh.scale_full[i], 1);
      mbar_init(&sh.scale_empty[i], kAdders<NT, kTurned> / 32);
    }
    mbar_init(&sh.drained, 1);
    fence_mbar_init();
  }
  if (warp == kProducer && lane == 0) {
    prefetch_tensormap(&amap);
    prefetch_tensormap(&bmap);
  }
  tc_fence_before();
  __syncthreads();
  if (kPair) {  // (each signals the other's barriers)
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  }
  tc_fence_after();
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const uint32_t tmem = sh.tmem;

  // 256 columns: 128 sums and more a thread, of the registers that the other four warps have left
  // (384 threads of 168 at launch: 256 of 232 and 128 of 40 are as many).
  int issued = 0;  // steps whose copies are on their way, or were
  if (warp >= kProducer) {
    if (NT > 128) asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
    if (warp == kProducer) {
      uint32_t tile = tile0;
      int at = 0, s = 0, ay = 0, by = 0;
      uint32_t turn = 0;
#pragma unroll 1
      for (; issued < total; ++issued) {
        if (at == 0) {  // (a division takes longer than a step has)
          int ta, tb;
          tile_at(p, (int)tile, ta, tb);
          ay = ta * (kPair ? 2 * kLanes : kLanes) + (kPair ? (int)rank * kLanes : 0);
          by = tb * p.cols + (kPair ? (int)rank * b_rows : 0);
        }
        if (!__all_sync(0xffffffffu, turn == 0 || mbar_wait_soon(&sh.empty[s], (turn - 1) & 1u))) {
          sh.dead = 1;
          break;
        }
        if (elect_one()) {
          uint8_t* a = ring + s * stage_bytes;
          const int kx = (step0 + at) * kStep;
          if (kPair) {  // (the first CTA's barrier counts both CTAs' copies)
            const uint32_t bar = mapa_u32(smem_u32(&sh.full[s]), 0);
            if (rank == 0) mbar_arrive_expect_tx(&sh.full[s], 2u * (uint32_t)stage_bytes);
            tma_load_2d_pair(a, &amap, bar, kx, ay);
            tma_load_2d_pair(a + kABytes, &bmap, bar, kx, by);
          } else {
            mbar_arrive_expect_tx(&sh.full[s], (uint32_t)stage_bytes);
            tma_load_2d(a, &amap, &sh.full[s], kx, ay);
            tma_load_2d(a + kABytes, &bmap, &sh.full[s], kx, by);
          }
        }
        __syncwarp();
        if (++at == steps) {
          at = 0;
          tile += tile_step;
        }
        if (++s == p.stages) {
          s = 0;
          ++turn;
        }
      }
    }
    // This warp, too, waits as one and a lane of it issues: these instructions take operands that are the
    // same in a warp, and cost a lane that is alone in a branch more (8192 x 14336 x 4096: 353 us so, 362
    // with the copies by lane 0, 390 with both).
    if (warp == kIssuer && (!kPair || rank == 0)) {
      const uint32_t idesc = idesc_e4m3_f32(kPair ? 2 * kLanes : kLanes, p.cols);
      const uint64_t ring_desc = smem_desc(smem_u32(ring), 16, 1024, 2);
      const uint32_t sums = __shfl_sync(0xffffffffu, tmem, 0);  // (of shared memory: the same in each lane)
      int s = 0;
      uint32_t turn = 0;
#pragma unroll 1
      for (int q = 0; q < total; ++q) {
        const int b = q % kSums;
        const bool good = (q < kSums || mbar_wait_soon(&sh.sum_empty[b], (uint32_t)(q / kSums - 1) & 1u)) && mbar_wait_soon(&sh.full[s], turn & 1u);
        if (!__all_sync(0xffffffffu, good)) {
          sh.dead = 1;
          break;
        }
        tc_fence_after();
        if (elect_one()) {
          const uint64_t ad = ring_desc + (uint64_t)((uint32_t)(s * stage_bytes) >> 4), bd = ad + (kABytes >> 4);
#pragma unroll
          for (int i = 0; i < kStep / 32; ++i) {
            if (kPair) umma_e4m3_pair(sums + b * NT, ad + 2 * i, bd + 2 * i, idesc, i > 0);
            else umma_e4m3(sums + b * NT, ad + 2 * i, bd + 2 * i, idesc, i > 0);
          }
          if (kPair) {
            umma_commit_pair(&sh.sum_full[b]);
            umma_commit_pair(&sh.empty[s]);
          } else {
            umma_commit(&sh.sum_full[b]);
            umma_commit(&sh.empty[s]);
          }
        }
        __syncwarp();
        if (++s == p.stages) {
          s = 0;
          ++turn;
        }
      }
    }
    if (warp == kScaler) {  // x's rows' scales, and those of the tile's blocks of w, of a few steps at a time
      uint32_t tile = tile0;
      int at = 0, chunks = (total + kScaleSteps - 1) / kScaleSteps, c = 0, rows = 0;
      const int64_t x_stride = (int64_t)p.steps * 32;
      const float *x_from = p.sx, *w_from = p.sw;
      for (; c < chunks; ++c) {
        const int slot = c % kScaleSlots;
        if (c >= kScaleSlots && !__all_sync(0xffffffffu, mbar_wait_soon(&sh.scale_empty[slot], (uint32_t)(c / kScaleSlots - 1) & 1u))) {
          sh.dead = 1;
          break;
        }
#pragma unroll 1
        for (int j = 0; j < kScaleSteps && c * kScaleSteps + j < total; ++j) {
          if (at == 0) {
            int ta, tb;
            tile_at(p, (int)tile, ta, tb);
            const int64_t r0 = (kTurned ? 0 : (int64_t)ta * (kPair ? 2 * kLanes : kLanes) + (kPair ? (int)rank * kLanes : 0)) + lane;
            rows = (int)max(int64_t(-1), min(int64_t(kRows), p.m - r0));
            x_from = p.sx + r0 * p.steps + step0;
            const int block = kTurned ? ta : min((int)(((int64_t)tb * p.cols + lane * 128) / 128), (p.n - 1) / 128);
            w_from = p.sw + (int64_t)block * p.steps + step0;
          }
          float* to = &x_scale[slot * kScaleSteps + j][lane];
          const float* from = x_from;
#pragma unroll
          for (int i = 0; i < kRows; i += 32, from += x_stride) copy_async4(to + i, i < rows ? from : p.sx, i < rows);
          if (lane < 2) copy_async4(&w_scale[slot * kScaleSteps + j][lane], w_from, true);
          ++x_from, ++w_from;
          if (++at == steps) {
            at = 0;
            tile += tile_step;
          }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        if (c >= kScaleAhead) {
          asm volatile("cp.async.wait_group %0;" ::"n"(kScaleAhead) : "memory");
          __syncwarp();
          if (lane == 0) mbar_arrive(&sh.scale_full[(c - kScaleAhead) % kScaleSlots]);
        }
      }
      asm volatile("cp.async.wait_all;" ::: "memory");
      __syncwarp();
      if (lane == 0)
        for (int i = max(0, c - kScaleAhead); i < c; ++i) mbar_arrive(&sh.scale_full[i % kScaleSlots]);
    }
    __syncwarp();
  } else {
    if (NT > 128) asm volatile("setmaxnreg.inc.sync.aligned.u32 232;");
    const int part = warp >> 2, row = (warp & 3) * 32 + lane;  // of the tile's columns; the lane's row of A
    // Of w's rows as lanes, the warps' shares of the columns are whole 16s (the last ones may have none).
    constexpr int kParts = kAdders<NT, kTurned> / 128;
    const int each = kTurned ? min((p.cols / kParts + 15) / 16 * 16, kOwn) : kOwn, off = part * each;
    const int mine = kTurned ? max(0, min(each, p.cols - off)) : kOwn;
    const uint32_t at_tmem = tmem + ((uint32_t)(warp & 3) << 21) + off;
    const uint32_t free_sum = kPair ? mapa_u32(smem_u32(&sh.sum_empty[0]), 0) : 0;
    uint64_t acc[kOwn / 2];
#pragma unroll
    for (int i = 0; i < kOwn / 2; ++i) acc[i] = 0;
    // A step's sums come in chunks.  x's rows as lanes: 32 columns of the thread's own lane at a time, the next while
    // these are added; two together where there are no more (all of a pair's two together: 566 us for 8192 x 14336 x
    // 4096, 393 so).  w's rows as lanes: a column has a factor of its own, and a thread that has all columns of one
    // lane reads as many factors as sums; so 16 lanes' columns, two of each 8, are spread over the warp, and four pairs
    // of sums share two factors (80 x 128256 x 4096: 107 us so, 140 with a factor of its own to each).
    constexpr bool kTwo = kOwn < 128;
    constexpr int kChunk = kTurned ? 16 : 32, kChunks = kOwn / kChunk;
    static_assert(kTurned ? kChunks == 2 : !kTwo || kChunks == 2, "");
    auto spread_col = [&](int i) { return i % (kOwn / 4) / 2 * 8 + 2 * (lane & 3); };  // of pair i of sums
    auto spread_lane = [&](int i) { return i / (kOwn / 4) * 16 + i % 2 * 8 + (lane >> 2); };
    // With factors a step's scales are read while the sums of the step before are on their way (13.0 and 102 us
    // for 13.3 and 107; without, as lanes' scales are, that takes longer, and so does any branch between a load of
    // sums and its wait).
    uint64_t scales[kTurned ? kOwn / 8 : 1];  // of the thread's columns
    float block_scale = 0.f;
    auto read_scales = [&](int slot) {
      block_scale = w_scale[slot][0];
#pragma unroll
      for (int g = 0; g < kOwn / 8; ++g) scales[g] = *reinterpret_cast<const uint64_t*>(&x_scale[slot][off + 8 * g + 2 * (lane & 3)]);
    };
    auto wait_scales = [&](int chunk) {
      return mbar_wait_soon(&sh.scale_full[chunk % kScaleSlots], (uint32_t)(chunk / kScaleSlots) & 1u);
    };
    bool good = !kTurned || wait_scales(0);
    if constexpr (kTurned) read_scales(0);
    int tile = (int)tile0, at = 0;
#pragma unroll 1
    for (int q = 0; q < total; ++q) {
      const int b = q % kSums, slot = q % (kScaleSlots * kScaleSteps), chunk = q / kScaleSteps;
      uint64_t by, factors[kTurned ? kOwn / 8 : 1];
      if constexpr (kTurned) {
        const uint64_t block = pair2(block_scale, block_scale);
#pragma unroll
        for (int g = 0; g < kOwn / 8; ++g) factors[g] = mul_pair(block, scales[g]);
      } else {
        good = q % kScaleSteps != 0 || wait_scales(chunk);
        const float own = w_scale[slot][part * kOwn / 128] * x_scale[slot][row];
        by = pair2(own, own);
      }
      good = mbar_wait_soon(&sh.sum_full[b], (uint32_t)(q / kSums) & 1u) && good;
      if (kTurned && (q + 1) % kScaleSteps == 0 && q + 1 < total) good = wait_scales(chunk + 1) && good;
      if (!__all_sync(0xffffffffu, good)) {
        sh.dead = 1;
        break;
      }
      tc_fence_after();
      uint32_t d[2][kChunk];
      const uint32_t from = at_tmem + b * NT;
      auto add = [&](int c) {
#pragma unroll
        for (int i = 0; i < kChunk / 2; ++i) {
          const uint64_t v = (uint64_t)d[c & 1][2 * i + 1] << 32 | d[c & 1][2 * i];
          acc[c * (kChunk / 2) + i] = fma_pair(v, kTurned ? factors[i / 2] : by, acc[c * (kChunk / 2) + i]);
        }
      };
      auto release = [&]() {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          if (kPair) mbar_arrive_cluster(free_sum + 8 * b);
          else mbar_arrive(&sh.sum_empty[b]);
        }
      };
      if constexpr (kTurned) {
        tmem_ld16_rows16(from, d[0]);
        tmem_ld16_rows16(from + (16u << 16), d[1]);
        read_scales((q + 1) % (kScaleSlots * kScaleSteps));  // (behind the last step: what is there, unused)
      } else {
        tmem_ld32(from, d[0]);
        if (kTwo) tmem_ld32(from + kChunk, d[1]);
      }
      if constexpr (kTwo) {
        tmem_load_wait(d[0], d[1]);
        release();
        add(0);
        add(1);
      } else {
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
          tmem_load_wait(d[c & 1], d[c & 1]);
          if (c + 1 < kChunks) tmem_ld32(from + (c + 1) * kChunk, d[(c + 1) & 1]);
          else release();
          add(c);
        }
      }
      if (q % kScaleSteps == kScaleSteps - 1) {
        __syncwarp();  // (the steps' scales have been read)
        if (lane == 0) mbar_arrive(&sh.scale_empty[chunk % kScaleSlots]);
      }
      if (++at < steps) continue;
      // The end of a tile.
      at = 0;
      int ta, tb;
      tile_at(p, tile, ta, tb);
      const int64_t a0 = (int64_t)ta * (kPair ? 2 * kLanes : kLanes) + (kPair ? (int)rank * kLanes : 0) + row;
      const int64_t b0 = (int64_t)tb * p.cols + off;
      tile += (int)tile_step;
      if (!kPair && p.split > 1) {  // (the ring is free: every copy has been read)
        if (kTurned) {
#pragma unroll
          for (int i = 0; i < kOwn / 2; ++i) {
            const int col = spread_col(i);
            if (col >= mine) continue;
            float v[2];
            unpair2(acc[i], v[0], v[1]);
            float* to = reinterpret_cast<float*>(ring) + (off + col) * kPartRow<kLanes> + (warp & 3) * 32 + spread_lane(i);
            to[0] = v[0];
            to[kPartRow<kLanes>] = v[1];
          }
        } else {
          float* to = reinterpret_cast<float*>(ring) + row * kPartRow<NT> + off;
#pragma unroll
          for (int i = 0; i < kOwn / 4; ++i) {
            if (4 * i >= mine) break;
            float v[4];
            unpair2(acc[2 * i], v[0], v[1]);
            unpair2(acc[2 * i + 1], v[2], v[3]);
            reinterpret_cast<float4*>(to)[i] = make_float4(v[0], v[1], v[2], v[3]);
          }
        }
        break;
      }
      const int es = p.out_f32 ? 4 : 2;
      if (kTurned) {
        const int count = (int)min((int64_t)mine, p.m - b0);
        const int64_t lane0 = a0 - lane;  // the warp's first row of w
#pragma unroll
        for (int i = 0; i < kOwn / 2; ++i) {
          const int col = spread_col(i);
          const int64_t n = lane0 + spread_lane(i);
          float v[2];
          unpair2(acc[i], v[0], v[1]);
          uint8_t* to = p.y + ((b0 + col) * p.y_stride + n) * es;
#pragma unroll
          for (int j = 0; j < 2; ++j) put_if(n < p.n && col + j < count, to + j * p.y_stride * es, p.out_f32, v[j]);
        }
      } else if (kPair) {
        // 128 bytes of each of the warp's rows make a box, which TMA writes while the next is filled.
        uint8_t* box = out + warp * kBox;
        const int x = (int)b0, y = (int)(a0 - lane);
        if (p.out_f32) {
#pragma unroll
          for (int c = 0; c < kOwn / 32; ++c) {
            if (lane == 0) bulk_wait_read();
            __syncwarp();
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              float v[4];
              unpair2(acc[c * 16 + 2 * i], v[0], v[1]);
              unpair2(acc[c * 16 + 2 * i + 1], v[2], v[3]);
              *reinterpret_cast<float4*>(box + lane * 128 + ((i ^ lane) & 7) * 16) = make_float4(v[0], v[1], v[2], v[3]);
            }
            send_box(p, ymap, box, x + c * 32, y, lane);
          }
        } else {
#pragma unroll
          for (int c = 0; c < kOwn / 64; ++c) {
            if (lane == 0) bulk_wait_read();
            __syncwarp();
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              float v[8];
#pragma unroll
              for (int j = 0; j < 4; ++j) unpair2(acc[c * 32 + 4 * i + j], v[2 * j], v[2 * j + 1]);
              *reinterpret_cast<uint4*>(box + lane * 128 + ((i ^ lane) & 7) * 16) =
                  make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
            }
            send_box(p, ymap, box, x + c * 64, y, lane);
          }
        }
      } else {
        // 64 bytes of each of the warp's rows at a time, by way of shared memory.
        uint32_t* words = stage + warp * 32 * kStageWords;
        const int64_t r0 = a0 - lane;
        uint8_t* to = p.y + (r0 * p.y_stride + b0) * es;
        const int rows = (int)min((int64_t)32, p.m - r0), count = (int)min((int64_t)kOwn, p.n - b0);
        if (p.out_f32) {
#pragma unroll
          for (int c = 0; c < kOwn / 16; ++c) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              float u, v;
              unpair2(acc[c * 8 + i], u, v);
              words[lane * kStageWords + 2 * i] = __float_as_uint(u);
              words[lane * kStageWords + 2 * i + 1] = __float_as_uint(v);
            }
            write_rows<4>(p, words, to + c * 64, rows, count - c * 16, lane);
          }
        } else {
#pragma unroll
          for (int c = 0; c < kOwn / 32; ++c) {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              float u, v;
              unpair2(acc[c * 16 + i], u, v);
              words[lane * kStageWords + i] = pack_bf16x2(u, v);
            }
            write_rows<2>(p, words, to + c * 64, rows, count - c * 32, lane);
          }
        }
      }
#pragma unroll
      for (int i = 0; i < kOwn / 2; ++i) acc[i] = 0;
    }
    if (kPair && lane == 0) bulk_wait();
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (!kPair && p.split > 1) {  // the parts, in order of k, by the CTA whose columns they are
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    // Of a CTA: some of w's lanes' columns, or of x's lanes.  Four sums at once, of every CTA together.
    const int lines = kTurned ? p.cols : kLanes, line = kTurned ? kLanes : NT, pitch = kPartRow<kTurned ? kLanes : NT>;
    const int l0 = lines * (int)rank / p.split, l1 = lines * (int)(rank + 1) / p.split;
    int ta, tb;
    tile_at(p, (int)tile0, ta, tb);
    const int64_t a0 = (int64_t)ta * kLanes, b0 = (int64_t)tb * p.cols;
    for (int e = threadIdx.x; e < (l1 - l0) * (line / 4); e += kFp8Threads<NT, kTurned>) {
      const int at = l0 + e / (line / 4), x = e % (line / 4) * 4;
      const uint32_t from = smem_u32(reinterpret_cast<float*>(ring) + at * pitch + x);
      float4 v[kMostSplit];
#pragma unroll
      for (int r = 0; r < kMostSplit; ++r) {
        if (r >= p.split) break;
        uint32_t there;
        asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(from), "r"(r));
        asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                     : "=f"(v[r].x), "=f"(v[r].y), "=f"(v[r].z), "=f"(v[r].w) : "r"(there) : "memory");
      }
      float sum[4] = {v[0].x, v[0].y, v[0].z, v[0].w};
#pragma unroll
      for (int r = 1; r < kMostSplit; ++r) {
        if (r >= p.split) break;
        sum[0] += v[r].x, sum[1] += v[r].y, sum[2] += v[r].z, sum[3] += v[r].w;
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (kTurned) write_one(p, b0 + at, a0 + x + j, sum[j]);
        else write_one(p, a0 + at, b0 + x + j, sum[j]);
      }
    }
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  }
  if (sh.dead) {  // copies and instructions in flight end before the memory that they use is given up
    if (threadIdx.x == 0 && p.dev_status) atomicOr(p.dev_status, RGD_DEV_WAIT_TIMEOUT);
    if (!kPair || rank == 0)  // (which counts both CTAs' copies)
      for (int i = max(0, issued - p.stages); i < issued; ++i) mbar_wait(&sh.full[i % p.stages], (uint32_t)(i / p.stages) & 1u);
    if (warp == kIssuer && (!kPair || rank == 0) && elect_one()) {  // (the lane that issued)
      if (kPair) umma_commit_pair(&sh.drained);
      else umma_commit(&sh.drained);
      mbar_wait(&sh.drained, 0);
    }
    __syncthreads();
  }
  if (kPair) {  // (the tensor cores read the other CTA's memory, and its barriers are signalled)
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  }
  if (warp == kIssuer) {
    if (kPair) tmem_dealloc_pair(tmem, kTmemCols);
    else tmem_dealloc(tmem, kTmemCols);
  }
}

// Boxes of 128 bytes of each of some rows, swizzled.
int encode_boxes(CUtensorMap* map, CUtensorMapDataType type, const void* base, int64_t cols, int64_t rows, int64_t stride,
                 int box_cols, int box_rows) {
  const auto encode = tensor_map_encoder();
  if (!encode) return set_error(RGD_ERR_CUDA, "cuTensorMapEncodeTiled is unavailable");
  const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)stride};
  const cuuint32_t box[2] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows}, ones[2] = {1, 1};
  const CUresult r = encode(map, type, 2, const_cast<void*>(base), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? RGD_OK : set_error(RGD_ERR_CUDA, "cuTensorMapEncodeTiled failed (%d)", (int)r);
}
int encode_rows(CUtensorMap* map, const void* base, int64_t k, int64_t rows, int64_t stride, int box_rows) {
  return encode_boxes(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, base, k, rows, stride, kStep, box_rows);
}

// How many CTAs share a tile, and the time that all tiles take, in steps.  Clusters of 2, 4 or 8 share
// one where that takes less: each round over the SMs costs the steps of its CTAs, and about eight more
// where tiles are shared (their start and their joined sums are not behind another tile's).  152 CTAs
// fit the SMs, as clusters of 4 144, of 8 120.
constexpr int kSms = 152;
struct Split {
  int split;
  int64_t cost;
};
Split best_split(int64_t tiles, int64_t steps) {
  constexpr int fit[4] = {152, 152, 144, 120};
  Split best{1, (tiles + kSms - 1) / kSms * steps};
  for (int i = 1; i < 4 && steps >= 2 << i; ++i) {
    const int64_t cost = ((tiles << i) + fit[i] - 1) / fit[i] * ((steps + (1 << i) - 1) / (1 << i) + 8);
    if (cost < best.cost) best = Split{1 << i, cost};
  }
  return best;
}

struct Fp8Operands {
  const uint8_t* x;
  const uint8_t* w;
  int64_t x_stride, w_stride, k;
};

template <int NT, bool kTurned, bool kPair = false>
int launch_fp8(const char* fn, Fp8Params& p, const Fp8Operands& o, cudaStream_t st) {
  static std::atomic<bool> done[kMaxDevices];
  auto k = fp8_kernel<NT, kTurned, kPair>;
  constexpr int fixed = kScaleSlots * kScaleSteps * 4 * (kTurned ? NT : kLanes) + (kTurned || kPair ? 0 : kAdders<NT, kTurned> * kStageWords * 4) + 1024;
  constexpr int boxes = kPair ? kAdders<NT, kTurned> / 32 * kBox : 0;
  constexpr int room = kRoom - fixed - boxes;
  if (int rc = ensure_smem(k, room + boxes + 1024, done)) return rc;
  p.cols = kTurned ? (p.m + 15) / 16 * 16 : NT;
  const int lanes = kPair ? 2 * kLanes : kLanes, b_rows = kPair ? p.cols / 2 : p.cols;
  const int64_t a_tiles = ((int64_t)(kTurned ? p.n : p.m) + lanes - 1) / lanes;
  const int64_t b_tiles = ((int64_t)(kTurned ? p.m : p.n) + p.cols - 1) / p.cols, tiles = a_tiles * b_tiles;
  if (tiles > 0x7fffffff / p.steps - 1) return set_error(RGD_ERR_UNSUPPORTED, "%s: too many tiles", fn);
  p.a_tiles = (int32_t)a_tiles;
  p.b_tiles = (int32_t)b_tiles;
  p.tiles = (int32_t)tiles;
  p.band = 8;
  const int stage = kABytes + b_rows * kStep;
  p.stages = std::min(kMostStages, room / stage);
  p.split = kPair ? 1 : best_split(tiles, p.steps).split;
  if (p.split > 1 && tiles * p.split > 0x7fffffff) p.split = 1;
  const int grid = p.split > 1 ? p.tiles * p.split : (int)std::min<int64_t>(kPair ? 2 * tiles : tiles, kSms);
  CUtensorMap amap, bmap;
  const uint8_t *a = kTurned ? o.w : o.x, *b = kTurned ? o.x : o.w;
  const int64_t as = kTurned ? o.w_stride : o.x_stride, bs = kTurned ? o.x_stride : o.w_stride;
  if (int rc = encode_rows(&amap, a, o.k, kTurned ? p.n : p.m, as, kLanes)) return rc;
  if (int rc = encode_rows(&bmap, b, o.k, kTurned ? p.m : p.n, bs, b_rows)) return rc;
  CUtensorMap ymap = amap;  // (read by pairs only)
  if (kPair)
    if (int rc = encode_boxes(&ymap, p.out_f32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, p.y, p.n, p.m,
                              p.y_stride * (p.out_f32 ? 4 : 2), p.out_f32 ? 32 : 64, 32)) return rc;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)grid);
  cfg.blockDim = dim3(kFp8Threads<NT, kTurned>);
  cfg.dynamicSmemBytes = (size_t)p.stages * stage + boxes + 1024;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim = {(unsigned)(kPair ? 2 : p.split), 1, 1};
  cfg.attrs = attr;
  cfg.numAttrs = kPair || p.split > 1 ? 2 : 1;
  cudaError_t e = cudaLaunchKernelEx(&cfg, k, p, amap, bmap, ymap);
  if (e == cudaSuccess) e = cudaGetLastError();
  return e == cudaSuccess ? RGD_OK : cuda_error(e, "fp8 product launch");
}

}  // namespace
}  // namespace rgd

using namespace rgd;

extern "C" int rgd_fp8_matmul(int32_t m, int32_t n, int32_t k, const uint8_t* x, int64_t x_stride, const float* x_scales,
                              const uint8_t* weights, int64_t w_stride, const float* w_scales, int32_t out_dtype, void* y,
                              int64_t y_stride, int32_t* dev_status, rgd_stream_t stream) {
  clear_error();
  const char* fn = "rgd_fp8_matmul";
  RGD_CHECK_ARG(m >= 0 && n >= 0 && k >= 1, "%s: m/n/k: m and n must not be negative and k at least 1", fn);
  RGD_CHECK_ARG(out_dtype == RGD_F32 || out_dtype == RGD_BF16, "%s: out_dtype must be RGD_F32 or RGD_BF16", fn);
  RGD_CHECK_ARG(k <= 1 << 24, "%s: k too large (max 2^24)", fn);
  RGD_CHECK_ARG(x_stride >= k && w_stride >= k && y_stride >= n, "%s: x_stride or w_stride is below k, or y_stride below n", fn);
  if (m > 1 << 30 || n > 1 << 30) return set_error(RGD_ERR_UNSUPPORTED, "%s: more than 2^30 rows", fn);
  if (m == 0 || n == 0) return RGD_OK;
  RGD_CHECK_ARG(x && x_scales && weights && w_scales && y, "%s: x/x_scales/weights/w_scales/y must be non-NULL", fn);
  RGD_CHECK_ARG(aligned16(x) && aligned16(weights) && aligned16(y) && x_stride % 16 == 0 && w_stride % 16 == 0,
                "%s: x, weights and y must be 16-byte aligned and x_stride and w_stride multiples of 16", fn);
  RGD_CHECK_ARG(reinterpret_cast<uintptr_t>(x_scales) % 4 == 0 && reinterpret_cast<uintptr_t>(w_scales) % 4 == 0,
                "%s: scales must be aligned to their elements", fn);
  RGD_CHECK_ARG(x_stride < (int64_t)1 << 40 && w_stride < (int64_t)1 << 40, "%s: strides must be below 2^40", fn);
  Fp8Params p{};
  p.m = m;
  p.n = n;
  p.steps = (int32_t)(((int64_t)k + kStep - 1) / kStep);
  p.sx = x_scales;
  p.sw = w_scales;
  p.y = static_cast<uint8_t*>(y);
  p.y_stride = y_stride;
  p.out_f32 = out_dtype == RGD_F32;
  p.vectors = y_stride * (p.out_f32 ? 4 : 2) % 16 == 0;
  p.dev_status = dev_status;
  const Fp8Operands o{x, weights, x_stride, w_stride, k};
  cudaStream_t st = (cudaStream_t)stream;
  if (m <= 32) return launch_fp8<32, true>(fn, p, o, st);
  if (m <= 64) return launch_fp8<64, true>(fn, p, o, st);
  if (m <= 128) return launch_fp8<128, true>(fn, p, o, st);
  // Pairs where that takes less time: a step of theirs is about 1.15 of a CTA's with 128 columns.  Their
  // results leave by TMA, which writes whole 16 bytes: rows of y start and end on them.
  const int64_t pairs = ((int64_t)m + 255) / 256 * (((int64_t)n + 255) / 256);
  const int64_t pair_cost = (pairs + kSms / 2 - 1) / (kSms / 2) * p.steps;
  const bool whole = p.vectors && (int64_t)n * (p.out_f32 ? 4 : 2) % 16 == 0;
  if (whole && pair_cost * 23 / 20 < best_split(((int64_t)m + 127) / 128 * (((int64_t)n + 127) / 128), p.steps).cost)
    return launch_fp8<256, false, true>(fn, p, o, st);
  return launch_fp8<128, false>(fn, p, o, st);
}
