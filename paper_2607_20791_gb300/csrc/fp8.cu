// Products of 8-bit floating-point activations and weights, each with a scale for every 128
// values of k:
//   y[i, j] = sum_b sx[i, b] sw[j / 128, b] sum_{k in block b} x[i, k] w[j, k].
//
// One block of k is four tensor core instructions (K = 32 each) into one of two TMEM
// accumulators; while the next block's run into the other, warps read the sums of the last
// one and add them, scaled, to what they hold in registers in fp32.  So a scale is applied
// once to 128 products' sum, whatever its value.
//
// The tensor core takes 128 rows (TMEM lanes) by up to 256 columns.  Many rows of x: x's are
// the lanes and w's the columns (a lane's scale is one number).  Few (up to 256): w's are the
// lanes and all of x's rows the columns, so that the weights are read once; bound by them.
// Where there are too few tiles for the SMs a cluster of CTAs shares one, each with a part
// of k, and they add their parts up in order: the same sums in every call.
//
// Warps: the first four (eight for 256 columns) add sums up, one copies tiles in by TMA, one
// issues the tensor core's instructions.
#include <cuda_bf16.h>

#include <algorithm>

#include "common.h"
#include "ptx.cuh"

namespace rgd {
namespace {

constexpr int kLanes = 128;              // rows of A a tile
constexpr int kStep = 128;               // values of k that share a scale: one step
constexpr int kABytes = kLanes * kStep;  // of a stage
constexpr int kMostStages = 12;
constexpr int kScaleSteps = 8;           // steps whose column scales are fetched together
constexpr int kRoom = 227 * 1024 - 1024;

struct Fp8Params {
  int32_t m, n, steps;  // steps of k
  const float* sx;
  const float* sw;
  uint8_t* y;
  int64_t y_stride;  // elements
  int32_t out_f32, vectors;
  int32_t a_tiles, tiles, split;  // tile t: A's tile t % a_tiles, B's t / a_tiles
  int32_t cols;                   // columns of a tile: the instructions' N
  int32_t stages;
  int32_t* dev_status;
};

struct Fp8Shared {
  uint64_t full[kMostStages], empty[kMostStages], sum_full[2], sum_empty[2], drained;
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
  const int part = lane & 3;
  const bool whole = p.vectors && (part + 1) * (16 / kSize) <= count;
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
  __syncwarp();
}

template <int NT>
constexpr int kFp8Threads = NT > 128 ? 384 : 192;

// NT: columns of a tile at most.  kTurned: w's rows are the lanes, x's the columns.
template <int NT, bool kTurned>
__global__ void __launch_bounds__(kFp8Threads<NT>, 1)
    fp8_kernel(const Fp8Params p, const __grid_constant__ CUtensorMap amap, const __grid_constant__ CUtensorMap bmap) {
  constexpr int kAdders = NT > 128 ? 256 : 128, kOwn = NT > 128 ? 128 : NT;  // threads that add up, columns of each
  constexpr int kProducer = kAdders / 32, kIssuer = kProducer + 1;
  constexpr uint32_t kTmemCols = 2 * NT < 32 ? 32 : 2 * NT;
  extern __shared__ uint8_t raw[];
  __shared__ Fp8Shared sh;
  __shared__ __align__(16) float scale[kTurned ? 2 : 1][kTurned ? kScaleSteps : 1][kTurned ? NT : 4];
  __shared__ uint32_t stage[kTurned ? 1 : kAdders * kStageWords];
  uint8_t* ring = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~uintptr_t(1023));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int stage_bytes = kABytes + p.cols * kStep;
  uint32_t rank = 0, tile0 = blockIdx.x, tile_step = gridDim.x;
  if (p.split > 1) {
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    asm volatile("mov.u32 %0, %%clusterid.x;" : "=r"(tile0));
    tile_step = (uint32_t)p.tiles;
  }
  const int step0 = (int)((int64_t)p.steps * rank / p.split), steps = (int)((int64_t)p.steps * (rank + 1) / p.split) - step0;
  const int total = ((p.tiles - 1 - (int)tile0) / (int)tile_step + 1) * steps;

  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");  // (a dependent waits for this kernel's end)
  if (warp == kIssuer) {
    tmem_alloc(&sh.tmem, kTmemCols);
    tmem_relinquish();
  }
  if (threadIdx.x == 0) {
    sh.dead = 0;
    for (int i = 0; i < p.stages; ++i) {
      mbar_init(&sh.full[i], 1);
      mbar_init(&sh.empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sh.sum_full[i], 1);
      mbar_init(&sh.sum_empty[i], kAdders / 32);
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
  tc_fence_after();
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const uint32_t tmem = sh.tmem;

  // 256 columns: 128 sums and more a thread, of the registers that the other four warps have left
  // (384 threads of 168 at launch: 256 of 232 and 128 of 40 are as many).
  int issued = 0;  // steps whose copies are on their way, or were
  if (warp >= kProducer) {
    if (NT > 128) asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
    if (warp == kProducer && lane == 0) {
      uint32_t tile = tile0;
      int at = 0, s = 0;
      uint32_t turn = 0;
      for (; issued < total; ++issued) {
        if (turn > 0 && !mbar_wait(&sh.empty[s], (turn - 1) & 1u)) {
          sh.dead = 1;
          break;
        }
        uint8_t* a = ring + s * stage_bytes;
        const int kx = (step0 + at) * kStep;
        mbar_arrive_expect_tx(&sh.full[s], (uint32_t)stage_bytes);
        tma_load_2d(a, &amap, &sh.full[s], kx, (int)(tile % (uint32_t)p.a_tiles) * kLanes);
        tma_load_2d(a + kABytes, &bmap, &sh.full[s], kx, (int)(tile / (uint32_t)p.a_tiles) * p.cols);
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
    if (warp == kIssuer && lane == 0) {
      const uint32_t idesc = idesc_e4m3_f32(kLanes, p.cols);
      int s = 0;
      uint32_t turn = 0;
      for (int q = 0; q < total; ++q) {
        const int b = q & 1;
        if ((q > 1 && !mbar_wait(&sh.sum_empty[b], (uint32_t)((q >> 1) - 1) & 1u)) || !mbar_wait(&sh.full[s], turn & 1u)) {
          sh.dead = 1;
          break;
        }
        tc_fence_after();
        uint64_t ad = smem_desc(smem_u32(ring + s * stage_bytes), 16, 1024, 2);
        uint64_t bd = smem_desc(smem_u32(ring + s * stage_bytes + kABytes), 16, 1024, 2);
#pragma unroll
        for (int i = 0; i < kStep / 32; ++i, ad += 2, bd += 2) umma_e4m3(tmem + b * NT, ad, bd, idesc, i > 0);
        umma_commit(&sh.empty[s]);
        umma_commit(&sh.sum_full[b]);
        if (++s == p.stages) {
          s = 0;
          ++turn;
        }
      }
    }
    __syncwarp();
  } else {
    if (NT > 128) asm volatile("setmaxnreg.inc.sync.aligned.u32 232;");
    const int half = warp >> 2, row = (warp & 3) * 32 + lane;  // of the tile's columns; the lane's row of A
    const int mine = kTurned ? min(max(p.cols - half * 128, 0), kOwn) : kOwn;
    const uint32_t at_tmem = tmem + ((uint32_t)(warp & 3) << 21) + half * 128;
    uint64_t acc[kOwn / 2];
#pragma unroll
    for (int i = 0; i < kOwn / 2; ++i) acc[i] = 0;
    // Column scales (w's lanes): of kScaleSteps steps together, a column a thread.
    float ahead[kScaleSteps];
    int ahead_at = 0;
    const float *ahead_x = p.sx + (int64_t)threadIdx.x * p.steps + step0, *ahead_w = p.sw + (int64_t)tile0 * p.steps + step0;
    auto fetch = [&](int count) {
#pragma unroll
      for (int i = 0; i < kScaleSteps; ++i) {
        ahead[i] = 0.f;
        if (i >= count) continue;
        if ((int)threadIdx.x < p.m) ahead[i] = __ldg(ahead_x + ahead_at) * __ldg(ahead_w + ahead_at);
        if (++ahead_at == steps) {  // (one column of tiles: the next is the next of w's rows)
          ahead_at = 0;
          ahead_w += (int64_t)tile_step * p.steps;
        }
      }
    };
    // The lane's scale (x's lanes), a step ahead.
    auto lane_scale = [&](int tile, int b) {
      const int64_t r = (int64_t)(tile % p.a_tiles) * kLanes + row;
      const int nb = min((int)(((int64_t)(tile / p.a_tiles) * p.cols + half * 128) / 128), (p.n - 1) / 128);
      return r < p.m ? __ldg(p.sx + r * p.steps + b) * __ldg(p.sw + (int64_t)nb * p.steps + b) : 0.f;
    };
    if (kTurned) fetch(total);
    int tile = (int)tile0, at = 0;
    float next = 0.f;
    if (!kTurned && total > 0) next = lane_scale(tile, step0);
#pragma unroll 1
    for (int q = 0; q < total; ++q) {
      const int b = q & 1;
      const float* columns = nullptr;
      uint64_t by = 0;
      if (kTurned) {
        const int part = q / kScaleSteps;
        if (q % kScaleSteps == 0) {
          if ((int)threadIdx.x < NT) {
#pragma unroll
            for (int i = 0; i < kScaleSteps; ++i) scale[part & 1][i][threadIdx.x] = ahead[i];
          }
          asm volatile("bar.sync 1, %0;" ::"n"(kAdders) : "memory");
          fetch(total - q - kScaleSteps);
        }
        columns = &scale[part & 1][q % kScaleSteps][half * 128];
      } else {
        by = pair2(next, next);
        const bool more = at + 1 < steps;
        if (q + 1 < total) next = lane_scale(more ? tile : tile + (int)tile_step, step0 + (more ? at + 1 : 0));
      }
      bool good = mbar_wait(&sh.sum_full[b], (uint32_t)(q >> 1) & 1u);
      good = __all_sync(0xffffffffu, good);
      if (!good) {
        sh.dead = 1;
        // (the others of this warp's barrier must not wait for it)
        if (kTurned)
          for (int c = (q / kScaleSteps + 1) * kScaleSteps; c < total; c += kScaleSteps) asm volatile("bar.sync 1, %0;" ::"n"(kAdders) : "memory");
        break;
      }
      tc_fence_after();
      uint32_t d[2][16];
      tmem_ld16(at_tmem + b * NT, d[0]);
#pragma unroll
      for (int c = 0; c < kOwn / 16; ++c) {
        if (c * 16 >= mine) break;
        tmem_ld_wait16(d[c & 1]);
        if ((c + 1) * 16 < mine && c + 1 < kOwn / 16) {
          tmem_ld16(at_tmem + b * NT + (c + 1) * 16, d[(c + 1) & 1]);
        } else {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&sh.sum_empty[b]);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          uint64_t f = by;
          if (kTurned) f = reinterpret_cast<const uint64_t*>(columns)[c * 8 + i];
          const uint64_t v = (uint64_t)d[c & 1][2 * i + 1] << 32 | d[c & 1][2 * i];
          acc[c * 8 + i] = fma_pair(v, f, acc[c * 8 + i]);
        }
      }
      if (mine == 0) {
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.sum_empty[b]);
      }
      if (++at < steps) continue;
      // The end of a tile.
      at = 0;
      const int64_t a0 = (int64_t)(tile % p.a_tiles) * kLanes + row, b0 = (int64_t)(tile / p.a_tiles) * p.cols + half * 128;
      tile += (int)tile_step;
      if (p.split > 1) {  // (the ring is free: every copy has been read)
        float* part = reinterpret_cast<float*>(ring) + half * 128 * (kLanes + 1) + row;
#pragma unroll
        for (int i = 0; i < kOwn / 2; ++i) {
          if (2 * i >= mine) break;
          float u, v;
          unpair2(acc[i], u, v);
          part[2 * i * (kLanes + 1)] = u;
          part[(2 * i + 1) * (kLanes + 1)] = v;
        }
        break;
      }
      const int es = p.out_f32 ? 4 : 2;
      if (kTurned) {
        const int count = a0 < p.n ? (int)min((int64_t)mine, p.m - b0) : 0;
        uint8_t* to = p.y + (b0 * p.y_stride + a0) * es;
#pragma unroll
        for (int i = 0; i < kOwn / 2; ++i) {
          float v[2];
          unpair2(acc[i], v[0], v[1]);
#pragma unroll
          for (int j = 0; j < 2; ++j, to += p.y_stride * es) put_if(2 * i + j < count, to, p.out_f32, v[j]);
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
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (p.split > 1) {  // the parts, in order of k, by the CTA whose columns they are
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    const int c0 = p.cols * (int)rank / p.split, c1 = p.cols * (int)(rank + 1) / p.split, width = c1 - c0;
    const int64_t a0 = (int64_t)(tile0 % (uint32_t)p.a_tiles) * kLanes, b0 = (int64_t)(tile0 / (uint32_t)p.a_tiles) * p.cols;
    for (int e = threadIdx.x; e < width * kLanes; e += kFp8Threads<NT>) {
      const int col = c0 + (kTurned ? e / kLanes : e % width), row = kTurned ? e % kLanes : e / width;
      const uint32_t from = smem_u32(reinterpret_cast<float*>(ring) + col * (kLanes + 1) + row);
      float v = 0.f;
      for (int r = 0; r < p.split; ++r) {
        uint32_t there;
        float x;
        asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(from), "r"(r));
        asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(x) : "r"(there) : "memory");
        v += x;
      }
      if (kTurned) write_one(p, b0 + col, a0 + row, v);
      else write_one(p, a0 + row, b0 + col, v);
    }
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  }
  if (sh.dead) {  // copies and instructions in flight end before the memory that they use is given up
    if (threadIdx.x == 0 && p.dev_status) atomicOr(p.dev_status, RGD_DEV_WAIT_TIMEOUT);
    for (int i = max(0, issued - p.stages); i < issued; ++i) mbar_wait(&sh.full[i % p.stages], (uint32_t)(i / p.stages) & 1u);
    if (warp == kIssuer && lane == 0) {
      umma_commit(&sh.drained);
      mbar_wait(&sh.drained, 0);
    }
    __syncthreads();
  }
  if (warp == kIssuer) tmem_dealloc(tmem, kTmemCols);
}

int encode_rows(CUtensorMap* map, const void* base, int64_t k, int64_t rows, int64_t stride, int box_rows) {
  const auto encode = tensor_map_encoder();
  if (!encode) return set_error(RGD_ERR_CUDA, "cuTensorMapEncodeTiled is unavailable");
  const cuuint64_t dims[2] = {(cuuint64_t)k, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)stride};
  const cuuint32_t box[2] = {kStep, (cuuint32_t)box_rows}, ones[2] = {1, 1};
  const CUresult r = encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dims, strides, box, ones,
                            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? RGD_OK : set_error(RGD_ERR_CUDA, "cuTensorMapEncodeTiled failed (%d)", (int)r);
}

struct Fp8Operands {
  const uint8_t* x;
  const uint8_t* w;
  int64_t x_stride, w_stride, k;
};

template <int NT, bool kTurned>
int launch_fp8(const char* fn, Fp8Params& p, const Fp8Operands& o, cudaStream_t st) {
  static std::atomic<bool> done[kMaxDevices];
  auto k = fp8_kernel<NT, kTurned>;
  constexpr int room = kRoom - (kTurned ? 2 * kScaleSteps * NT * 4 : (NT > 128 ? 256 : 128) * kStageWords * 4) - 512;
  if (int rc = ensure_smem(k, room + 1024, done)) return rc;
  p.cols = kTurned ? (p.m + 15) / 16 * 16 : NT;
  const int64_t a_tiles = ((int64_t)(kTurned ? p.n : p.m) + kLanes - 1) / kLanes;
  const int64_t b_tiles = ((int64_t)(kTurned ? p.m : p.n) + p.cols - 1) / p.cols, tiles = a_tiles * b_tiles;
  if (tiles > 0x7fffffff / p.steps - 1) return set_error(RGD_ERR_UNSUPPORTED, "%s: too many tiles", fn);
  p.a_tiles = (int32_t)a_tiles;
  p.tiles = (int32_t)tiles;
  const int stage = kABytes + p.cols * kStep;
  p.stages = std::min(kMostStages, room / stage);
  // Too few tiles for the SMs: clusters of up to 8 CTAs share one, each with two steps at least.
  constexpr int sms = 152;
  p.split = (int)std::max<int64_t>(1, std::min<int64_t>({8, sms / tiles, p.steps / 2}));
  const int grid = p.split > 1 ? p.tiles * p.split : (int)std::min<int64_t>(tiles, sms);
  CUtensorMap amap, bmap;
  const uint8_t *a = kTurned ? o.w : o.x, *b = kTurned ? o.x : o.w;
  const int64_t as = kTurned ? o.w_stride : o.x_stride, bs = kTurned ? o.x_stride : o.w_stride;
  if (int rc = encode_rows(&amap, a, o.k, kTurned ? p.n : p.m, as, kLanes)) return rc;
  if (int rc = encode_rows(&bmap, b, o.k, kTurned ? p.m : p.n, bs, p.cols)) return rc;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)grid);
  cfg.blockDim = dim3(kFp8Threads<NT>);
  cfg.dynamicSmemBytes = (size_t)p.stages * stage + 1024;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim = {(unsigned)p.split, 1, 1};
  cfg.attrs = attr;
  cfg.numAttrs = p.split > 1 ? 2 : 1;
  cudaError_t e = cudaLaunchKernelEx(&cfg, k, p, amap, bmap);
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
  if (m <= 256) return launch_fp8<256, true>(fn, p, o, st);
  if (((int64_t)m + 127) / 128 * (((int64_t)n + 255) / 256) >= 152) return launch_fp8<256, false>(fn, p, o, st);
  return launch_fp8<128, false>(fn, p, o, st);
}
