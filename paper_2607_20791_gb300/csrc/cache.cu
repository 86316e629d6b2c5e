// The paged KV cache's own operations: pages for new tokens (with a copy of a shared
// page before it is written), the tokens' keys and values into them, rows forked and
// trimmed, pages copied, and the pool compacted.
//
// A page is free exactly if its count in page_refs is 0, and an allocation takes the
// free page of the lowest number.  So there is no free list that could disagree with the
// counts, giving a page back is one atomic decrement, in any order, and every result is
// a function of the tables and counts alone.  The price is a look through the counts
// when pages are needed: one cluster of eight blocks, 16 counts a thread at a time, takes
// 10 us for 2048 rows and 69 thousand pages where one block of 4 counts a thread took 19.
#include <algorithm>
#include <cmath>

#include "common.h"
#include "ptx.cuh"

namespace rgd {
namespace {

constexpr int kPageSize = 16;
constexpr int kPlanThreads = 1024;
constexpr int kCopyThreads = 256;

struct CacheView {
  int32_t layers, pages, heads, dim;
  int64_t layer_stride;  // elements between a layer's pool and the next
};

__device__ __forceinline__ void begin_dependent() {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");  // (a dependent waits for this kernel's end)
  asm volatile("griddepcontrol.wait;" ::: "memory");
}
__device__ __forceinline__ void flag(int32_t* dev_status, int32_t bit) {
  if (dev_status) atomicOr(dev_status, bit);
}

// Exclusive prefix sum over the block's threads, and the total.
__device__ __forceinline__ int32_t block_scan(int32_t v, int32_t* part, int32_t& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int32_t incl = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int32_t x = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += x;
  }
  __syncthreads();  // (part may still be read from the scan before)
  if (lane == 31) part[warp] = incl;
  __syncthreads();
  int32_t w = part[lane];
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int32_t x = __shfl_up_sync(0xffffffffu, w, o);
    if (lane >= o) w += x;
  }
  total = __shfl_sync(0xffffffffu, w, 31);
  const int32_t before = __shfl_sync(0xffffffffu, w, (warp + 31) & 31);
  return incl - v + (warp ? before : 0);
}

// A plan is made by one cluster of blocks, each with an equal share of the rows and of the pages.
constexpr int kPlanBlocks = 8;
constexpr int kEach = 16;                         // counts a thread looks at together
constexpr int kSweep = kPlanThreads * kEach;      // ... and a block

struct PlanShared {
  int32_t part[32];
  int32_t sums[2][2][kPlanBlocks];  // two sums of every block, for up to two exchanges
  int32_t copies;
};

// Of all the plan's threads; what was written before it is seen after it.
__device__ __forceinline__ void plan_barrier(int blocks) {
  if (blocks == 1) {
    __syncthreads();
  } else {
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  }
}

// Gives every block the sums a and b of all blocks, and waits for it: `before` those of the
// blocks of lower rank, `total` those of all.
__device__ __forceinline__ void plan_exchange(PlanShared& sh, int which, int32_t a, int32_t b, int rank, int blocks,
                                              int32_t (&before)[2], int32_t (&total)[2]) {
  if (blocks == 1) {
    before[0] = before[1] = 0;
    total[0] = a;
    total[1] = b;
    return;
  }
  if (threadIdx.x < 2 * blocks) {
    const uint32_t slot = smem_u32(&sh.sums[which][threadIdx.x & 1][rank]);
    uint32_t at;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(slot), "r"(threadIdx.x >> 1));
    asm volatile("st.shared::cluster.b32 [%0], %1;" ::"r"(at), "r"((threadIdx.x & 1) ? b : a) : "memory");
  }
  plan_barrier(blocks);
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    before[k] = total[k] = 0;
    for (int i = 0; i < blocks; ++i) {
      before[k] += i < rank ? sh.sums[which][k][i] : 0;
      total[k] += sh.sums[which][k][i];
    }
  }
}

// Which of pages base .. base + 15 are in use, as bits; those from `end` on are `outside`.
__device__ __forceinline__ uint32_t used_mask(const int32_t* refs, int64_t base, int64_t end, bool outside) {
  uint32_t mask = 0;
  if (base + kEach <= end && (reinterpret_cast<uintptr_t>(refs + base) & 15u) == 0) {
    int4 v[kEach / 4];
#pragma unroll
    for (int i = 0; i < kEach / 4; ++i) v[i] = *reinterpret_cast<const int4*>(refs + base + 4 * i);
#pragma unroll
    for (int i = 0; i < kEach / 4; ++i)
      mask |= ((v[i].x > 0 ? 1u : 0u) | (v[i].y > 0 ? 2u : 0u) | (v[i].z > 0 ? 4u : 0u) | (v[i].w > 0 ? 8u : 0u)) << (4 * i);
    return mask;
  }
#pragma unroll
  for (int i = 0; i < kEach; ++i) mask |= (base + i < end ? refs[base + i] > 0 : outside) ? 1u << i : 0u;
  return mask;
}

// ---------------------------------------------------------------------------
// copies of pages
// ---------------------------------------------------------------------------
struct CopyParams {
  CacheView c;
  uint16_t* pool[2];  // keys, values
  const int32_t* count;  // copies to make (NULL: n)
  int32_t n;
  const int32_t* src;
  const int32_t* dst;
  const int32_t* slots;  // leading slots of each to copy (NULL: all)
  int32_t* dev_status;
  // compaction: tables whose entries at or above *live move as `place` says
  const int32_t* live;
  const int32_t* place;
  int32_t* table[2];
  int64_t entries[2];
};

// A warp copies one layer's, pool's and head's part of copy i: up to 16 x D elements,
// contiguous on both sides, all loads before the stores.
__device__ __forceinline__ void copy_piece(const CopyParams& p, int32_t i, int32_t part, int lane) {
  const int32_t head = part % p.c.heads, pool = part / p.c.heads % 2, layer = part / p.c.heads / 2;
  const int32_t s = p.src[i], d = p.dst[i];
  if (s < 0 || s >= p.c.pages || d < 0 || d >= p.c.pages) {
    flag(p.dev_status, RGD_DEV_BAD_PAGE);
    return;
  }
  const int32_t vecs = (p.slots ? p.slots[i] : kPageSize) * p.c.dim / 8;
  uint16_t* base = p.pool[pool] + layer * p.c.layer_stride;
  const int64_t page = (int64_t)kPageSize * p.c.dim;
  const uint4* from = reinterpret_cast<const uint4*>(base + ((int64_t)s * p.c.heads + head) * page);
  uint4* to = reinterpret_cast<uint4*>(base + ((int64_t)d * p.c.heads + head) * page);
  for (int v = lane; v < vecs; v += 32 * 8) {
    uint4 x[8];
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (v + k * 32 < vecs) x[k] = from[v + k * 32];
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (v + k * 32 < vecs) to[v + k * 32] = x[k];
  }
}

__global__ void __launch_bounds__(kCopyThreads) copy_kernel(const CopyParams p) {
  begin_dependent();
  const int lane = threadIdx.x & 31;
  const int64_t warps = (int64_t)gridDim.x * (kCopyThreads / 32);
  const int64_t w0 = (int64_t)blockIdx.x * (kCopyThreads / 32) + (threadIdx.x >> 5);
  if (p.live) {
    const int32_t live = *p.live;
    for (int k = 0; k < 2; ++k)
      for (int64_t i = w0 * 32 + lane; i < p.entries[k]; i += warps * 32) {
        const int32_t e = p.table[k][i];
        if (e < live) continue;
        const int32_t to = e < p.c.pages ? p.place[e] : -1;
        if (to < 0) flag(p.dev_status, RGD_DEV_BAD_PAGE);
        p.table[k][i] = to;
      }
  }
  const int32_t n = p.count ? *p.count : p.n;
  const int per_page = p.c.layers * 2 * p.c.heads;
  for (int64_t w = w0; w < (int64_t)n * per_page; w += warps) {
    copy_piece(p, (int32_t)(w / per_page), (int32_t)(w % per_page), lane);
  }
}

// ---------------------------------------------------------------------------
// pages for new tokens
// ---------------------------------------------------------------------------
struct ReserveParams {
  int32_t rows, cols, pages;
  int32_t* table;
  const int32_t* length;
  const int32_t* n_new;
  const uint8_t* row_active;
  int32_t* refs;
  uint8_t* row_ok;
  int32_t* num_copies;  // workspace: copies to make, then source, target and slots of each
  int32_t* src;
  int32_t* dst;
  int32_t* slots;
  int32_t* need;   // workspace [rows]: where the row's pages start among its block's
  int32_t* fresh;  // workspace [pages]: the free pages in order, as many as are needed
  int32_t* dev_status;
  int32_t copy_here;  // the copies are few enough for this kernel
  CopyParams copy;
};

// A row's new tokens: the columns they fall into, and which of those want a page (the first
// 32 as bits).
struct NewTokens {
  int32_t len, first, last, pages;
  uint32_t wants;
  bool bad;
};
__device__ __forceinline__ bool wants_page(const ReserveParams& p, int32_t page) {
  return page < 0 || (page < p.pages && p.refs[page] > 1);
}
__device__ __forceinline__ NewTokens look_at(const ReserveParams& p, int r, bool in_turn) {
  NewTokens t = {};
  if (!in_turn) return t;
  t.len = p.length[r];  // (all three at once)
  const int32_t n = p.n_new[r];
  if (p.row_active && !p.row_active[r]) return {};
  t.bad = t.len < 0 || n < 0 || (int64_t)t.len + n > (int64_t)p.cols * kPageSize;
  if (t.bad || n == 0) return t;
  t.first = t.len / kPageSize;
  t.last = (t.len + n + kPageSize - 1) / kPageSize;
  for (int j = t.first; j < t.last; ++j) {
    const int32_t page = p.table[(int64_t)r * p.cols + j];
    t.bad = t.bad || page >= p.pages;
    if (!wants_page(p, page)) continue;
    ++t.pages;
    if (j - t.first < 32) t.wants |= 1u << (j - t.first);
  }
  if (t.bad) t.pages = 0;
  return t;
}

__global__ void __launch_bounds__(kPlanThreads) reserve_kernel(const ReserveParams p) {
  __shared__ PlanShared sh;
  uint32_t rank_u, blocks_u;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank_u));
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(blocks_u));
  const int rank = (int)rank_u, blocks = (int)blocks_u, tid = threadIdx.x;
  if (blocks > 1) plan_barrier(blocks);  // (every block has started)
  begin_dependent();
  const int share = (p.rows + blocks - 1) / blocks, r0 = min(rank * share, p.rows), r1 = min(r0 + share, p.rows);
  const int64_t span = ((int64_t)p.pages + blocks * 4 - 1) / (blocks * 4) * 4;
  const int64_t p0 = min(rank * span, (int64_t)p.pages), p1 = min(p0 + span, (int64_t)p.pages);
  int32_t* copies_made = blocks == 1 ? &sh.copies : p.num_copies;
  if (rank == 0 && tid == 0) *copies_made = 0;
  // the counts' first sweep is on its way while the rows are looked at
  const uint32_t used = used_mask(p.refs, p0 + tid * kEach, p1, true);
  // how many pages each row needs, and where they start among the block's
  const bool once = share <= kPlanThreads;  // (a thread then keeps what it knows of its row)
  NewTokens t = {};
  int32_t needed = 0, at = 0;
  for (int base = r0; base < r1; base += kPlanThreads) {
    const int r = base + tid;
    t = look_at(p, r, r < r1);
    if (t.bad) flag(p.dev_status, RGD_DEV_BAD_PAGE);
    int32_t total;
    at = needed + block_scan(t.pages, sh.part, total);
    if (!once && r < r1) p.need[r] = at;
    needed += total;
  }
  int32_t free = 0;
  for (int64_t base = p0; base < p1; base += kSweep) {
    const uint32_t m = base == p0 ? used : used_mask(p.refs, base + tid * kEach, p1, true);
    int32_t total;
    block_scan(kEach - __popc(m), sh.part, total);
    free += total;
  }
  int32_t before[2], all[2];
  plan_exchange(sh, 0, needed, free, rank, blocks, before, all);
  // the free pages of the lowest numbers, as many as are needed
  int32_t found = before[1];
  for (int64_t base = p0; base < p1 && found < all[0]; base += kSweep) {
    const int64_t first = base + tid * kEach;
    uint32_t m = ~(base == p0 ? used : used_mask(p.refs, first, p1, true)) & ((1u << kEach) - 1);
    int32_t total;
    int32_t to = found + block_scan(__popc(m), sh.part, total);
    found += total;
    for (; m && to < all[0]; m &= m - 1) p.fresh[to++] = (int32_t)(first + __ffs(m) - 1);
  }
  plan_barrier(blocks);
  // the rows' pages, in order, as far as they go; pages given up are noted, so that no
  // count changes while rows still read them
  for (int r = r0 + tid; r < r1; r += kPlanThreads) {
    if (!once) {
      t = look_at(p, r, true);
      at = p.need[r];
    }
    at += before[0];
    const bool ok = !t.bad && at + t.pages <= all[1] && (!p.row_active || p.row_active[r]);
    if (p.row_ok) p.row_ok[r] = ok;
    if (t.pages == 0) continue;
    if (!ok) {
      flag(p.dev_status, RGD_DEV_NO_PAGE);
      continue;
    }
    int32_t* row = p.table + (int64_t)r * p.cols;
    for (int j = t.first; j < t.last; ++j) {
      const bool known = j - t.first < 32;
      if (known && !(t.wants >> (j - t.first) & 1u)) continue;
      const int32_t old = row[j];
      if (!known && !wants_page(p, old)) continue;
      const int32_t page = p.fresh[at++];
      if (old >= 0) {
        const int32_t i = atomicAdd(copies_made, 1);
        p.src[i] = old;
        p.dst[i] = page;
        p.slots[i] = j == t.first ? t.len % kPageSize : 0;
      }
      row[j] = page;
      p.refs[page] = 1;
    }
  }
  plan_barrier(blocks);
  const int32_t copies = blocks == 1 ? sh.copies : __ldcg(p.num_copies);
  if (blocks == 1 && tid == 0) *p.num_copies = copies;
  for (int i = rank * kPlanThreads + tid; i < copies; i += blocks * kPlanThreads) atomicSub(p.refs + p.src[i], 1);
  if (!p.copy_here) return;
  const int per_page = p.copy.c.layers * 2 * p.copy.c.heads;
  for (int w = rank * (kPlanThreads / 32) + (tid >> 5); w < copies * per_page; w += blocks * (kPlanThreads / 32))
    copy_piece(p.copy, w / per_page, w % per_page, tid & 31);
}

// ---------------------------------------------------------------------------
// keys and values of new tokens
// ---------------------------------------------------------------------------
struct WriteParams {
  CacheView c;
  uint16_t* pool[2];
  const uint16_t* fresh[2];
  int64_t row_stride, token_stride;
  int32_t rows, tokens, cols;
  const int32_t* n_new;
  const int32_t* table;
  const int32_t* length;
  const uint8_t* row_ok;
  int32_t* dev_status;
};

// A warp writes one token's keys and values.
__global__ void __launch_bounds__(kCopyThreads) write_kernel(const WriteParams p) {
  begin_dependent();
  const int lane = threadIdx.x & 31;
  const int64_t w = (int64_t)blockIdx.x * (kCopyThreads / 32) + (threadIdx.x >> 5);
  const int32_t r = (int32_t)(w / p.tokens), i = (int32_t)(w % p.tokens);
  if (r >= p.rows) return;
  const int32_t n = p.n_new[r], len = p.length[r];
  if (p.row_ok && !p.row_ok[r]) return;
  if (i == 0 && lane == 0 && (n < 0 || n > p.tokens)) flag(p.dev_status, RGD_DEV_BAD_PAGE);
  if (i >= n) return;
  const int32_t per = p.c.dim / 8, vecs = p.c.heads * per;
  const int64_t at = r * p.row_stride + i * p.token_stride;
  const uint4* fresh[2] = {reinterpret_cast<const uint4*>(p.fresh[0] + at), reinterpret_cast<const uint4*>(p.fresh[1] + at)};
  // The first vectors are on their way while the page is looked up, eight a lane (one after the
  // other, 2048 rows of 8 tokens took 36 us with their pages' plan, so 33).
  constexpr int kBatch = 4;
  uint4 v[2][kBatch];
  auto load = [&](int first) {
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int b = 0; b < kBatch; ++b)
        if (first + 32 * b < vecs) v[s][b] = __ldcs(fresh[s] + first + 32 * b);
  };
  load(lane);
  const int64_t pos = (int64_t)len + i;
  const int32_t page = pos >= 0 && pos < (int64_t)p.cols * kPageSize ? p.table[(int64_t)r * p.cols + pos / kPageSize] : -1;
  if (page < 0 || page >= p.c.pages) {
    if (lane == 0) flag(p.dev_status, RGD_DEV_BAD_PAGE);
    return;
  }
  const int64_t to = ((int64_t)page * p.c.heads * kPageSize + pos % kPageSize) * per;
#pragma unroll 1
  for (int first = lane;;) {
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      const int x = first + 32 * b, h = x / per;
      if (x >= vecs) continue;
      const int64_t o = to + (int64_t)h * kPageSize * per + (x - h * per);
      reinterpret_cast<uint4*>(p.pool[0])[o] = v[0][b];
      reinterpret_cast<uint4*>(p.pool[1])[o] = v[1][b];
    }
    first += 32 * kBatch;
    if (first >= vecs) return;
    load(first);
  }
}

// ---------------------------------------------------------------------------
// pages taken up and given back with rows
// ---------------------------------------------------------------------------
// A warp per row gives back its pages past the row's length.
__global__ void __launch_bounds__(kCopyThreads)
    trim_kernel(int32_t rows, int32_t cols, int32_t pages, int32_t* table, const int32_t* length, const uint8_t* row_active,
                int32_t* refs, int32_t* dev_status) {
  begin_dependent();
  const int r = blockIdx.x * (kCopyThreads / 32) + (threadIdx.x >> 5);
  if (r >= rows || (row_active && !row_active[r])) return;
  const int32_t len = length[r];
  if (len < 0) {
    flag(dev_status, RGD_DEV_BAD_PAGE);
    return;
  }
  for (int64_t j = ((int64_t)len + kPageSize - 1) / kPageSize + (threadIdx.x & 31); j < cols; j += 32) {
    int32_t* e = table + (int64_t)r * cols + j;
    const int32_t page = *e;
    if (page < 0) continue;
    if (page < pages) atomicSub(refs + page, 1);
    else flag(dev_status, RGD_DEV_BAD_PAGE);
    *e = -1;
  }
}

// A warp per pair gives the child the parent's pages and length.
__global__ void __launch_bounds__(kCopyThreads)
    fork_kernel(int32_t n, int32_t rows, int32_t cols, int32_t pages, const int32_t* parent, const int32_t* child,
                int32_t* table, int32_t* length, int32_t* refs, int32_t* dev_status) {
  begin_dependent();
  const int i = blockIdx.x * (kCopyThreads / 32) + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  if (i >= n) return;
  const int32_t a = parent[i], b = child[i];
  const int32_t len = a >= 0 && a < rows ? length[a] : -1;
  if (b < 0 || b >= rows || a == b || len < 0 || len > (int64_t)cols * kPageSize) {
    flag(dev_status, RGD_DEV_BAD_PAGE);
    return;
  }
  const int32_t held = (int32_t)(((int64_t)len + kPageSize - 1) / kPageSize);
  for (int j = lane; j < cols; j += 32) {
    const int32_t page = j < held ? table[(int64_t)a * cols + j] : -1;
    if (page >= 0 && page < pages) atomicAdd(refs + page, 1);
    else if (j < held) flag(dev_status, RGD_DEV_BAD_PAGE);
    table[(int64_t)b * cols + j] = page;
  }
  if (lane == 0) length[b] = len;
}

// ---------------------------------------------------------------------------
// the pool compacted
// ---------------------------------------------------------------------------
// The i-th page in use at or above the number of pages in use moves to the i-th free page
// below it: the fewest moves, and no target is a source.
__global__ void __launch_bounds__(kPlanThreads)
    compact_kernel(int32_t pages, int32_t* refs, int32_t* num_live, int32_t* num_moves, int32_t* src, int32_t* dst,
                   int32_t* place) {
  __shared__ PlanShared sh;
  uint32_t rank_u, blocks_u;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank_u));
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(blocks_u));
  const int rank = (int)rank_u, blocks = (int)blocks_u, tid = threadIdx.x;
  if (blocks > 1) plan_barrier(blocks);  // (every block has started)
  begin_dependent();
  const int64_t span = ((int64_t)pages + blocks * 4 - 1) / (blocks * 4) * 4;
  const int64_t p0 = min(rank * span, (int64_t)pages), p1 = min(p0 + span, (int64_t)pages);
  constexpr uint32_t kAll = (1u << kEach) - 1;
  uint32_t first_sweep = used_mask(refs, p0 + tid * kEach, p1, false);
  auto used_at = [&](int64_t base) { return base == p0 ? first_sweep : used_mask(refs, base + tid * kEach, p1, false); };
  int32_t mine = 0, before[2], all[2], total;
  for (int64_t base = p0; base < p1; base += kSweep) {
    block_scan(__popc(used_at(base)), sh.part, total);
    mine += total;
  }
  plan_exchange(sh, 0, mine, 0, rank, blocks, before, all);
  const int32_t live = all[0];
  // Of a thread's pages: those that move, and the places that are free for them.
  auto split = [&](int64_t base, uint32_t& movers, uint32_t& holes) {
    const int64_t at = base + tid * kEach;
    const uint32_t used = used_at(base);
    const uint32_t low = at >= live ? 0 : live - at >= kEach ? kAll : (1u << (live - at)) - 1;  // pages below `live`
    movers = used & ~low;
    holes = ~used & low;  // (pages past this block's end are not below `live` of it: see the count)
    if (at >= p1) holes = 0;
    else if (at + kEach > p1) holes &= (1u << (p1 - at)) - 1;
  };
  int32_t moving = 0, open = 0;
  for (int64_t base = p0; base < p1; base += kSweep) {
    uint32_t movers, holes;
    split(base, movers, holes);
    block_scan(__popc(movers) << 16 | __popc(holes), sh.part, total);  // (at most 16384 of each)
    moving += total >> 16;
    open += total & 0xffff;
  }
  plan_exchange(sh, 1, moving, open, rank, blocks, before, all);
  const int32_t moves = all[0];
  for (int64_t base = p0; base < p1; base += kSweep) {
    const int64_t at = base + tid * kEach;
    uint32_t movers, holes;
    split(base, movers, holes);
    const int32_t scan = block_scan(__popc(movers) << 16 | __popc(holes), sh.part, total);
    int32_t m = before[0] + (scan >> 16), h = before[1] + (scan & 0xffff);
    before[0] += total >> 16;
    before[1] += total & 0xffff;
    for (int i = 0; i < kEach; ++i)
      if (at + i >= live && at + i < p1 && !(movers >> i & 1u)) place[at + i] = -1;
    for (; movers; movers &= movers - 1) src[m++] = (int32_t)(at + __ffs(movers) - 1);
    for (; holes; holes &= holes - 1) dst[h++] = (int32_t)(at + __ffs(holes) - 1);
  }
  plan_barrier(blocks);
  for (int i = rank * kPlanThreads + tid; i < moves; i += blocks * kPlanThreads) {
    const int32_t from = __ldcg(src + i), to = __ldcg(dst + i);
    place[from] = to;
    refs[to] = refs[from];
    refs[from] = 0;
  }
  if (rank == 0 && tid == 0) {
    *num_live = live;
    *num_moves = moves;
  }
}

// Launches a plan's cluster, as a programmatic dependent.
template <typename... P, typename... A>
cudaError_t launch_plan(void (*kernel)(P...), int blocks, cudaStream_t st, A&&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)blocks);
  cfg.blockDim = dim3(kPlanThreads);
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim = {(unsigned)blocks, 1, 1};
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = blocks > 1 ? attr : attr + 1;
  cfg.numAttrs = blocks > 1 ? 2 : 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, P(args)...);
  return e == cudaSuccess ? cudaGetLastError() : e;
}

// Blocks of a plan: one does for what it sees in a single sweep.
int plan_blocks(int32_t rows, int32_t pages) { return rows <= kPlanThreads && pages <= kSweep ? 1 : kPlanBlocks; }

int check_shape(const char* fn, const rgd_cache_shape* s, CacheView& c) {
  RGD_CHECK_ARG(s != nullptr, "%s: shape is NULL", fn);
  RGD_CHECK_ARG(s->num_layers >= 1 && s->num_pages >= 1 && s->num_kv_heads >= 1 && s->head_dim >= 1,
                "%s: num_layers/num_pages/num_kv_heads/head_dim must be >= 1", fn);
  RGD_CHECK_ARG(s->reserved == 0, "%s: reserved must be 0", fn);
  if (s->page_size != kPageSize) return set_error(RGD_ERR_UNSUPPORTED, "%s: page_size must be 16", fn);
  if (s->head_dim % 8 != 0 || s->head_dim > 1024)
    return set_error(RGD_ERR_UNSUPPORTED, "%s: head_dim must be a multiple of 8, at most 1024", fn);
  if (s->num_kv_heads > 4096 || s->num_layers > 4096)
    return set_error(RGD_ERR_UNSUPPORTED, "%s: at most 4096 heads and layers", fn);
  const int64_t pool = (int64_t)s->num_pages * s->num_kv_heads * kPageSize * s->head_dim;
  RGD_CHECK_ARG(s->layer_stride == 0 || (s->layer_stride >= pool && s->layer_stride % 8 == 0),
                "%s: layer_stride must be 0 or a multiple of 8 no smaller than a layer's pool", fn);
  c = CacheView{s->num_layers, s->num_pages, s->num_kv_heads, s->head_dim, s->layer_stride ? s->layer_stride : pool};
  return RGD_OK;
}

constexpr int kWarpsEach = kCopyThreads / 32;
// Rows (or pairs, or tokens) at most: the numbers that a last block gives to those past the end are still an int.
constexpr int32_t kMaxRows = 0x7fffffff - kPlanThreads;

int launch_copies(const CopyParams& p, int64_t most, cudaStream_t st) {
  const int64_t warps = std::max(most * p.c.layers * 2 * p.c.heads, (p.entries[0] + p.entries[1] + 31) / 32);
  const int grid = blocks_for(std::max<int64_t>(warps, 1), kWarpsEach, 152 * 8);
  const cudaError_t e = launch_dependent(copy_kernel, grid, kCopyThreads, 0, st, p);
  return e == cudaSuccess ? RGD_OK : cuda_error(e, "cache copy launch");
}

}  // namespace
}  // namespace rgd

using namespace rgd;

extern "C" size_t rgd_cache_workspace_size(const rgd_cache_shape* shape, int32_t rows) {
  clear_error();
  CacheView c;
  if (check_shape("rgd_cache_workspace_size", shape, c)) return 0;
  if (rows < 0) {
    set_error(RGD_ERR_INVALID_ARG, "rgd_cache_workspace_size: rows < 0");
    return 0;
  }
  return 256 + 4 * (4 * (size_t)c.pages + (size_t)rows);
}

extern "C" int rgd_cache_reserve(const rgd_cache_shape* shape, int32_t rows, int32_t max_pages, int32_t* block_table,
                                 const int32_t* length, const int32_t* n_new, const uint8_t* row_active,
                                 int32_t* page_refs, rgd_bf16* k_pages, rgd_bf16* v_pages, uint8_t* row_ok,
                                 void* workspace, size_t workspace_bytes, int32_t* dev_status, rgd_stream_t stream) {
  clear_error();
  const char* fn = "rgd_cache_reserve";
  CacheView c;
  if (int rc = check_shape(fn, shape, c)) return rc;
  RGD_CHECK_ARG(rows >= 0 && max_pages >= 1, "%s: bad rows/max_pages", fn);
  if (rows == 0) return RGD_OK;
  // (the kernel adds up the pages that rows want in 32 bits)
  if ((int64_t)rows * max_pages > 0x7fffffff)
    return set_error(RGD_ERR_UNSUPPORTED, "%s: block_table must have fewer than 2^31 entries", fn);
  RGD_CHECK_ARG(rows <= kMaxRows, "%s: too many rows", fn);
  RGD_CHECK_ARG(block_table && length && n_new && page_refs && k_pages && v_pages && workspace,
                "%s: block_table/length/n_new/page_refs/k_pages/v_pages/workspace must be non-NULL", fn);
  RGD_CHECK_ARG(aligned16(k_pages) && aligned16(v_pages) && aligned16(workspace),
                "%s: k_pages/v_pages/workspace must be 16-byte aligned", fn);
  RGD_CHECK_ARG(workspace_bytes >= rgd_cache_workspace_size(shape, rows), "%s: workspace too small", fn);
  RGD_CHECK_ARG(max_pages <= 0x7fffffff / kPageSize, "%s: max_pages too large", fn);
  cudaStream_t st = (cudaStream_t)stream;
  int32_t* ws = static_cast<int32_t*>(workspace);
  ReserveParams p{};
  p.rows = rows;
  p.cols = max_pages;
  p.pages = c.pages;
  p.table = block_table;
  p.length = length;
  p.n_new = n_new;
  p.row_active = row_active;
  p.refs = page_refs;
  p.row_ok = row_ok;
  p.num_copies = ws;
  p.src = ws + 64;
  p.dst = p.src + c.pages;
  p.slots = p.dst + c.pages;
  p.fresh = p.slots + c.pages;
  p.need = p.fresh + c.pages;
  p.dev_status = dev_status;
  CopyParams& q = p.copy;
  q.c = c;
  q.pool[0] = k_pages;
  q.pool[1] = v_pages;
  q.count = p.num_copies;
  q.src = p.src;
  q.dst = p.dst;
  q.slots = p.slots;
  q.dev_status = dev_status;
  const int blocks = plan_blocks(rows, c.pages);
  // up to four pieces a warp are copied by the plan's own block: a second kernel costs more
  // (about 2 us on the host and on the GPU)
  p.copy_here = (int64_t)rows * c.layers * 2 * c.heads <= 4 * (kPlanThreads / 32) * blocks;
  const cudaError_t e = launch_plan(reserve_kernel, blocks, st, p);
  if (e != cudaSuccess) return cuda_error(e, "cache reserve launch");
  return p.copy_here ? RGD_OK : launch_copies(q, rows, st);
}

extern "C" int rgd_cache_write(const rgd_cache_shape* shape, int32_t layer, int32_t rows, int32_t max_new,
                               const rgd_bf16* k_new, const rgd_bf16* v_new, int64_t row_stride, int64_t token_stride,
                               const int32_t* n_new, int32_t max_pages, const int32_t* block_table,
                               const int32_t* length, const uint8_t* row_active, rgd_bf16* k_pages, rgd_bf16* v_pages,
                               int32_t* dev_status, rgd_stream_t stream) {
  clear_error();
  const char* fn = "rgd_cache_write";
  CacheView c;
  if (int rc = check_shape(fn, shape, c)) return rc;
  RGD_CHECK_ARG(rows >= 0 && max_new >= 0 && max_pages >= 1, "%s: bad rows/max_new/max_pages", fn);
  RGD_CHECK_ARG(layer >= 0 && layer < c.layers, "%s: layer outside [0, num_layers)", fn);
  RGD_CHECK_ARG(row_stride >= 0 && token_stride >= 0, "%s: strides must not be negative", fn);
  if (rows == 0 || max_new == 0) return RGD_OK;
  RGD_CHECK_ARG(k_new && v_new && n_new && block_table && length && k_pages && v_pages,
                "%s: k_new/v_new/n_new/block_table/length/k_pages/v_pages must be non-NULL", fn);
  RGD_CHECK_ARG(aligned16(k_new) && aligned16(v_new) && aligned16(k_pages) && aligned16(v_pages) &&
                    row_stride % 8 == 0 && token_stride % 8 == 0,
                "%s: tensors must be 16-byte aligned and strides multiples of 8 elements", fn);
  RGD_CHECK_ARG((int64_t)rows * max_new <= kMaxRows, "%s: too many tokens", fn);
  WriteParams p{};
  p.c = c;
  p.pool[0] = k_pages + layer * c.layer_stride;
  p.pool[1] = v_pages + layer * c.layer_stride;
  p.fresh[0] = k_new;
  p.fresh[1] = v_new;
  p.row_stride = row_stride;
  p.token_stride = token_stride;
  p.rows = rows;
  p.tokens = max_new;
  p.cols = max_pages;
  p.n_new = n_new;
  p.table = block_table;
  p.length = length;
  p.row_ok = row_active;
  p.dev_status = dev_status;
  const cudaError_t e =
      launch_dependent(write_kernel, blocks_for((int64_t)rows * max_new, kWarpsEach), kCopyThreads, 0, (cudaStream_t)stream, p);
  return e == cudaSuccess ? RGD_OK : cuda_error(e, "cache write launch");
}

extern "C" int rgd_cache_trim(int32_t rows, int32_t max_pages, int32_t num_pages, int32_t* block_table,
                              const int32_t* length, const uint8_t* row_active, int32_t* page_refs,
                              int32_t* dev_status, rgd_stream_t stream) {
  clear_error();
  const char* fn = "rgd_cache_trim";
  RGD_CHECK_ARG(rows >= 0 && max_pages >= 1 && num_pages >= 1, "%s: bad rows/max_pages/num_pages", fn);
  if (rows == 0) return RGD_OK;
  RGD_CHECK_ARG(rows <= kMaxRows, "%s: too many rows", fn);
  RGD_CHECK_ARG(block_table && length && page_refs, "%s: block_table/length/page_refs must be non-NULL", fn);
  const cudaError_t e = launch_dependent(trim_kernel, blocks_for(rows, kWarpsEach), kCopyThreads, 0, (cudaStream_t)stream, rows,
                                         max_pages, num_pages, block_table, length, row_active, page_refs, dev_status);
  return e == cudaSuccess ? RGD_OK : cuda_error(e, "cache trim launch");
}

extern "C" int rgd_cache_fork(int32_t pairs, const int32_t* parent, const int32_t* child, int32_t rows,
                              int32_t max_pages, int32_t num_pages, int32_t* block_table, int32_t* length,
                              int32_t* page_refs, int32_t* dev_status, rgd_stream_t stream) {
  clear_error();
  const char* fn = "rgd_cache_fork";
  RGD_CHECK_ARG(pairs >= 0 && rows >= 0 && max_pages >= 1 && num_pages >= 1, "%s: bad pairs/rows/max_pages/num_pages", fn);
  if (pairs == 0) return RGD_OK;
  RGD_CHECK_ARG(pairs <= kMaxRows, "%s: too many pairs", fn);
  RGD_CHECK_ARG(parent && child && block_table && length && page_refs,
                "%s: parent/child/block_table/length/page_refs must be non-NULL", fn);
  const cudaError_t e = launch_dependent(fork_kernel, blocks_for(pairs, kWarpsEach), kCopyThreads, 0, (cudaStream_t)stream, pairs,
                                         rows, max_pages, num_pages, parent, child, block_table, length, page_refs,
                                         dev_status);
  return e == cudaSuccess ? RGD_OK : cuda_error(e, "cache fork launch");
}

extern "C" int rgd_cache_copy(const rgd_cache_shape* shape, int32_t n, const int32_t* src, const int32_t* dst,
                              rgd_bf16* k_pages, rgd_bf16* v_pages, int32_t* dev_status, rgd_stream_t stream) {
  clear_error();
  const char* fn = "rgd_cache_copy";
  CacheView c;
  if (int rc = check_shape(fn, shape, c)) return rc;
  RGD_CHECK_ARG(n >= 0, "%s: n < 0", fn);
  if (n == 0) return RGD_OK;
  RGD_CHECK_ARG(src && dst && k_pages && v_pages, "%s: src/dst/k_pages/v_pages must be non-NULL", fn);
  RGD_CHECK_ARG(aligned16(k_pages) && aligned16(v_pages), "%s: k_pages/v_pages must be 16-byte aligned", fn);
  CopyParams q{};
  q.c = c;
  q.pool[0] = k_pages;
  q.pool[1] = v_pages;
  q.n = n;
  q.src = src;
  q.dst = dst;
  q.dev_status = dev_status;
  return launch_copies(q, n, (cudaStream_t)stream);
}

extern "C" int rgd_cache_compact(const rgd_cache_shape* shape, int32_t rows_a, int32_t max_pages_a,
                                 int32_t* block_table_a, int32_t rows_b, int32_t max_pages_b, int32_t* block_table_b,
                                 int32_t* page_refs, rgd_bf16* k_pages, rgd_bf16* v_pages, int32_t* num_live,
                                 void* workspace, size_t workspace_bytes, int32_t* dev_status, rgd_stream_t stream) {
  clear_error();
  const char* fn = "rgd_cache_compact";
  CacheView c;
  if (int rc = check_shape(fn, shape, c)) return rc;
  RGD_CHECK_ARG(rows_a >= 0 && rows_b >= 0 && max_pages_a >= 0 && max_pages_b >= 0, "%s: bad rows/max_pages", fn);
  RGD_CHECK_ARG(page_refs && k_pages && v_pages && num_live && workspace,
                "%s: page_refs/k_pages/v_pages/num_live/workspace must be non-NULL", fn);
  const int64_t na = block_table_a ? (int64_t)rows_a * max_pages_a : 0, nb = block_table_b ? (int64_t)rows_b * max_pages_b : 0;
  RGD_CHECK_ARG(aligned16(k_pages) && aligned16(v_pages) && aligned16(workspace),
                "%s: k_pages/v_pages/workspace must be 16-byte aligned", fn);
  RGD_CHECK_ARG(workspace_bytes >= rgd_cache_workspace_size(shape, 0), "%s: workspace too small", fn);
  cudaStream_t st = (cudaStream_t)stream;
  int32_t* ws = static_cast<int32_t*>(workspace);
  CopyParams q{};
  q.c = c;
  q.pool[0] = k_pages;
  q.pool[1] = v_pages;
  int32_t *src = ws + 64, *dst = src + c.pages, *place = dst + c.pages;
  const cudaError_t e =
      launch_plan(compact_kernel, plan_blocks(0, c.pages), st, c.pages, page_refs, num_live, ws, src, dst, place);
  if (e != cudaSuccess) return cuda_error(e, "cache compact launch");
  q.count = ws;
  q.src = src;
  q.dst = dst;
  q.dev_status = dev_status;
  q.live = num_live;
  q.place = place;
  q.table[0] = block_table_a;
  q.table[1] = block_table_b;
  q.entries[0] = na;
  q.entries[1] = nb;
  return launch_copies(q, c.pages, st);
}
