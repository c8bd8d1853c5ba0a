// Page tables of a cache: the next table from the last one, pages to the front, and the copies that both ask for.
//
// A table is a compressed structure (rows: sequences, columns: pages).  Everything here but the copies is a few bytes a row or page: what it
// costs is launches and dependent loads, so that ranks (the k-th free page) are found by counting bits in a flag list, as the
// product's kernels rank columns.  No result depends on the order of atomics: they count, take minima, or set bits.
// us, without copies: a fork of 8 rows 2.6 + 2.8 + 2.8 + 4.1 (by one workgroup 17), 512 rows from 384 3.2 + 8.4 + 3.3 + 7.0 (gather: atomics on pages that many rows share);
// compacting 2048 pages 1.7 + 4.5 + 2.0 + 3.9.
#pragma once
#include "cache_kernels.hpp"

namespace spg {

constexpr int kPageBlock = 1024;     // pages whose flags are counted together: 32 words

struct PageMoves {        // what the kernels leave for the copies and for the host
  int error;
  unsigned moves;
  long long nnz;          // entries of the new table
  long long live;         // pages in use
};

struct PageFlags {        // a bit a page: in use; and how many are in use in every block of pages
  unsigned* words;
  unsigned* counts;
  int64_t pages;
};

struct ForkArgs {
  TableView t;            // the last table, its lengths
  int64_t pages;
  const int32_t* parent;
  const int32_t* new_lens;
  int rows;               // of the new table
  int64_t* ptr;           // rows + 1
  int32_t* page;
  int64_t room;           // entries that `page` can hold
  int32_t* refs;          // pages
  int32_t* owner;         // pages: the first row that ends inside the page, -1 where a row has it whole
  int64_t* fresh;         // rows: new pages of the rows before
  PageFlags used;
  int32_t *src, *dst;     // rows: the copies
  PageMoves* out;
};

// What row r keeps of its parent: tokens, their pages, where those are in the last table; and how many pages it needs.  error: kForkInput, or
// kForkPages for a row longer than the cache.
constexpr int kForkInput = 1, kForkPages = 2;
struct Kept { int64_t tokens, at; int pages, need, error; };
__device__ __forceinline__ Kept kept_of(const ForkArgs& a, int r) {
  const int p = a.parent[r];
  const int64_t len = a.new_lens[r];
  Kept k{0, 0, 0, 0, p >= -1 && p < a.t.seqs && len >= 0 ? 0 : kForkInput};
  if (k.error) return k;
  k.need = page_need(len, a.pages);
  if (k.need < 0) { k.need = 0; k.error = kForkPages; return k; }
  if (p >= 0) {
    const int64_t had = a.t.lens[p], b = a.t.ptr[p], e = a.t.ptr[p + 1];
    k.tokens = had < len ? had : len;
    k.at = b;
    k.pages = k.tokens > 0 ? (int)((k.tokens + kPage - 1) / kPage) : 0;
    if (had < 0 || b < 0 || e < b || e > a.t.nnz || k.pages > e - b) { k.error = kForkInput; k.pages = 0; k.tokens = 0; }
  }
  return k;
}

// Exclusive sums of value(0) .. value(n - 1) by one workgroup of 1024 threads; store(i, sum before i); the total is returned to all.
template <typename V, typename S>
__device__ __forceinline__ int64_t block_scan(int64_t n, V value, S store) {
  __shared__ int64_t waves[16];
  int64_t before = 0;
  for (int64_t i0 = 0; i0 < n; i0 += 1024) {
    const int64_t i = i0 + threadIdx.x;
    const int v = i < n ? value(i) : 0;
    const int sum = wave_incl_scan(v);
    if (lane_id() == kWave - 1) waves[threadIdx.x / kWave] = sum;
    __syncthreads();
    int64_t mine = before, all = before;
    for (int w = 0; w < 16; ++w) {
      if (w < (int)threadIdx.x / kWave) mine += waves[w];
      all += waves[w];
    }
    if (i < n) store(i, mine + sum - v);
    before = all;
    __syncthreads();
  }
  return before;
}

// The new table's row pointer, by one workgroup of 1024 threads.
__device__ __forceinline__ void fork_rows(const ForkArgs& a) {
  __shared__ int bad;
  if (threadIdx.x == 0) bad = 0;
  __syncthreads();
  const int64_t nnz = block_scan(
      a.rows,
      [&](int64_t r) {
        const Kept k = kept_of(a, (int)r);
        if (k.error) atomicOr(&bad, k.error);
        return k.need;
      },
      [&](int64_t r, int64_t sum) { a.ptr[r] = sum; });
  __syncthreads();
  if (threadIdx.x == 0) {
    a.ptr[a.rows] = nnz;
    *a.out = PageMoves{bad & kForkInput || nnz > a.room ? kForkInput : bad, 0u, nnz, 0};
  }
}

__device__ __forceinline__ void fork_clear(const ForkArgs& a, int64_t first, int64_t step) {
  for (int64_t p = first; p < a.pages; p += step) {
    a.refs[p] = 0;
    a.owner[p] = 0x7fffffff;
  }
}

// Pages that a row takes over, by a wave.
__device__ __forceinline__ void fork_gather(const ForkArgs& a, int r) {
  const Kept k = kept_of(a, r);
  const int64_t to = a.ptr[r];
  for (int j = lane_id(); j < k.pages; j += kWave) {
    const int p = a.t.page[k.at + j];
    if (p < 0 || p >= a.pages) { a.out->error = kForkInput; continue; }
    a.page[to + j] = p;
    atomicAdd(&a.refs[p], 1);
    atomicMin(&a.owner[p], (int64_t)(j + 1) * kPage > k.tokens ? r : -1);
  }
}

// Whether row r has to copy the last page that it keeps: it ends inside the page, and another row has the page whole or comes first.
__device__ __forceinline__ bool copies_last(const ForkArgs& a, int r, const Kept& k) {
  if (k.tokens % kPage == 0 || k.pages == 0) return false;
  const int p = a.t.page[k.at + k.pages - 1];
  return p >= 0 && p < a.pages && a.owner[p] != r;
}

// How many new pages the rows before each row take, by one workgroup of 1024 threads.
__device__ __forceinline__ void fork_fresh(const ForkArgs& a) {
  block_scan(
      a.rows,
      [&](int64_t r) {
        const Kept k = kept_of(a, (int)r);
        return k.need - k.pages + (copies_last(a, (int)r, k) ? 1 : 0);
      },
      [&](int64_t r, int64_t sum) { a.fresh[r] = sum; });
}

// Flags and count of a block of pages in use, by 1024 threads.
__device__ __forceinline__ void fork_flags(const ForkArgs& a, int64_t block) {
  __shared__ unsigned counts[16];
  const int64_t p = block * kPageBlock + threadIdx.x;
  const unsigned long long b = __ballot(p < a.pages && a.refs[p] > 0);
  if (lane_id() == 0) {
    const int64_t w = p / 32;
    a.used.words[w] = (unsigned)b;
    a.used.words[w + 1] = (unsigned)(b >> 32);
    counts[threadIdx.x / kWave] = __popcll(b);
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    unsigned n = 0;
    for (int i = 0; i < 16; ++i) n += counts[i];
    a.used.counts[block] = n;
  }
  __syncthreads();
}

// The k-th page (from 0) that is not in use, or -1.  (Blocks are walked one after the other, then words: a cache of 60 000 pages that is nearly full takes up to 60
// dependent loads and 32 more.)
__device__ __forceinline__ int64_t free_page(const PageFlags& f, int64_t k) {
  const int64_t blocks = (f.pages + kPageBlock - 1) / kPageBlock;
  for (int64_t b = 0; b < blocks; ++b) {
    const int64_t in = f.pages - b * kPageBlock < kPageBlock ? f.pages - b * kPageBlock : kPageBlock;
    const int64_t n = in - f.counts[b];
    if (k >= n) { k -= n; continue; }
    for (int w = 0; w < kPageBlock / 32; ++w) {
      unsigned z = ~f.words[b * (kPageBlock / 32) + w];
      const int c = __popc(z);
      if (k >= c) { k -= c; continue; }
      for (; k > 0; --k) z &= z - 1;
      return b * kPageBlock + w * 32 + __ffs(z) - 1;
    }
  }
  return -1;
}

// New pages of a row, by a wave: the k-th new one, rows in order, is the k-th page that no row of the new table kept.
__device__ __forceinline__ void fork_assign(const ForkArgs& a, int r) {
  const Kept k = kept_of(a, r);
  const int copy = copies_last(a, r, k) ? 1 : 0;
  const int64_t to = a.ptr[r], rank = a.fresh[r];
  for (int j = lane_id(); j < k.need - k.pages + copy; j += kWave) {
    const int64_t p = free_page(a.used, rank + j);
    if (p < 0) { a.out->error = kForkPages; continue; }
    const int at = k.pages - copy + j;
    if (copy && j == 0) {
      const int old = a.t.page[k.at + at];
      atomicSub(&a.refs[old], 1);
      const unsigned i = atomicAdd(&a.out->moves, 1u);
      a.src[i] = old;
      a.dst[i] = (int)p;
    }
    a.page[to + at] = (int)p;
    a.refs[p] = 1;
  }
}

// The steps as kernels.  (An error is set by a step before, or in assigning, where every row that finds no page sets it.)
__global__ void __launch_bounds__(1024) k_fork_rows(ForkArgs a) {
  if (blockIdx.x == 0) fork_rows(a);
  else fork_clear(a, (int64_t)(blockIdx.x - 1) * 1024 + threadIdx.x, (int64_t)(gridDim.x - 1) * 1024);
}
__global__ void __launch_bounds__(256) k_fork_gather(ForkArgs a) {
  const int r = blockIdx.x * 4 + threadIdx.x / kWave;
  if (r < a.rows && !a.out->error) fork_gather(a, r);
}
__global__ void __launch_bounds__(1024) k_fork_flags(ForkArgs a) {
  if (a.out->error) return;
  if (blockIdx.x == gridDim.x - 1) fork_fresh(a);
  else fork_flags(a, blockIdx.x);
}
__global__ void __launch_bounds__(256) k_fork_assign(ForkArgs a) {
  const int r = blockIdx.x * 4 + threadIdx.x / kWave;
  if (r < a.rows && !a.out->error) fork_assign(a, r);
}

// ---- pages to the front -------------------------------------------------------------------------

struct CompactArgs {
  TableView t;
  PageFlags live;
  int32_t *movers, *holes;  // pages in use at or behind their number, and the places before it that are free: the i-th goes to the i-th
  int32_t* rank;          // pages: of a mover, its place among them
  int32_t* page;          // the new table's entries
  PageMoves* out;
};

__global__ void __launch_bounds__(256) k_compact_clear(CompactArgs a) {
  const int64_t words = (a.live.pages + kPageBlock - 1) / kPageBlock * (kPageBlock / 32);
  for (int64_t w = (int64_t)blockIdx.x * 256 + threadIdx.x; w < words; w += (int64_t)gridDim.x * 256) a.live.words[w] = 0;
  if (blockIdx.x == 0 && threadIdx.x == 0) *a.out = PageMoves{0, 0u, a.t.nnz, 0};
}

__global__ void __launch_bounds__(256) k_compact_mark(CompactArgs a) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < a.t.nnz; i += (int64_t)gridDim.x * 256) {
    const int p = a.t.page[i];
    if (p < 0 || p >= a.live.pages) { a.out->error = 1; continue; }
    atomicOr(&a.live.words[p / 32], 1u << (p % 32));
  }
}

__global__ void __launch_bounds__(256) k_compact_count(CompactArgs a) {
  const int64_t b = (int64_t)blockIdx.x * 4 + threadIdx.x / kWave;
  if (b >= (a.live.pages + kPageBlock - 1) / kPageBlock) return;
  int n = lane_id() < kPageBlock / 32 ? __popc(a.live.words[b * (kPageBlock / 32) + lane_id()]) : 0;
  for (int d = 1; d < kPageBlock / 32; d *= 2) n += __shfl_xor(n, d);
  if (lane_id() == 0) {
    a.live.counts[b] = n;
    atomicAdd(reinterpret_cast<unsigned long long*>(&a.out->live), (unsigned long long)n);
  }
}

// Movers and holes in order, a workgroup a block of pages.  Page p has `before` pages in use before it, a hole so p - before holes; of the movers, those
// before it are the ones in use before p but not before `live`.
__global__ void __launch_bounds__(kPageBlock) k_compact_map(CompactArgs a) {
  if (a.out->error) return;                        // (set by earlier kernels only)
  __shared__ unsigned sums[2][16], ballots[16];
  const int64_t live = a.out->live, first = (int64_t)blockIdx.x * kPageBlock, p = first + threadIdx.x;
  const int wave = threadIdx.x / kWave;
  // pages in use in all blocks before this one, and in all before `live`
  unsigned here = 0, front = 0;
  for (int64_t b = threadIdx.x; b < (int64_t)blockIdx.x || b < live / kPageBlock; b += kPageBlock) {
    const unsigned n = a.live.counts[b];
    here += b < (int64_t)blockIdx.x ? n : 0;
    front += b < live / kPageBlock ? n : 0;
  }
  if (threadIdx.x < kPageBlock / 32) {             // the block that `live` cuts
    const int64_t w = live / kPageBlock * (kPageBlock / 32) + threadIdx.x;
    if (w * 32 < live) front += __popc(a.live.words[w] & (live - w * 32 < 32 ? (1u << (live - w * 32)) - 1 : ~0u));
  }
  for (int d = 1; d < kWave; d *= 2) { here += __shfl_xor(here, d); front += __shfl_xor(front, d); }
  const bool used = p < a.live.pages && (a.live.words[p / 32] >> (p % 32) & 1);
  const unsigned long long mask = __ballot(used);
  if (lane_id() == 0) { sums[0][wave] = here; sums[1][wave] = front; ballots[wave] = __popcll(mask); }
  __syncthreads();
  int64_t before = __popcll(mask & ((1ULL << lane_id()) - 1)), in_front = 0;
  for (int w = 0; w < 16; ++w) {
    before += sums[0][w] + (w < wave ? ballots[w] : 0);
    in_front += sums[1][w];
  }
  if (used && p >= live) {
    a.movers[before - in_front] = (int)p;
    a.rank[p] = (int)(before - in_front);
  }
  if (!used && p < live) a.holes[p - before] = (int)p;
  if (blockIdx.x == 0 && threadIdx.x == 0) a.out->moves = (unsigned)(live - in_front);
}

// ---- copies --------------------------------------------------------------------------------------

struct CopyArgs {
  unsigned char *k, *v;
  float *k_scale, *v_scale;
  int64_t pages;
  int layers, heads;
  int64_t page_bytes;     // of keys (or values) in one layer
  const int32_t *src, *dst;
  int64_t count;          // of them, or
  const PageMoves* in;    // ... what kernels before have found
  PageMoves* report;      // pinned host memory that gets `in`, or null
  // the table after k_compact_map's moves, or null
  const int32_t *old_page, *rank;
  int32_t* new_page;
  int64_t nnz;
};

constexpr int kCopyPiece = 16384;    // bytes that a workgroup copies at a time: four loads of 16 bytes in flight a lane

// Destinations are distinct and no source, so the copies need no order.  Memory bounds it: 237 MB read and written 40 us, 5.9 TB/s; 530 MB 117 us, 4.5.
__global__ void __launch_bounds__(256) k_page_copy(CopyArgs a) {
  if (a.report && blockIdx.x == 0 && threadIdx.x == 0) *a.report = *a.in;
  if (a.in && a.in->error) return;
  const int64_t moves = a.in ? a.in->moves : a.count;
  const int64_t pieces = (a.page_bytes + kCopyPiece - 1) / kCopyPiece, per = 2 * pieces;
  for (int64_t u = blockIdx.x; u < moves * a.layers * per; u += gridDim.x) {
    const int64_t move = u / (a.layers * per), layer = u / per % a.layers;
    const int piece = (int)(u % per);
    const int64_t from = a.src[move], to = a.dst[move];
    if (from < 0 || to < 0 || from >= a.pages || to >= a.pages) continue;
    unsigned char* base = piece < pieces ? a.k : a.v;
    const int64_t off = (int64_t)(piece % (int)pieces) * kCopyPiece;
    const int64_t bytes = a.page_bytes - off < kCopyPiece ? a.page_bytes - off : kCopyPiece;
    const u32x4* s = reinterpret_cast<const u32x4*>(base + (layer * a.pages + from) * a.page_bytes + off);
    u32x4* d = reinterpret_cast<u32x4*>(base + (layer * a.pages + to) * a.page_bytes + off);
    u32x4 w[kCopyPiece / 4096];
#pragma unroll
    for (int i = 0; i < kCopyPiece / 4096; ++i)
      if (i * 4096 + (int)threadIdx.x * 16 < bytes) w[i] = s[i * 256 + threadIdx.x];
#pragma unroll
    for (int i = 0; i < kCopyPiece / 4096; ++i)
      if (i * 4096 + (int)threadIdx.x * 16 < bytes) d[i * 256 + threadIdx.x] = w[i];
    if (piece % (int)pieces == 0) {
      float* scale = piece < pieces ? a.k_scale : a.v_scale;
      for (int h = threadIdx.x; h < a.heads; h += 256)
        scale[(layer * a.pages + to) * a.heads + h] = scale[(layer * a.pages + from) * a.heads + h];
    }
  }
  if (a.new_page) {
    const int64_t live = a.in->live;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < a.nnz; i += (int64_t)gridDim.x * 256) {
      const int p = a.old_page[i];
      a.new_page[i] = p < live ? p : a.dst[a.rank[p]];
    }
  }
}

}  // namespace spg
