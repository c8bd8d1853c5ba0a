// The structure of a mask: bounds of its rows, of groups of rows and of columns, and a pattern's flags.  Bandwidth does not matter here (28 bytes a row);
// what a plan costs is its launches: two, or one where the mask is small (and then one more for a pattern).  us: 257 tokens 4.4; 4096 in eleven documents
// 4.8 + 4.5; 8192 4.9 + 6.8; 5003 queries over 11 147 keys with a pattern 5.0 + 6.3 (its flags in a launch of their own: 4.8 more).
#pragma once
#include "attn_common.hpp"

namespace spg {

struct MaskView {
  int q_len, k_len, docs, causal, window;
  const int64_t* q_ptr;     // docs + 1, or null: one document of everything
  const int64_t* k_ptr;
  const int64_t* prefix;    // docs, or null
  const int64_t* pat_ptr;   // of the pattern's rows of tiles, or null
  const int32_t* pat_col;
  int64_t pat_nnz;
};

__device__ __forceinline__ int clamp_to(int64_t v, int lo, int hi) { return v < lo ? lo : v > hi ? hi : (int)v; }

// Row i of the mask.  Bounds come out in ascending order over the rows (also of rows that see nothing: lo >= hi there), which k_plan_cols bisects.
__device__ inline RowBound row_bound(const MaskView& m, int i) {
  int qe = m.q_len, kb = 0, ke = m.k_len;
  int64_t prompt = 0;
  if (m.q_ptr) {
    if (i < m.q_ptr[0]) return {0, 0, 0, 0};
    int a = 0, b = m.docs;               // the last document that begins at or before i
    while (b - a > 1) {
      const int c = a + (b - a) / 2;
      if (m.q_ptr[c] <= i) a = c; else b = c;
    }
    qe = clamp_to(m.q_ptr[a + 1], 0, m.q_len);
    kb = clamp_to(m.k_ptr[a], 0, m.k_len);
    ke = clamp_to(m.k_ptr[a + 1], kb, m.k_len);
    if (i >= qe) return {m.k_len, m.k_len, 0, 0};   // behind the last document: behind every tile of keys too
    if (m.prefix) prompt = clamp_to(m.prefix[a], 0, m.k_len);
  } else if (m.prefix) {
    prompt = clamp_to(m.prefix[0], 0, m.k_len);
  }
  const int diag = i + ke - qe;
  int lo = kb, hi = ke;
  if (m.causal) {
    const int64_t p = kb + prompt;
    hi = clamp_to(p > diag + 1 ? p : diag + 1, kb, ke);
  }
  if (m.window) lo = clamp_to((int64_t)diag - m.window + 1, kb, ke);
  return {lo, hi, diag, 0};
}

// Row i of the mask by a thread, its group from the lanes of a half wave.
__device__ __forceinline__ void plan_row(const MaskView& m, const PlanView& p, int i) {
  RowBound r{0, 0, 0, 0};
  if (i < m.q_len) {
    r = row_bound(m, i);
    p.rows[i] = r;
  }
  GroupBound g{r.lo < r.hi ? r.lo : 0x7fffffff, r.lo < r.hi ? r.hi : 0, i < m.q_len ? r.lo : 0, i < m.q_len ? r.hi : 0x7fffffff};
#pragma unroll
  for (int d = kRowGroup / 2; d; d >>= 1) {
    g.lo = min(g.lo, __shfl_xor(g.lo, d)); g.hi = max(g.hi, __shfl_xor(g.hi, d));
    g.all_lo = max(g.all_lo, __shfl_xor(g.all_lo, d)); g.all_hi = min(g.all_hi, __shfl_xor(g.all_hi, d));
  }
  if (i % kRowGroup == 0 && i < m.q_len) p.groups[i / kRowGroup] = {g.hi ? g.lo : 0, g.hi, g.all_lo, g.all_hi};
}

// The flags of a pattern, before k_plan_pattern sets them.
__device__ __forceinline__ void clear_flags(const MaskView& m, const PlanView& p, int first, int64_t step) {
  const int64_t words = (int64_t)ceil_div_d(m.q_len, kPatTile) * p.seen_words, by_words = (int64_t)ceil_div_d(m.k_len, kPatTile) * p.seen_by_words;
  for (int64_t w = first; w < words; w += step) p.seen[w] = 0;
  for (int64_t w = first; w < by_words; w += step) p.seen_by[w] = 0;
}

// By one workgroup.
__device__ __forceinline__ void check_documents(const MaskView& m, const PlanView& p) {
  __shared__ int bad;
  if (threadIdx.x == 0) bad = 0;
  __syncthreads();
  if (m.q_ptr) {
    for (int d = threadIdx.x; d < m.docs; d += blockDim.x) {
      const int64_t a = m.q_ptr[d], b = m.q_ptr[d + 1], c = m.k_ptr[d], e = m.k_ptr[d + 1];
      if (a < 0 || b < a || b > m.q_len || c < 0 || e < c || e > m.k_len) bad = 1;
      if (m.prefix && m.prefix[d] < 0) bad = 1;
    }
  } else if (m.prefix && threadIdx.x == 0 && m.prefix[0] < 0) {
    bad = 1;
  }
  __syncthreads();
  if (threadIdx.x == 0) *p.error = bad;
}

__global__ void __launch_bounds__(256) k_plan_rows(MaskView m, PlanView p) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  clear_flags(m, p, i, (int64_t)gridDim.x * 256);
  plan_row(m, p, i);
  if (blockIdx.x == 0) {
    check_documents(m, p);
    if (threadIdx.x == 0) p.totals[0] = p.totals[1] = 0;
  }
}

// The keys that the rows of tile i see: from .x to before .y; nothing is 0, 0.
__device__ __forceinline__ int2 query_tile_reach(const PlanView& p, int q_len, int i) {
  int lo = 0x7fffffff, hi = 0;
  for (int g = i * (kPatTile / kRowGroup); g < (i + 1) * (kPatTile / kRowGroup) && g < ceil_div_d(q_len, kRowGroup); ++g) {
    const GroupBound b = p.groups[g];
    if (b.hi > b.lo) { lo = min(lo, b.lo); hi = max(hi, b.hi); }
  }
  return hi > lo ? make_int2(lo, hi) : make_int2(0, 0);
}

// The queries that can see any key of tile c, by a wave: from the first row that ends behind its first key to before the first that begins behind its last.
__device__ __forceinline__ int2 key_tile_reach(const PlanView& p, int q_len, int k_len, int c) {
  const int first = c * kKeyTile, last = k_len - first > kKeyTile ? first + kKeyTile : k_len;
  const int from = wave_count_below(q_len, (int64_t)first + 1, [&](int i) { return p.rows[i].hi; });
  const int to = wave_count_below(q_len, last, [&](int i) { return p.rows[i].lo; });
  return to > from ? make_int2(from, to) : make_int2(0, 0);
}
__device__ __forceinline__ unsigned query_tiles(int2 r) { return ceil_div_d(r.y, kQueryTile) - r.x / kQueryTile; }
__device__ __forceinline__ unsigned key_tiles(int2 r) { return ceil_div_d(r.y, kKeyTile) - r.x / kKeyTile; }

// Tiles 0 .. n - 1 by falling work, by one workgroup of 256 threads: order[place] = tile and what reach(tile) says.  Up to 256 of them count how many come before
// each; more are sorted as far as 256 steps of the largest tell them apart.  (Which of two alike comes first may then differ from call to call; it
// decides only when their workgroups run.)
constexpr int kOrderKept = 2048;                 // works that LDS holds between the passes; with more tiles they are made again
template <typename F>
__device__ __forceinline__ void order_by_work(int n, F reach, int4* order) {
  __shared__ unsigned most, count[256];
  __shared__ int kept[kOrderKept];
  if (n <= 256) {
    const int i = threadIdx.x;
    const int2 r = i < n ? reach(i) : make_int2(0, 0);
    const int mine = r.y - r.x;
    kept[i] = i < n ? mine : -1;
    __syncthreads();
    int place = 0;
#pragma unroll 16
    for (int k = 0; k < ceil_div_d(n, 16) * 16; ++k) place += (kept[k] > mine) | ((kept[k] == mine) & (k < i));
    if (i < n) order[place] = make_int4(i, r.x, r.y, 1);
    return;
  }
  auto work = [&](int i) { const int2 r = reach(i); return r.y - r.x; };
  if (threadIdx.x == 0) most = 1;
  count[threadIdx.x] = 0;
  __syncthreads();
  int top = 0;
  for (int i = threadIdx.x; i < n; i += 256) {
    const int w = work(i);
    if (n <= kOrderKept) kept[i] = w;
    top = w > top ? w : top;
  }
  atomicMax(&most, (unsigned)top);
  __syncthreads();
  auto bucket = [&](int i) { return 255 - (int)((uint64_t)(n <= kOrderKept ? kept[i] : work(i)) * 255 / most); };
  for (int i = threadIdx.x; i < n; i += 256) atomicAdd(&count[bucket(i)], 1u);
  __syncthreads();
  if (threadIdx.x < kWave) {                     // exclusive sums, four numbers a lane
    int v[4], sum = 0;
    for (int j = 0; j < 4; ++j) { v[j] = count[threadIdx.x * 4 + j]; sum += v[j]; }
    int before = wave_incl_scan(sum) - sum;
    for (int j = 0; j < 4; ++j) { count[threadIdx.x * 4 + j] = before; before += v[j]; }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += 256) {
    const int2 r = reach(i);
    order[atomicAdd(&count[bucket(i)], 1u)] = make_int4(i, r.x, r.y, 1);
  }
}

// The pattern's flags, a wave a row of tiles r.  Bits are only set, so neither the order of a row's columns nor repeated ones matter.
__device__ __forceinline__ void set_flags(const MaskView& m, const PlanView& p, int r) {
  const int rows = ceil_div_d(m.q_len, kPatTile), cols = ceil_div_d(m.k_len, kPatTile);
  if (r >= rows) return;
  const int64_t a = m.pat_ptr[r], b = m.pat_ptr[r + 1];
  if (a < 0 || b < a || b > m.pat_nnz) {
    if (lane_id() == 0) *p.error = 1;
    return;
  }
  for (int64_t e = a + lane_id(); e < b; e += kWave) {
    const int c = m.pat_col[e];
    if (c < 0 || c >= cols) { *p.error = 1; continue; }
    atomicOr(&p.seen[(int64_t)r * p.seen_words + c / 32], 1u << (c % 32));
    atomicOr(&p.seen_by[(int64_t)c * p.seen_by_words + r / 32], 1u << (r % 32));
  }
}
__global__ void __launch_bounds__(256) k_plan_pattern(MaskView m, PlanView p) { set_flags(m, p, blockIdx.x * 4 + threadIdx.x / kWave); }

// What both kinds of tiles reach, a wave a tile of keys; those of queries by a workgroup of its own, which also brings them into order of work: the card
// holds a few workgroups a compute unit, and long rows that begin late are waited for (two documents of 4000 tokens, tiles from the last row
// backwards: 1.3 waves a SIMD on average where two fit).  Few tiles all run at once and need no order.  (Tiles of keys are ordered beside
// k_attn_facts: here that would have to wait for all waves, and a forward pass does not need it; 4096 tokens 8.0 -> 6.7 us, by counting 5.2.)
// Workgroups behind those of the keys set a pattern's flags.
constexpr int kOrderQueries = 17;
__global__ void __launch_bounds__(256) k_plan_cols(MaskView m, PlanView p) {
  const int q_len = m.q_len, k_len = m.k_len;
  const int q_tiles = ceil_div_d(q_len, kPatTile), k_tiles = ceil_div_d(k_len, kKeyTile);
  if (blockIdx.x == gridDim.x - 1) {
    auto reach = [&](int i) { return query_tile_reach(p, q_len, i); };
    unsigned long long sum = 0;
    for (int i = threadIdx.x; i < q_tiles; i += 256) {
      const int2 r = reach(i);
      sum += key_tiles(r);
      if (q_tiles < kOrderQueries) p.q_order[q_tiles - 1 - i] = make_int4(i, r.x, r.y, 1);
    }
    if (sum) atomicAdd(&p.totals[0], sum);
    if (q_tiles >= kOrderQueries) order_by_work(q_tiles, reach, p.q_order);
    return;
  }
  const int c = blockIdx.x * 4 + threadIdx.x / kWave, behind = c - ceil_div_d(k_tiles, 4) * 4;
  if (behind >= 0) set_flags(m, p, behind);
  if (c >= k_tiles) return;
  const int2 r = key_tile_reach(p, q_len, k_len, c);
  if (lane_id() == 0) {
    p.cols[c] = r;
    atomicAdd(&p.totals[1], (unsigned long long)query_tiles(r));
  }
}

// The same for a small mask, whose tiles need no order, by one workgroup: a thread a row, a wave a tile of keys.  us in one launch | in two: 257 tokens 4.6 | 5.0,
// and 4 less on the host; 2003 tokens by the same kernel 8.5 | 7.5.
constexpr int kSmallMask = 1024;
static_assert(kSmallMask / kPatTile < kOrderQueries && kSmallMask / kKeyTile <= kSmallMask / kWave, "no order, a wave a tile");
__global__ void __launch_bounds__(kSmallMask) k_plan_small(MaskView m, PlanView p) {
  __shared__ unsigned totals[2];
  if (threadIdx.x < 2) totals[threadIdx.x] = 0;
  clear_flags(m, p, threadIdx.x, kSmallMask);
  plan_row(m, p, threadIdx.x);
  check_documents(m, p);
  __syncthreads();
  const int q_tiles = ceil_div_d(m.q_len, kPatTile), k_tiles = ceil_div_d(m.k_len, kKeyTile);
  const int i = threadIdx.x, c = threadIdx.x / kWave;
  if (i < q_tiles) {
    const int2 r = query_tile_reach(p, m.q_len, i);
    atomicAdd(&totals[0], key_tiles(r));
    p.q_order[q_tiles - 1 - i] = make_int4(i, r.x, r.y, 1);
  }
  if (c < k_tiles) {
    const int2 r = key_tile_reach(p, m.q_len, m.k_len, c);
    if (lane_id() == 0) {
      atomicAdd(&totals[1], query_tiles(r));
      p.cols[c] = r;
    }
  }
  __syncthreads();
  if (threadIdx.x < 2) p.totals[threadIdx.x] = totals[threadIdx.x];
}

}  // namespace spg
