// Trees of drafted tokens: their structure, and the attention of their nodes over the paged cache.
//
// out = sum_j 2^(x_j - m) v_j / sum_j 2^(x_j - m) over the keys that a node sees, in one pass with the running maximum m, the sums in 32 bits.  A row is a node and a head that shares the key head; a wave has 32 of
// them as right operands and takes a page of 64 tokens in two products of 32 keys (32 x 32 x 16 form, attn_common.hpp).  The order of a page's keys in the first product is chosen so that a lane's probabilities
// are neighbouring keys, which is what the second product's left operand (a value's channel, held along the tokens) reads in one piece: nothing moves between lanes.
//
// All rows of a tree read the same pages, so what matters is how many rows share a read of them.  With more than 64 rows a page is widened to 16 bits once, into LDS, for four waves of 32 rows; with fewer the waves
// take pages in turn, from memory to registers.  Measured (bfloat16 unless said; calls one after another, structure and join included; then the kernel and the join alone, means of a few launches under the profiler): four
// sequences of 50 000 to 65 011 tokens, up to 60 nodes, 32 heads on 8 of 128 channels 244 us, 0.63 PFLOP/s; 271 (least 255) and 9.  Vector instructions issue in 48 % of the cycles and matrix instructions run in 35 %, what two waves
// a SIMD reach together; a quarter of the cycles of LDS go to bank conflicts, those of the widened pages' stores.  48 sequences of 20 to 4000 tokens, up to 26 nodes, capped, two layers 113 us; 46 and 10 a layer: a workgroup's
// chain (its piece 2 us, the first page 2, each page 2.3, the end 2.7) about twice over.  24 sequences, 17 nodes, 8 heads of 80 channels, window 900, distances, float16, three layers 63 us; 16 and 4 a layer.  One of 712
// tokens, 12 nodes, 24 us; 9.7 and 4.
#pragma once
#include "cache_kernels.hpp"
#include "draft_pieces.hpp"

namespace spg {

constexpr int kMostNodes = 256, kNodeWords = kMostNodes / 64;

struct TreeNode { int parent, eldest, depth; };      // parent: -1 without one; eldest: the parent's first child
struct TreeView {
  const int64_t* ptr;             // rows + 1
  int rows, most, words;          // words: of 64 bits, that a node's ancestors take
  int64_t tokens;
  unsigned long long* up;         // [tokens][words]: the node's ancestors and itself
  TreeNode* node;                 // [tokens]
  int4* place;                    // [tokens]: the first of the node's tree, how many it has (0: a node of none), its sequence
};

struct Tree { int64_t first; int n; };
__device__ __forceinline__ int64_t tree_begin(const TreeView& t, int s) {
  const int64_t v = t.ptr[s];
  return v < 0 ? 0 : v > t.tokens ? t.tokens : v;
}
__device__ __forceinline__ Tree tree_of(const TreeView& t, int s) {
  const int64_t b = tree_begin(t, s), n = tree_begin(t, s + 1) - b;
  return {b, n < 0 ? 0 : n < t.most ? (int)n : t.most};
}

// ---- structure --------------------------------------------------------------------------------

// A workgroup has a tree.  A node's ancestors are found by doubling: it takes over what the node that it points to has, and then points to where that one points; a tree of depth d is done
// after log d rounds.  12 nodes 3.3 us, 48 trees of up to 26 nodes 5 us: a chain of loads and LDS steps.
__global__ void __launch_bounds__(kMostNodes) k_trees(TreeView t, const int32_t* parent) {
  __shared__ int jump[kMostNodes], child[kMostNodes];
  __shared__ unsigned long long ups[kNodeWords][kMostNodes];
  const Tree tree = tree_of(t, blockIdx.x);
  const int i = threadIdx.x;
  int p = -1;
  if (i < tree.n) {
    p = parent[tree.first + i];
    p = p >= 0 && p < i ? p : -1;
  }
  unsigned long long up[kNodeWords];
#pragma unroll
  for (int w = 0; w < kNodeWords; ++w) ups[w][i] = up[w] = i / 64 == w ? 1ull << (i % 64) : 0ull;
  int to = p;
  jump[i] = p;
  child[i] = kMostNodes;
  __syncthreads();
  if (p >= 0) atomicMin(&child[p], i);      // (a minimum is the same in any order)
  while (__syncthreads_or(to >= 0)) {
    int next = -1;
    if (to >= 0) {
#pragma unroll
      for (int w = 0; w < kNodeWords; ++w)
        if (w < t.words) up[w] |= ups[w][to];
      next = jump[to];
    }
    __syncthreads();
    to = next;
    jump[i] = to;
#pragma unroll
    for (int w = 0; w < kNodeWords; ++w) ups[w][i] = up[w];
  }
  // nodes that no tree has: those behind a tree's `most` first, and what ptr leaves out in front and behind
  const int64_t begin = blockIdx.x == 0 ? 0 : tree.first, end = (int)blockIdx.x == t.rows - 1 ? t.tokens : tree_begin(t, blockIdx.x + 1);
  for (int64_t x = begin + i; x < end; x += kMostNodes)
    if (x < tree.first || x >= tree.first + tree.n) t.place[x] = make_int4(0, 0, 0, 0);
  if (i >= tree.n) return;
  int depth = -1;
#pragma unroll
  for (int w = 0; w < kNodeWords; ++w) {
    depth += __popcll(up[w]);
    if (w < t.words) t.up[(tree.first + i) * t.words + w] = up[w];
  }
  t.node[tree.first + i] = TreeNode{p, p >= 0 ? child[p] : i, depth};
  t.place[tree.first + i] = make_int4((int)tree.first, tree.n, (int)blockIdx.x, 0);
}

// Is anything wrong with the trees?  One workgroup looks at all of them.
__global__ void __launch_bounds__(1024) k_trees_check(TreeView t, const int32_t* parent, int* error) {
  int bad = 0;
  for (int s = threadIdx.x; s < t.rows; s += 1024) {
    const int64_t b = t.ptr[s], e = t.ptr[s + 1];
    bad |= b < 0 || e < b || e > t.tokens || e - b > t.most || (s == 0 && b != 0) || (s == t.rows - 1 && e != t.tokens);
    if (bad) break;
    for (int64_t i = b; i < e; ++i) bad |= parent[i] < -1 || parent[i] >= i - b;
  }
  bad |= t.rows == 0 && t.tokens != 0;
  bad = __syncthreads_or(bad);
  if (threadIdx.x == 0) *error = bad;
}

// ---- attention --------------------------------------------------------------------------------

constexpr int kTreeRows = 128;    // rows of a workgroup, at most: 32 a wave
constexpr int tree_resident(int room) { return room == 64 ? 3 : 2; }      // workgroups of a compute unit (registers)

struct TreeAttendArgs {
  CacheView c;
  TableView t;
  TreeView trees;
  HeadTensor q, o;          // row ptr[s] + i: node i of sequence s
  int heads, group, window;
  int tiles;                // of 128 rows, that a tree can have
  int places;               // workgroups that the card holds at once
  int chunk;                // pages of a workgroup where sequences are many; 0: Schedule says
  int part_rows;            // rows that a cell has places for
  int64_t cells;            // (row pointers that do not ascend could ask for more: such pieces are left out)
  ScoreShape score;
  float* part;              // [cells][part_rows][R]: sums of what the workgroups saw, not divided
  float2* part_ml;          // [cells][part_rows]: maximum (units of log 2) and sum
  int4* cuts;               // of every sequence with something to do: Cut
};

// Sequence s: its tree, its tokens and the pages first .. last - 1 that its nodes see.
struct TreePages { Tree tree; int64_t at; int len, ctx, lo, first, last; };
__device__ __forceinline__ int64_t first_page(const TableView& t, int s) {
  const int64_t b = t.ptr[s];
  return b < 0 ? 0 : b > t.nnz ? t.nnz : b;
}
__device__ __forceinline__ TreePages tree_pages(const TreeAttendArgs& a, int s) {
  const int64_t b = first_page(a.t, s);
  int64_t e = first_page(a.t, s + 1);
  e = e < b ? b : e;
  const int64_t most = (e - b) * kPage;
  const int64_t len = a.t.lens[s];
  TreePages r;
  r.tree = tree_of(a.trees, s);
  r.at = b;
  r.len = len < 0 ? 0 : (int)(len < most ? len : most);
  r.ctx = r.len - r.tree.n;
  r.lo = a.window && r.ctx - a.window + 1 > 0 ? r.ctx - a.window + 1 : 0;
  r.first = r.lo / kPage;
  r.last = r.tree.n > 0 ? ceil_div_d(r.len, kPage) : r.first;
  return r;
}

// Units of work and how they are cut: draft_pieces.hpp.  There are cells where the sums of cut units' pieces wait to be joined.  Every workgroup finds `per` and its piece by itself, from the lengths of all sequences, a lane
// each; that is one chain of loads more or less as long as a search for its sequence would be.
struct Piece {
  TreePages sp;                    // of its sequence
  int kv, tile, piece, pieces;     // pieces: of the unit; 0 where there is nothing to do
  int64_t cell;                    // -1 where the unit is not cut
};
// What the join has to know of a sequence: cell of the first piece of its first unit, how far the next piece's is, how many pieces.
typedef int4 Cut;

__device__ __forceinline__ float wave_total(float v) {
  v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x111, 0xf, 0xf, true));    // row_shr:1, 2, 4, 8; the last lanes of rows to the next, of two rows to the next two
  v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x112, 0xf, 0xf, true));
  v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x114, 0xf, 0xf, true));
  v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x118, 0xf, 0xf, true));
  v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x142, 0xa, 0xf, false));
  v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x143, 0xc, 0xf, false));
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), kWave - 1));
}
__device__ __forceinline__ int64_t of_lane(int64_t v, int lane) {
  return (int64_t)((uint64_t)(unsigned)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32 | (unsigned)__builtin_amdgcn_readlane((int)v, lane));
}

// Piece number `at` of the list: those of cut units first, which take longest; sequence by sequence; of one its pieces, of those the key heads, of those the tiles.  By the whole wave.
__device__ __forceinline__ Piece schedule(const TreeAttendArgs& a, int64_t at) {
  float work = 0.0f, units = 0.0f;
  TreePages sp;
  int pages = 0, tiles = 0;
  auto look = [&](int b) {
    const int s = b + lane_id();
    pages = tiles = 0;
    if (s < a.t.seqs) {
      sp = tree_pages(a, s);
      pages = max(sp.last - sp.first, 0);
      tiles = pages ? ceil_div_d(sp.tree.n * a.group, kTreeRows) : 0;
    }
  };
  for (int b = 0; b < a.t.seqs; b += kWave) {
    look(b);
    work += (float)pages * (float)tiles;
    units += (float)tiles;
  }
  const int per = uniform(pages_of_piece(wave_total(work) * (float)a.c.heads, wave_total(units) * (float)a.c.heads, a.places, [](float x) { return fast_rcp(x); }));
  Piece p{};
  int64_t before = 0;              // pieces of cut units, then of all, of the sequences before these 64
  for (int cut = 1; cut >= 0 && p.pieces == 0; --cut)
    for (int b = 0; b < a.t.seqs; b += kWave) {
      if (a.t.seqs > kWave) look(b);
      const int pieces = ceil_div_d(pages, per), each = tiles * a.c.heads, count = (pieces > 1) == (cut == 1) ? pieces * each : 0;
      const int upto = wave_incl_scan(count);
      const unsigned long long hit = __ballot(count > 0 && at >= before + upto - count && at < before + upto);
      if (hit) {
        const int lane = uniform(__builtin_ctzll(hit));
        auto its = [&](int v) { return __builtin_amdgcn_readlane(v, lane); };
        p.sp = TreePages{Tree{of_lane(sp.tree.first, lane), its(sp.tree.n)}, of_lane(sp.at, lane), its(sp.len), its(sp.ctx), its(sp.lo), its(sp.first), its(sp.last)};
        p.pieces = its(pieces);
        p.cell = cut ? at : -1;
        const int first = its(upto - count), i = (int)(at - before) - first, n = its(tiles), stride = its(each);
        p.tile = i % n;
        p.kv = i / n % a.c.heads;
        p.piece = i / stride;
        if (i == 0 && threadIdx.x == 0) a.cuts[b + lane] = make_int4((int)at, stride, p.pieces, n);
        break;
      }
      before += __builtin_amdgcn_readlane(upto, kWave - 1);
    }
  return p;
}

// Of the tree's nodes first .. first + 63 (first may be negative) those that node i, whose ancestors are at `up`, sees: bits; above: how many of its ancestors and itself come behind them.
struct Seen { unsigned long long bits; int above; };
__device__ __forceinline__ Seen seen_nodes(const unsigned long long* up, int words, int first, int window) {
  Seen r{0, 0};
  if (first > -64) {
    const int w0 = first >> 6, sh = first & 63;            // (of a negative first: the word before the first one)
#pragma unroll
    for (int w = -1; w < kNodeWords; ++w) {
      const unsigned long long v = w >= 0 && w < words ? up[w] : 0;
      if (w == w0) { r.bits |= v >> sh; }
      else if (w == w0 + 1) {
        r.bits |= sh ? v << (64 - sh) : 0;
        r.above += __popcll(sh ? v >> sh : v);
      } else if (w > w0 + 1) r.above += __popcll(v);
    }
  }
  if (window) {
    if (r.above >= window) r.bits = 0;
    while (__popcll(r.bits) > window - r.above && r.bits) r.bits &= r.bits - 1;
  }
  return r;
}

// ... and of a page's first `upto` tokens, which lie before the tree, those from `from` on.  (Of keys before the sequence's first there is no page: where ctx is below 0, the first page's bits begin with a later node.)
__device__ __forceinline__ unsigned long long seen_context(int upto, int from) {
  upto = max(upto, 0);
  from = min(max(from, 0), kPage);
  return (upto >= kPage ? ~0ull : (1ull << upto) - 1) & (from == kPage ? 0ull : ~0ull << from);
}

constexpr float kTreeLazy = 3.0f;      // probabilities stay below 2^3 times those of the maximum that the sums are in units of ...
constexpr int kTreeShift = 12;         // ... and are operands 2^12 times as large: at most 2^15, in full digits down to 2^-26
constexpr int kUnitRoom = 6;           // a page's scale may be so much smaller than the sums' unit (powers of two) before that changes

// 32 rows of a wave: what a lane knows of its row (column lane % 32 of the products) and has summed up of it.
template <typename T, int R, bool CAP, bool BIAS>
struct TreeRows {
  static constexpr int kBlocks = R / 32;
  f32x16 acc[kBlocks];             // channels 32 j + 8 (i / 4) + 4 half + i % 4, in units of 2^(unit - 127 - kTreeShift)
  float m, l;                      // what the sums are in units of (log 2), the probabilities' sum
  int unit, most;                  // the largest exponent of a scale of values so far
  float scale2, cap2, slope2;
  int diag, row_lo;                // where the node stands, the first of the context's tokens that it sees
  int64_t token;                   // its row

  __device__ __forceinline__ void begin(const TreeAttendArgs& a, const TreePages& sp, int64_t token_, int head, bool real) {
#pragma unroll
    for (int j = 0; j < kBlocks; ++j) acc[j] = f32x16{};
    m = -INFINITY;
    l = 0.0f;
    unit = most = 0;
    token = token_;
    scale2 = CAP ? a.score.scale / a.score.cap * (2.0f * kLog2e) : a.score.scale * kLog2e;
    cap2 = a.score.cap * kLog2e;
    slope2 = BIAS && real ? a.score.slopes[head] * kLog2e : 0.0f;
    diag = sp.ctx + (real ? a.trees.node[token].depth : 0);
    row_lo = a.window ? diag - a.window + 1 : 0;
  }

  // From the products q.k of a page's keys to its probabilities.  x[t][i] is key H half + 32 t + i (H 16) or 32 t + 16 (i / 8) + i % 8 (H 8) of the page; p[2 t + i / 8][i % 8] becomes its probability, as an
  // operand, 0 where the page's values are too small for them to show: the product is made all the same, so that a value that is NaN reaches the rows.
  template <int H>
  static __device__ __forceinline__ constexpr int key(int t, int i) { return H == 16 ? 32 * t + i : 32 * t + 16 * (i / 8) + i % 8; }
  template <int H>
  __device__ __forceinline__ void weigh(const TreeAttendArgs& a, const TreePages& sp, f32x16 (&x)[2], int k0, bool whole, float ks, float vs, int half, vec8<f16_t> (&p)[4]) {
    const float c = fmaxf(scale2 * ks, 1.17549435e-38f);      // (above 0: what is not seen is -inf times it)
    // a score, in units of log 2, is zero + unit2 x; with a cap alone x is 1 / (e^2y + 1), of which the tanh is 1 - 2 x, so that a smaller x is a larger score and what is not seen has x = inf
    constexpr bool kFalls = CAP && !BIAS;
    constexpr float kUnseen = kFalls ? INFINITY : -INFINITY;
    const float unit2 = kFalls ? -2.0f * cap2 : BIAS ? 1.0f : c, zero = kFalls ? cap2 : 0.0f;
    if constexpr (CAP || BIAS) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          float y = x[t][i] * c;
          if constexpr (kFalls) y = fast_rcp(fast_exp2(y) + 1.0f);
          else if constexpr (CAP) y = tanh_of(y) * cap2;
          x[t][i] = y;
        }
    }
    if (whole) {
      if constexpr (BIAS) {
        const float away = (float)(diag - k0 - H * half);
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int i = 0; i < 16; ++i) x[t][i] -= slope2 * (away - (float)key<H>(t, i));
      }
    } else {
      const Seen nodes = seen_nodes(a.trees.up + token * a.trees.words, a.trees.words, k0 - sp.ctx, a.window);
      const int upto = min(max(sp.ctx - k0, 0), kPage);
      const unsigned long long mine = (seen_context(upto, row_lo - k0) | nodes.bits) >> (H * half), own = nodes.bits >> (H * half);
      const unsigned lo = (unsigned)mine, hi = (unsigned)(mine >> 32), own_lo = (unsigned)own, own_hi = (unsigned)(own >> 32);
      const int context = upto - H * half, away = diag - k0 - H * half;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int b = key<H>(t, i);
          const bool sees = (b < 32 ? lo : hi) >> (b % 32) & 1;
          if constexpr (BIAS) {
            // nodes between: those of the ancestors that come behind the key
            const unsigned above = b % 32 == 31 ? 0u : ~0u << (b % 32 + 1);
            const int between = nodes.above + (b < 32 ? __popc(own_lo & above) + __popc(own_hi) : __popc(own_hi & above));
            x[t][i] -= slope2 * (float)(b < context ? away - b : between);
          }
          x[t][i] = sees ? x[t][i] : kUnseen;
        }
    }
    float top = kFalls ? __builtin_elementwise_minimum(x[0][0], x[1][0]) : __builtin_elementwise_maximum(x[0][0], x[1][0]);      // (NaN where a score is: then nothing else matters of the row)
#pragma unroll
    for (int i = 1; i < 16; ++i) top = kFalls ? min3(top, x[0][i], x[1][i]) : max3(top, x[0][i], x[1][i]);
    top = max_halves(__builtin_fmaf(top, unit2, zero));
    // The sums go to a new unit only where some row's maximum has grown by more than 2^3, or the page's scale is larger than the unit or much smaller.  Not further down than 2^-64 of the
    // largest scale so far: a page of zeros has the scale 2^-100, next to which sums of large values would overflow.
    const int exponent = uniform((int)(__float_as_uint(vs) >> 23));
    most = max(most, exponent);
    const bool other = exponent > unit || exponent < unit - kUnitRoom;
    if (other || __any(top > m + kTreeLazy)) {
      const float now = top > m + kTreeLazy ? top : m;                            // (a row's own: what its neighbours hold changes none of its bits)
      const float by = m == now ? 1.0f : fast_exp2(m - now);
      const int new_unit = other ? max(exponent, most - 64) : unit, shift = unit - new_unit;
      m = now;
      unit = new_unit;
      l *= by;
#pragma unroll
      for (int j = 0; j < kBlocks; ++j)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[j][i] = __builtin_amdgcn_ldexpf(acc[j][i] * by, shift);
    }
    const int below = max(exponent - unit, -40);                                  // 0 and less; what lies further down only the sum of probabilities shows
    const float base = (m == -INFINITY ? 0.0f : m) - (float)(kTreeShift + below) - zero;
    float sum = 0.0f;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float e = fast_exp2(__builtin_fmaf(x[t][i], unit2, -base));
        sum += e;
        p[2 * t + i / 8][i % 8] = (f16_t)e;
      }
    l += __builtin_amdgcn_ldexpf(sum, -kTreeShift - below);
    if (exponent - unit != below)
#pragma unroll
      for (int i = 0; i < 4; ++i) p[i] = vec8<f16_t>{};
  }
};

// The bytes of a word of four tokens whose bits are set.
__device__ __forceinline__ unsigned bytes_of(unsigned bits) { return ((bits & 15u) * 0x00204081u & 0x01010101u) * 0xffu; }
// The highest bit of every byte that is NaN (0x7f, 0xff).
__device__ __forceinline__ unsigned nan_bytes(unsigned w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }
// Values of a page that some rows do not see as a whole: the product multiplies all of them, by 0 where a row does not see them, so what is NaN becomes 0; the rows that see it become NaN in the end.
__device__ __forceinline__ unsigned proper_bytes(unsigned w, bool& strange) {
  const unsigned nan = nan_bytes(w);
  strange |= nan != 0;
  return w & ~((nan >> 7) * 0xffu);
}

// Where a workgroup is: its sequence, its pages begin .. end - 1, its rows, and the cell that its sums go to (-1: nothing to join with).
struct TreePlace {
  TreePages sp;
  int64_t cell;
  int kv, tile, begin, end, rows;
};

// The pages of a piece, one after another: the table's entries come 64 at a time, one a lane.
struct PageList {
  const int32_t* entries;
  int64_t pages;
  int first, end, mine;           // mine: of the lane's page, first + lane
  __device__ __forceinline__ PageList(const TreeAttendArgs& a, const TreePlace& at) : entries(a.t.page + at.sp.at), pages(a.c.pages), end(at.end) { fetch(at.begin); }
  __device__ __forceinline__ void fetch(int n) {
    first = n;
    mine = n + lane_id() < end ? entries[n + lane_id()] : -1;
  }
  // -1 where the cache has no such page.  n does not fall.
  __device__ __forceinline__ int64_t operator()(int n) {
    if (n >= end) return -1;
    if (n >= first + kWave) fetch(n);
    const int p = __builtin_amdgcn_readlane(mine, n - first);
    return p >= 0 && p < pages ? p : (int64_t)-1;
  }
};

// The scales of a page, asked for with its bytes: as vector loads, for waits on scalar ones (which come out of order) would be waits on everything in LDS.
struct Scales {
  float k, v;
  __device__ __forceinline__ void load(const TreeAttendArgs& a, int64_t page, int kv) {
    const int64_t at = page * a.c.heads + kv + in_loop(0);
    k = a.c.k_scale[at];
    v = a.c.v_scale[at];
  }
};
__device__ __forceinline__ float uniform_of(float v) { return __uint_as_float((unsigned)uniform((int)__float_as_uint(v))); }

// At most 64 rows: the four waves take the pages in turn (with more than 32 rows two pairs of them do), each page from memory to registers, and are joined in LDS.
template <typename T, int R, bool CAP, bool BIAS>
__device__ __forceinline__ bool tree_few_rows(const TreeAttendArgs& a, const TreePlace& at, TreeRows<T, R, CAP, BIAS>& rows, int block, int blocks, const vec8<T>* q) {
  constexpr int kSteps = R / 16, kBlocks = R / 32;
  const TreePages& sp = at.sp;
  const int lane = lane_id(), half = lane >> 5, col = lane & 31, wave = uniform(threadIdx.x / kWave), turns = 4 / blocks;
  const int last_lo = a.window ? sp.ctx + sp.tree.n - a.window : 0;                 // no node's window begins behind it
  u32x4 kw[2][kBlocks], vw[kBlocks][2];

  PageList page_of(a, at);
  Scales scales;
  const int key = 16 * ((col >> 2) & 1) + 4 * (col >> 3) + (col & 3);
  auto load_k = [&](int64_t page) {
    const unsigned char* p = a.c.k + (page * a.c.heads + at.kv) * (kPage * R) + key * R + 16 * half;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < kBlocks; ++i) kw[t][i] = *reinterpret_cast<const u32x4*>(p + 32 * t * R + 32 * i);
  };
  auto load_v = [&](int64_t page) {
    const unsigned char* p = a.c.v + (page * a.c.heads + at.kv) * (kPage * R) + col * kPage + 16 * half;
#pragma unroll
    for (int j = 0; j < kBlocks; ++j)
#pragma unroll
      for (int t = 0; t < 2; ++t) vw[j][t] = *reinterpret_cast<const u32x4*>(p + 32 * j * kPage + 32 * t);
  };

  bool strange = false;
  int n = block * 32 < at.rows ? at.begin + wave / blocks : at.end;
  int64_t page = page_of(n);
  if (page >= 0) { scales.load(a, page, at.kv); load_k(page); load_v(page); }
  while (n < at.end) {
    const int next = n + turns;
    const int64_t next_page = page_of(next);
    if (page >= 0) {
      const float ks = uniform_of(scales.k), vs = uniform_of(scales.v);
      if (a.c.bytes8 < R) {                        // channels behind the head's may hold anything, and 0 times NaN is NaN
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
          const unsigned keep = 32 * (i / 2) + 16 * half + 8 * (i % 2) < a.c.bytes8 ? ~0u : 0u;
#pragma unroll
          for (int t = 0; t < 2; ++t) { kw[t][i / 2][2 * (i % 2)] &= keep; kw[t][i / 2][2 * (i % 2) + 1] &= keep; }
        }
      }
      f32x16 x[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        x[t] = f32x16{};
#pragma unroll
        for (int i = 0; i < kSteps; ++i) x[t] = mma(widen(u32x2{kw[t][i / 2][2 * (i % 2)], kw[t][i / 2][2 * (i % 2) + 1]}, T()), q[i], x[t]);
      }
      if (next_page >= 0) { scales.load(a, next_page, at.kv); load_k(next_page); }
      const int k0 = n * kPage;
      const bool whole = k0 + kPage <= sp.ctx && k0 >= last_lo;
      vec8<f16_t> p[4];
      rows.template weigh<16>(a, sp, x, k0, whole, ks, vs, half, p);
      if (!whole) {
        const unsigned long long live = seen_context(sp.len - k0, sp.lo - k0) >> in_loop(16 * half);
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            const unsigned bytes = bytes_of((unsigned)(live >> (32 * t + 4 * w)));
#pragma unroll
            for (int j = 0; j < kBlocks; ++j) vw[j][t][w] = proper_bytes(vw[j][t][w] & bytes, strange);
          }
      }
#pragma unroll
      for (int j = 0; j < kBlocks; ++j)
#pragma unroll
        for (int u = 0; u < 4; ++u) rows.acc[j] = mma(widen(u32x2{vw[j][u / 2][2 * (u % 2)], vw[j][u / 2][2 * (u % 2) + 1]}, f16_t()), p[u], rows.acc[j]);
      if (next_page >= 0) load_v(next_page);
    } else if (next_page >= 0) {
      scales.load(a, next_page, at.kv);
      load_k(next_page);
      load_v(next_page);
    }
    n = next;
    page = next_page;
  }
  return strange;
}

// More than 64 rows: a wave has its own 32, and all go over the same pages.  A page is widened to 16 bits once, on its way to LDS, where the four waves read it; the next one's bytes come to registers
// meanwhile.  Keys lie there in the order of the products' rows: row 16 c + 8 a + 4 h + b holds key 16 c + 8 h + 4 a + b, so that half h of the wave has 8 neighbouring keys of every 16, one read of a value's channel.
template <typename T, int R>
struct TreeTiles {
  __align__(16) unsigned char k[2][kPage * R * 2], v[2][kPage * R * 2];
};
template <typename T, int R, bool CAP, bool BIAS>
__device__ __forceinline__ bool tree_many_rows(const TreeAttendArgs& a, const TreePlace& at, TreeRows<T, R, CAP, BIAS>& rows, const vec8<T>* q, bool busy, TreeTiles<T, R>& tiles) {
  using SK = TileShape<R>;
  using SV = TileShape<64>;
  constexpr int kSteps = R / 16, kBlocks = R / 32, kPieces = kPage * R / 16 / 256;        // 16 bytes of a page that a thread brings
  const TreePages& sp = at.sp;
  const int lane = lane_id(), half = lane >> 5, tid = threadIdx.x;
  const int last_lo = a.window ? sp.ctx + sp.tree.n - a.window : 0;
  u32x4 kw[kPieces], vw[kPieces];
  PageList page_of(a, at);
  Scales scales;
  auto load = [&](int64_t page) {
    const int64_t at0 = (page * a.c.heads + at.kv) * (kPage * R) + tid * 16;
    scales.load(a, page, at.kv);
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      kw[i] = *reinterpret_cast<const u32x4*>(a.c.k + at0 + i * 4096);
      vw[i] = *reinterpret_cast<const u32x4*>(a.c.v + at0 + i * 4096);
    }
  };
  bool strange = false;
  auto whole_page = [&](int n) { return n * kPage + kPage <= sp.ctx && n * kPage >= last_lo; };
  auto store = [&](int n, int into) {
    const bool whole = whole_page(n);
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int piece = tid + 256 * i;
      {
        const int key = piece / (R / 16), chunk = piece % (R / 16) * 2, row = (key & 0x33) | (key & 4) << 1 | (key & 8) >> 1;
        u32x4 w = kw[i];
        if (a.c.bytes8 < R) {                        // channels behind the head's may hold anything, and 0 times NaN is NaN
          if (chunk * 8 >= a.c.bytes8) w[0] = w[1] = 0;
          if (chunk * 8 + 8 >= a.c.bytes8) w[2] = w[3] = 0;
        }
        unsigned char* to = tiles.k[into] + row * SK::kRowBytes;
        *reinterpret_cast<vec8<T>*>(to + ((chunk ^ SK::swizzle(row)) << 4)) = widen(u32x2{w[0], w[1]}, T());
        *reinterpret_cast<vec8<T>*>(to + (((chunk + 1) ^ SK::swizzle(row)) << 4)) = widen(u32x2{w[2], w[3]}, T());
      }
      {
        const int channel = piece / 4, chunk = piece % 4 * 2;
        u32x4 w = vw[i];
        if (!whole) {
          const unsigned live = (unsigned)(seen_context(sp.len - n * kPage, sp.lo - n * kPage) >> in_loop(chunk * 8));      // (in_loop: not computed where it is not wanted)
#pragma unroll
          for (int j = 0; j < 4; ++j) w[j] = proper_bytes(w[j] & bytes_of(live >> (4 * j)), strange);
        }
        unsigned char* to = tiles.v[into] + channel * SV::kRowBytes;
        *reinterpret_cast<vec8<f16_t>*>(to + ((chunk ^ SV::swizzle(channel)) << 4)) = widen(u32x2{w[0], w[1]}, f16_t());
        *reinterpret_cast<vec8<f16_t>*>(to + (((chunk + 1) ^ SV::swizzle(channel)) << 4)) = widen(u32x2{w[2], w[3]}, f16_t());
      }
    }
  };
  const int k_base = SK::row_base(lane), v_base = SV::row_base(lane);
  int n = at.begin;
  int64_t page = page_of(n);
  float ks = 0.0f, vs = 0.0f;
  if (page >= 0) {
    load(page);
    store(n, 0);
    ks = uniform_of(scales.k);
    vs = uniform_of(scales.v);
  }
  for (int from = 0; n < at.end; ++n, from ^= 1) {
    const int64_t next = page_of(n + 1);
    if (next >= 0) load(next);
    __syncthreads();                                 // the page is there; the one before it is not read any more
    if (page >= 0 && busy) {
      const unsigned char *kt = tiles.k[from], *vt = tiles.v[from];
      f32x16 x[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        x[t] = f32x16{};
#pragma unroll
        for (int i = 0; i < kSteps; ++i) x[t] = mma(SK::template row<T>(kt, k_base, 32 * t, i), q[i], x[t]);
      }
      const bool whole = whole_page(n);
      vec8<f16_t> p[4];
      rows.template weigh<8>(a, sp, x, n * kPage, whole, ks, vs, half, p);
#pragma unroll
      for (int j = 0; j < kBlocks; ++j)
#pragma unroll
        for (int u = 0; u < 4; ++u) rows.acc[j] = mma(SV::template row<f16_t>(vt, v_base, 32 * j, u), p[u], rows.acc[j]);
    }
    if (next >= 0) {
      store(n + 1, from ^ 1);
      ks = uniform_of(scales.k);
      vs = uniform_of(scales.v);
    }
    page = next;
  }
  return strange;
}

// A workgroup has `chunk` pages of a sequence, a key head and up to 128 rows.  The second product is in float16 whatever the type: e4m3 values are exact in it, and probabilities keep 11 digits instead of bfloat16's 8.
template <typename T, int R, bool CAP, bool BIAS>
__global__ void __launch_bounds__(256, tree_resident(R)) k_tree_attend(TreeAttendArgs a) {
  constexpr int kSteps = R / 16, kBlocks = R / 32;
  const int lane = lane_id(), half = lane >> 5, col = lane & 31, wave = uniform(threadIdx.x / kWave);
  TreePlace at;
  // workgroups go to the eight dies in turn: 16 neighbours of the list stay on one, whose L2 cache then has the pages for all tiles of a unit
  const unsigned die = blockIdx.x % 8, turn = blockIdx.x / 8;
  const int64_t number = (int64_t)(turn / 16 * 8 + die) * 16 + turn % 16;
  if (a.chunk == 0) {
    const Piece mine = schedule(a, number);
    if (mine.pieces == 0) return;
    at.sp = mine.sp;
    at.kv = mine.kv;
    at.tile = mine.tile;
    const int pages = ceil_div_d(at.sp.last - at.sp.first, mine.pieces);
    at.begin = uniform(at.sp.first + mine.piece * pages);
    at.end = uniform(min(at.begin + pages, at.sp.last));
    at.cell = mine.cell;
  } else {
    // many sequences: places of chunks, found without knowing the lengths.  s has ptr[s] / chunk + s and on
    at.tile = (int)(number % a.tiles);
    at.kv = (int)(number / a.tiles % a.c.heads);
    const int64_t slot = number / a.tiles / a.c.heads;
    const int s = uniform(find_seq(a.t.seqs, slot, [&](int i) { return first_page(a.t, i) / a.chunk + i; }));
    at.sp = tree_pages(a, s);
    const int64_t piece = slot - (at.sp.at / a.chunk + s);
    if (piece < 0 || piece * a.chunk >= at.sp.last) return;
    at.begin = uniform(max(at.sp.first, (int)piece * a.chunk));
    at.end = uniform(min(at.sp.last, (int)(piece + 1) * a.chunk));
    at.cell = at.sp.first / a.chunk == (at.sp.last - 1) / a.chunk ? -1 : ((chunk_cell(at.sp.at, a.chunk) + piece) * a.c.heads + at.kv) * a.tiles + at.tile;
  }
  const TreePages& sp = at.sp;
  at.rows = uniform(min(sp.tree.n * a.group - at.tile * kTreeRows, kTreeRows));
  if (at.rows <= 0 || at.begin >= at.end || at.cell >= a.cells) return;
  const int blocks = at.rows <= 32 ? 1 : at.rows <= 64 ? 2 : 4;        // blocks of rows
  const int block = wave % blocks;

  const int r = block * 32 + col, rr = at.tile * kTreeRows + r, head = at.kv * a.group + rr % a.group;
  const bool real = r < at.rows;
  const int64_t token = sp.tree.first + (real ? rr / a.group : 0);
  TreeRows<T, R, CAP, BIAS> rows;
  rows.begin(a, sp, token, head, real);
  vec8<T> q[kSteps];
  {
    const RowSource src = a.q.of(real ? head : 0);
    const unsigned char* p = src.base + token * src.stride;
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      const int d = blocks == 4 ? 16 * i + 8 * half : 32 * (i / 2) + 16 * half + 8 * (i % 2);
      u32x4 w = {0, 0, 0, 0};
      if (real && d < a.c.bytes8) w = *reinterpret_cast<const u32x4*>(p + d * 2);
      q[i] = __builtin_bit_cast(vec8<T>, w);
    }
  }
  struct Joined {
    float ms[4][32], ls[4][32], by[4][32];             // by: what a wave's sums of a row are multiplied by
    int64_t to[kTreeRows];                             // bytes from the results' first element, of a row that is written there
    unsigned long long nan[R];                         // of a page's channels: the tokens whose value is NaN
    __align__(16) float sums[4][32][R + 4];
  };
  __shared__ __align__(16) union { TreeTiles<T, R> tiles; Joined joined; } lds;
  bool strange;
  if (blocks == 4) strange = tree_many_rows<T, R, CAP, BIAS>(a, at, rows, q, block * 32 < at.rows, lds.tiles);
  else strange = tree_few_rows<T, R, CAP, BIAS>(a, at, rows, block, blocks, q);
  strange = __syncthreads_or(strange);             // (and the tiles are not read any more)
  const float m = rows.m, l = add_halves(rows.l);

  // join the waves of the same rows by their maxima
  Joined& j = lds.joined;
  if (half == 0) { j.ms[wave][col] = m; j.ls[wave][col] = l; }
#pragma unroll
  for (int c = 0; c < kBlocks; ++c)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f32x4 v;
#pragma unroll
      for (int b = 0; b < 4; ++b) v[b] = __builtin_amdgcn_ldexpf(rows.acc[c][4 * i + b], rows.unit - 127 - kTreeShift);
      *reinterpret_cast<f32x4*>(&j.sums[wave][col][32 * c + 8 * i + 4 * half]) = v;
    }
  __syncthreads();
  if (strange) {
    // rows that see a value that is NaN: of every page whose values were made proper the tokens that are, channel by channel, and then two threads a row.  (Of pages that all rows see the product has made the rows NaN.)
    const int last_lo = a.window ? sp.ctx + sp.tree.n - a.window : 0, rt = threadIdx.x / 2;
    for (int n = at.begin; n < at.end; ++n) {
      const int k0 = n * kPage;
      const int64_t page = a.t.page[sp.at + n];
      if ((k0 + kPage <= sp.ctx && k0 >= last_lo) || page < 0 || page >= a.c.pages) continue;
      if (threadIdx.x < R) {
        const u32x4* v = reinterpret_cast<const u32x4*>(a.c.v + (page * a.c.heads + at.kv) * (kPage * R) + threadIdx.x * kPage);
        unsigned long long nan = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const u32x4 w = v[i];
#pragma unroll
          for (int b = 0; b < 4; ++b) nan |= (unsigned long long)((nan_bytes(w[b]) >> 7) * 0x10204080u >> 28) << (16 * i + 4 * b);      // (a bit for each byte)
        }
        j.nan[threadIdx.x] = nan;
      }
      __syncthreads();
      if (rt < at.rows) {
        const int64_t its = sp.tree.first + (at.tile * kTreeRows + rt) / a.group;
        const int stands = sp.ctx + a.trees.node[its].depth;
        const unsigned long long sees = seen_context(min(max(sp.ctx - k0, 0), kPage), a.window ? stands - a.window + 1 - k0 : 0) |
                                        seen_nodes(a.trees.up + its * a.trees.words, a.trees.words, k0 - sp.ctx, a.window).bits;
        for (int d = threadIdx.x % 2; d < R; d += 2)
          if (sees & j.nan[d]) j.sums[rt / 32][rt % 32][d] = NAN;
      }
      __syncthreads();
    }
  }
  const int row = threadIdx.x;
  if (row < at.rows) {
    const int first = row / 32, mine = row % 32;
    float top = -INFINITY, sum = 0.0f;
    for (int w = first; w < 4; w += blocks) top = fmaxf(top, j.ms[w][mine]);
    const float base = top == -INFINITY ? 0.0f : top;
    for (int w = first; w < 4; w += blocks) {
      const float f = fast_exp2(j.ms[w][mine] - base);
      sum += j.ls[w][mine] * f;
      j.by[w][mine] = f;
    }
    if (at.cell < 0) {
      const float by = sum == 0.0f ? 0.0f : 1.0f / sum;
      for (int w = first; w < 4; w += blocks) j.by[w][mine] *= by;
      const int rt = at.tile * kTreeRows + row;
      j.to[row] = (sp.tree.first + rt / a.group) * a.o.stride + (int64_t)(at.kv * a.group + rt % a.group) * a.o.head;
    } else {
      a.part_ml[at.cell * a.part_rows + row] = make_float2(top, sum);
    }
  }
  __syncthreads();
  // a thread has four channels of every (1024 / R)-th row
  constexpr int kThreads = R / 4, kStep = 256 / kThreads;
  const int d = threadIdx.x % kThreads * 4;
  for (int i = threadIdx.x / kThreads; i < at.rows; i += kStep) {
    f32x4 v = *reinterpret_cast<const f32x4*>(&j.sums[i / 32][i % 32][d]) * j.by[i / 32][i % 32];
    for (int w = i / 32 + blocks; w < 4; w += blocks) v += *reinterpret_cast<const f32x4*>(&j.sums[w][i % 32][d]) * j.by[w][i % 32];
    if (at.cell >= 0) *reinterpret_cast<f32x4*>(a.part + (at.cell * a.part_rows + i) * R + d) = v;
    else if (d < a.c.bytes8) {
      T out[4];
#pragma unroll
      for (int b = 0; b < 4; ++b) out[b] = (T)v[b];
      *reinterpret_cast<u32x2*>(a.o.base + j.to[i] + d * 2) = __builtin_bit_cast(u32x2, out);
    }
  }
}

// Joins the pieces of a unit; rows that no piece has (no tokens) become zero.  A workgroup has a node and a key head: R / 4 lanes go over every (256 / R)-th piece of a row, four channels each, and what they
// have is joined in order; the four waves take the rows of the heads that share the key head in turn.
template <typename T, int R>
__global__ void __launch_bounds__(256) k_tree_join(TreeAttendArgs a) {
  constexpr int kThreads = R / 4, kLanes = kWave / kThreads;
  const int64_t token = blockIdx.x;
  const int kv = blockIdx.y;
  const int4 place = load_uniform(a.trees.place + token);
  if (place.y == 0) return;
  const TreePages sp = tree_pages(a, place.z);
  const int64_t node = token - sp.tree.first;
  if (node < 0 || node >= sp.tree.n) return;
  int pieces = 0;
  int64_t cell0 = 0, stride = 0;         // cell0: of key head kv, the first tile, the first piece
  int tiles = a.tiles;
  if (sp.first < sp.last) {
    if (a.chunk == 0) {
      const Cut cut = load_uniform(a.cuts + place.z);
      pieces = cut.z == 1 ? 1 : (int)min((int64_t)cut.z, a.cells);      // (no cut unit has more; of rows whose pointers do not ascend the launch may not have come to write this)
      tiles = cut.w;
      cell0 = cut.x;
      stride = cut.y;
    } else {
      const int c0 = sp.first / a.chunk;
      pieces = (sp.last - 1) / a.chunk + 1 - c0;
      cell0 = (chunk_cell(sp.at, a.chunk) + c0) * a.c.heads * a.tiles;
      stride = (int64_t)a.c.heads * a.tiles;
    }
    if (pieces == 1) return;
  }
  const int first = (int)node * a.group;
  for (int g = threadIdx.x / kWave; g < a.group; g += 4) {
    const int rr = first + g, d = lane_id() % kThreads * 4, mine = lane_id() / kThreads;
    const int64_t cell = cell0 + (int64_t)kv * tiles + rr / kTreeRows;
    float top = -INFINITY, sum = 0.0f;
    f32x4 v = {0, 0, 0, 0};
#pragma unroll 4
    for (int c = mine; c < pieces; c += kLanes) {
      if ((uint64_t)(cell + c * stride) >= (uint64_t)a.cells) break;
      const int64_t row = (cell + c * stride) * a.part_rows + rr % kTreeRows;
      const float2 ml = a.part_ml[row];
      const f32x4 w = *reinterpret_cast<const f32x4*>(a.part + row * R + d);
      const float now = fmaxf(top, ml.x), base = now == -INFINITY ? 0.0f : now;
      const float f = fast_exp2(top - base), g2 = fast_exp2(ml.x - base);
      v = v * f + w * g2;
      sum = sum * f + ml.y * g2;
      top = now;
    }
#pragma unroll
    for (int step = kThreads; step < kWave; step *= 2) {
      const float other = __shfl_xor(top, step), all = fmaxf(top, other), base = all == -INFINITY ? 0.0f : all;
      const float f = fast_exp2(top - base), g2 = fast_exp2(other - base);
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = v[j] * f + __shfl_xor(v[j], step) * g2;
      sum = sum * f + __shfl_xor(sum, step) * g2;
      top = all;
    }
    if (mine || d >= a.c.bytes8) continue;
    const float by = sum == 0.0f ? 0.0f : 1.0f / sum;
    const RowSource dst = a.o.of(kv * a.group + g);
    T out[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) out[j] = (T)(v[j] * by);
    *reinterpret_cast<u32x2*>(const_cast<unsigned char*>(dst.base) + token * dst.stride + d * 2) = __builtin_bit_cast(u32x2, out);
  }
}

}  // namespace spg
