// Trees of drafted tokens: their structure, and the attention of their nodes over the paged cache.
//
// A wave has 32 rows (a node and a head that shares the key head) as right operands and takes a page of 64 tokens in two products of 32 keys (32 x 32 x 16 form, attn_common.hpp).  Row 8a + 4h + b
// of product t is key 32 t + 16 h + 4 a + b, so that half h of the wave, whose lanes have the rows 8a + 4h + b of a result, has the 16 neighbouring keys 32 t + 16 h and on of a page: in the order in
// which 16 bytes of a value's channel hold them.  So the probabilities are the second product's right operand as they leave the first, and
// pages go from memory to registers, 16 bytes a lane and load, without LDS.
#pragma once
#include "cache_kernels.hpp"

namespace spg {

constexpr int kMostNodes = 256, kNodeWords = kMostNodes / 64;

struct TreeView {
  const int64_t* ptr;             // rows + 1
  int rows, most, words;          // words: of 64 bits, that a node's ancestors take
  int64_t tokens;
  unsigned long long* up;         // [tokens][words]: the node's ancestors and itself
  int4* node;                     // [tokens]: parent, first child, next node of the same parent (each -1: none), depth
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

// A workgroup has a tree: a thread walks up from its node through the parents in LDS, and looks through all nodes for its first child and its next sibling.
__global__ void __launch_bounds__(kMostNodes) k_trees(TreeView t, const int32_t* parent) {
  __shared__ int par[kMostNodes];
  const Tree tree = tree_of(t, blockIdx.x);
  const int i = threadIdx.x;
  int p = -1;
  if (i < tree.n) {
    p = parent[tree.first + i];
    p = p >= 0 && p < i ? p : -1;
  }
  par[i] = p;
  __syncthreads();
  if (i >= tree.n) return;
  unsigned long long up[kNodeWords] = {};
  int depth = -1;
  for (int a = i; a >= 0; a = par[a]) {
    ++depth;
#pragma unroll
    for (int w = 0; w < kNodeWords; ++w) up[w] |= a / 64 == w ? 1ull << (a % 64) : 0ull;
  }
  int child = -1, next = -1;
  for (int j = tree.n - 1; j > 0; --j) {
    const int pj = par[j];
    child = pj == i ? j : child;
    next = j > i && pj == p ? j : next;
  }
  t.node[tree.first + i] = make_int4(p, child, next, depth);
#pragma unroll
  for (int w = 0; w < kNodeWords; ++w)
    if (w < t.words) t.up[(tree.first + i) * t.words + w] = up[w];
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

struct TreeAttendArgs {
  CacheView c;
  TableView t;
  TreeView trees;
  HeadTensor q, o;          // row ptr[s] + i: node i of sequence s
  int heads, group, tiles, window;
  int chunk;                // pages of a workgroup
  int64_t slots;            // places of chunks
  int part_rows;            // rows that a workgroup's part has places for
  ScoreShape score;
  float* part;              // [slots][key heads][tiles][part_rows][R]: sums of what the workgroups saw, not divided
  float2* part_ml;          // [slots][key heads][tiles][part_rows]: maximum (units of log 2) and sum
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

constexpr float kTreeLazy = 3.0f;      // probabilities stay below 2^3 times those of the maximum that the sums are in units of ...
constexpr int kTreeShift = 12;         // ... and are operands 2^12 times as large: at most 2^15, in full digits down to 2^-26
constexpr int kUnitRoom = 6;           // a page's scale may be so much smaller than the sums' unit (powers of two) before that changes

// A workgroup has `chunk` pages of a sequence, a key head and up to 128 rows.  With at most 32 rows its four waves take the pages in turn, with at most 64 two pairs of them, else each has its own rows; waves of
// the same rows are joined in LDS.  The second product is in float16 whatever the type: e4m3 values are exact in it, and probabilities keep 11 digits instead of bfloat16's 8.
template <typename T, int R, bool CAP, bool BIAS>
__global__ void __launch_bounds__(256, 2) k_tree_attend(TreeAttendArgs a) {
  constexpr int kSteps = R / 16, kBlocks = R / 32;
  const int lane = lane_id(), half = lane >> 5, col = lane & 31, wave = uniform(threadIdx.x / kWave);
  // tiles of the same pages go to one die, one after the other: its L2 cache then has the pages for all of them
  const unsigned die = blockIdx.x % 8, turn = blockIdx.x / 8;
  const int tile = turn % a.tiles;
  const int64_t unit_no = (int64_t)(turn / a.tiles) * 8 + die;
  const int kv = (int)(unit_no % a.c.heads);
  const int64_t slot = unit_no / a.c.heads;
  if (slot >= a.slots) return;
  const int s = uniform(find_seq(a.t.seqs, slot, [&](int i) { return first_page(a.t, i) / a.chunk + i; }));
  const TreePages sp = tree_pages(a, s);
  const int rows = uniform(min(sp.tree.n * a.group - tile * kTreeRows, kTreeRows));
  const int64_t piece = slot - (sp.at / a.chunk + s);
  if (rows <= 0 || piece < 0 || piece * a.chunk >= sp.last) return;
  const int begin = uniform(max(sp.first, (int)piece * a.chunk)), end = uniform(min(sp.last, (int)(piece + 1) * a.chunk));
  if (begin >= end) return;
  const bool alone = sp.first / a.chunk == (sp.last - 1) / a.chunk;    // nothing to join with
  const int blocks = rows <= 32 ? 1 : rows <= 64 ? 2 : 4, turns = 4 / blocks;      // blocks of rows; waves that take the pages of one in turn
  const int block = wave % blocks;

  const int r = block * 32 + col, rr = tile * kTreeRows + r, node = rr / a.group, head = kv * a.group + rr % a.group;
  const bool real = r < rows;
  const int64_t token = sp.tree.first + (real ? node : 0);
  vec8<T> q[kSteps];
  {
    const RowSource src = a.q.of(real ? head : 0);
    const unsigned char* p = src.base + token * src.stride;
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      const int d = 32 * (i / 2) + 16 * half + 8 * (i % 2);
      u32x4 w = {0, 0, 0, 0};
      if (real && d < a.c.bytes8) w = *reinterpret_cast<const u32x4*>(p + d * 2);
      q[i] = __builtin_bit_cast(vec8<T>, w);
    }
  }
  const float scale2 = CAP ? a.score.scale / a.score.cap * (2.0f * kLog2e) : a.score.scale * kLog2e, cap2 = a.score.cap * kLog2e;
  const float slope2 = BIAS && real ? a.score.slopes[head] * kLog2e : 0.0f;
  const int diag = sp.ctx + (real ? a.trees.node[token].w : 0);                     // where the node stands
  const int row_lo = a.window ? diag - a.window + 1 : 0;
  const int last_lo = a.window ? sp.ctx + sp.tree.n - a.window : 0;                 // no node's window begins behind it

  f32x16 acc[kBlocks];
#pragma unroll
  for (int j = 0; j < kBlocks; ++j) acc[j] = f32x16{};
  float m = -INFINITY, l = 0.0f;                   // what the sums are in units of (log 2), the probabilities' sum
  int unit = 0, most = 0;                          // acc is in units of 2^(unit - 127 - kTreeShift); the largest exponent of a scale of values so far
  u32x4 kw[2][kBlocks], vw[kBlocks][2];

  auto page_of = [&](int n) {
    const int64_t p = load_uniform(a.t.page + sp.at + n);
    return p >= 0 && p < a.c.pages ? p : (int64_t)-1;
  };
  const int key = 16 * ((col >> 2) & 1) + 4 * (col >> 3) + (col & 3);
  auto load_k = [&](int64_t page) {
    const unsigned char* p = a.c.k + (page * a.c.heads + kv) * (kPage * R) + key * R + 16 * half;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < kBlocks; ++i) kw[t][i] = *reinterpret_cast<const u32x4*>(p + 32 * t * R + 32 * i);
  };
  auto load_v = [&](int64_t page) {
    const unsigned char* p = a.c.v + (page * a.c.heads + kv) * (kPage * R) + col * kPage + 16 * half;
#pragma unroll
    for (int j = 0; j < kBlocks; ++j)
#pragma unroll
      for (int t = 0; t < 2; ++t) vw[j][t] = *reinterpret_cast<const u32x4*>(p + 32 * j * kPage + 32 * t);
  };

  int n = block * 32 < rows ? begin + wave / blocks : end;
  int64_t page = n < end ? page_of(n) : -1;
  if (page >= 0) { load_k(page); load_v(page); }
  while (n < end) {
    const int next = n + turns;
    const int64_t next_page = next < end ? page_of(next) : -1;
    if (page >= 0) {
      const float ks = load_uniform(a.c.k_scale + page * a.c.heads + kv), vs = load_uniform(a.c.v_scale + page * a.c.heads + kv);
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
      if (next_page >= 0) load_k(next_page);
      const int k0 = n * kPage;
      const float c = fmaxf(scale2 * ks, 1.17549435e-38f);      // (above 0: what is not seen is -inf times it)
      float unit2 = c;                              // of x, in units of log 2
      if constexpr (CAP || BIAS) {
        unit2 = BIAS ? 1.0f : cap2;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            float y = x[t][i] * c;
            if constexpr (CAP) y = tanh_of(y);
            if constexpr (CAP && BIAS) y *= cap2;
            x[t][i] = y;
          }
      }
      const bool whole = k0 + kPage <= sp.ctx && k0 >= last_lo;
      unsigned seen[2] = {0xffffu, 0xffffu};        // of the lane's keys 32 t + 16 half + i
      if (whole) {
        if constexpr (BIAS) {
          const float away = (float)(diag - k0 - 16 * half);
#pragma unroll
          for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) x[t][i] -= slope2 * (away - (float)(32 * t + i));
        }
      } else {
        const Seen nodes = seen_nodes(a.trees.up + token * a.trees.words, a.trees.words, k0 - sp.ctx, a.window);
        const int upto = min(max(sp.ctx - k0, 0), kPage), from = min(max(row_lo - k0, 0), kPage);
        const unsigned long long before = upto == kPage ? ~0ull : (1ull << upto) - 1, behind = from == kPage ? 0ull : ~0ull << from;
        // (keys before the sequence's first are never asked for: a node's bits begin at ctx, which is below 0 only where k0 is 0)
        const unsigned long long bits = (before & behind) | (upto == kPage ? 0ull : nodes.bits >> upto << upto);
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          seen[t] = (unsigned)(bits >> (32 * t + 16 * half)) & 0xffffu;
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            if constexpr (BIAS) {
              const int b = 32 * t + 16 * half + i;
              const int far = b < upto ? diag - k0 - b : nodes.above + __popcll(b == 63 ? 0ull : nodes.bits >> (b + 1));
              x[t][i] -= slope2 * (float)far;
            }
            x[t][i] = seen[t] >> i & 1 ? x[t][i] : -INFINITY;
          }
        }
        // what no row of the sequence sees may hold anything: as values it becomes zero
        unsigned strange = 0;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const int off = k0 + 32 * t + 16 * half, dead = sp.lo - off, live = sp.len - off;       // keys below dead and from live on
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            unsigned mask = 0;
#pragma unroll
            for (int b = 0; b < 4; ++b) mask |= 4 * w + b >= dead && 4 * w + b < live ? 0xffu << (8 * b) : 0u;
#pragma unroll
            for (int j = 0; j < kBlocks; ++j) {
              vw[j][t][w] &= mask;
              strange |= ((vw[j][t][w] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
            }
          }
        }
        // a NaN among the values (0x7f, 0xff) reaches the rows that see it and no others, though the product multiplies it by the zeros of all: it is taken
        // out, and a product of what is seen with 1 in its place says whose results it makes NaN
        if (__any(strange != 0)) {
          vec8<f16_t> sees[4];
#pragma unroll
          for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int i = 0; i < 8; ++i) sees[u][i] = seen[u / 2] >> (8 * (u % 2) + i) & 1 ? (f16_t)1.0f : (f16_t)0.0f;
#pragma unroll
          for (int j = 0; j < kBlocks; ++j) {
            f32x16 hit = {};
#pragma unroll
            for (int u = 0; u < 4; ++u) {
              vec8<f16_t> is;
#pragma unroll
              for (int i = 0; i < 8; ++i) {
                const unsigned w = vw[j][u / 2][2 * (u % 2) + i / 4];
                is[i] = (w >> (8 * (i % 4)) & 0x7fu) == 0x7fu ? (f16_t)1.0f : (f16_t)0.0f;
              }
              hit = mma(is, sees[u], hit);
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[j][i] = hit[i] > 0.0f ? NAN : acc[j][i];
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
              for (int w = 0; w < 4; ++w) {
                const unsigned nan = ((vw[j][t][w] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;      // its byte's highest bit
                vw[j][t][w] &= ~((nan >> 7) * 0xffu);
              }
          }
        }
      }
      float top = max3(x[0][0], x[0][1], x[0][2]);
#pragma unroll
      for (int i = 3; i < 15; i += 2) top = fmaxf(top, fmaxf(x[0][i], x[0][i + 1]));
      top = fmaxf(top, x[0][15]);
#pragma unroll
      for (int i = 0; i < 16; i += 2) top = fmaxf(top, fmaxf(x[1][i], x[1][i + 1]));
      top = max_halves(top) * unit2;
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
      const float base = (m == -INFINITY ? 0.0f : m) - (float)(kTreeShift + below);
      vec8<f16_t> p[4];
      float sum = 0.0f;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float e = fast_exp2(__builtin_fmaf(x[t][i], unit2, -base));
          sum += e;
          p[2 * t + i / 8][i % 8] = (f16_t)e;
        }
      if (exponent - unit < below)
#pragma unroll
        for (int u = 0; u < 4; ++u) p[u] = vec8<f16_t>{};
      l += __builtin_amdgcn_ldexpf(sum, -kTreeShift - below);
#pragma unroll
      for (int j = 0; j < kBlocks; ++j)
#pragma unroll
        for (int u = 0; u < 4; ++u) acc[j] = mma(widen(u32x2{vw[j][u / 2][2 * (u % 2)], vw[j][u / 2][2 * (u % 2) + 1]}, f16_t()), p[u], acc[j]);
      if (next_page >= 0) load_v(next_page);
    } else if (next_page >= 0) {
      load_k(next_page);
      load_v(next_page);
    }
    n = next;
    page = next_page;
  }
  l = add_halves(l);

  // join the waves of the same rows by their maxima
  __shared__ float ms[4][32], ls[4][32];
  __shared__ __align__(16) float sums[4][32][R + 4];
  if (half == 0) { ms[wave][col] = m; ls[wave][col] = l; }
#pragma unroll
  for (int j = 0; j < kBlocks; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f32x4 v;
#pragma unroll
      for (int b = 0; b < 4; ++b) v[b] = __builtin_amdgcn_ldexpf(acc[j][4 * i + b], unit - 127 - kTreeShift);
      *reinterpret_cast<f32x4*>(&sums[wave][col][32 * j + 8 * i + 4 * half]) = v;
    }
  __syncthreads();
  const int64_t cell = (slot * a.c.heads + kv) * a.tiles + tile;
  for (int i = threadIdx.x; i < rows * (R / 4); i += 256) {
    const int row = i / (R / 4), d = i % (R / 4) * 4, at = row % 32;
    float top = -INFINITY;
    for (int w = row / 32; w < 4; w += blocks) top = fmaxf(top, ms[w][at]);
    const float base = top == -INFINITY ? 0.0f : top;
    f32x4 v = {0, 0, 0, 0};
    float sum = 0.0f;
    for (int w = row / 32; w < 4; w += blocks) {
      const float f = fast_exp2(ms[w][at] - base);
      v += *reinterpret_cast<const f32x4*>(&sums[w][at][d]) * f;
      sum += ls[w][at] * f;
    }
    if (alone) {
      if (d < a.c.bytes8) {
        const float by = sum == 0.0f ? 0.0f : 1.0f / sum;
        const int rt = tile * kTreeRows + row;
        const RowSource dst = a.o.of(kv * a.group + rt % a.group);
        T out[4];
#pragma unroll
        for (int b = 0; b < 4; ++b) out[b] = (T)(v[b] * by);
        *reinterpret_cast<u32x2*>(const_cast<unsigned char*>(dst.base) + (sp.tree.first + rt / a.group) * dst.stride + d * 2) = __builtin_bit_cast(u32x2, out);
      }
    } else {
      *reinterpret_cast<f32x4*>(a.part + (cell * a.part_rows + row) * R + d) = v;
      if (d == 0) a.part_ml[cell * a.part_rows + row] = make_float2(top, sum);
    }
  }
}

// Joins a row's chunks; rows that no chunk has (no tokens) become zero.  A workgroup has a node and a head: R / 4 threads go over every (1024 / R)-th
// chunk, four channels each, and their sums are joined in order.
template <typename T, int R>
__global__ void __launch_bounds__(256) k_tree_join(TreeAttendArgs a) {
  constexpr int kThreads = R / 4, kLanes = 256 / kThreads;
  const int64_t token = blockIdx.x;
  const int head = blockIdx.y, kv = head / a.group;
  const int s = uniform(find_seq(a.trees.rows, token, [&](int i) { return tree_begin(a.trees, i); }));
  const TreePages sp = tree_pages(a, s);
  const int64_t node = token - sp.tree.first;
  if (node < 0 || node >= sp.tree.n) return;
  const bool none = sp.first >= sp.last;
  const int c0 = none ? 0 : sp.first / a.chunk, c1 = none ? 0 : (sp.last - 1) / a.chunk + 1;
  if (c1 - c0 == 1) return;
  const int rr = (int)node * a.group + head % a.group, d = threadIdx.x % kThreads * 4, mine = threadIdx.x / kThreads;
  const int64_t slot = sp.at / a.chunk + s;
  float top = -INFINITY, sum = 0.0f;
  f32x4 v = {0, 0, 0, 0};
#pragma unroll 4
  for (int c = c0 + mine; c < c1; c += kLanes) {
    const int64_t row = (((slot + c) * a.c.heads + kv) * a.tiles + rr / kTreeRows) * a.part_rows + rr % kTreeRows;
    const float2 ml = a.part_ml[row];
    const f32x4 w = *reinterpret_cast<const f32x4*>(a.part + row * R + d);
    const float now = fmaxf(top, ml.x), base = now == -INFINITY ? 0.0f : now;
    const float f = fast_exp2(top - base), g = fast_exp2(ml.x - base);
    v = v * f + w * g;
    sum = sum * f + ml.y * g;
    top = now;
  }
  __shared__ __align__(16) f32x4 vs[256];
  __shared__ float2 mls[kLanes];
  vs[threadIdx.x] = v;
  if (d == 0) mls[mine] = make_float2(top, sum);
  __syncthreads();
  if (mine || d >= a.c.bytes8) return;
  float all = -INFINITY, total = 0.0f;
#pragma unroll
  for (int i = 0; i < kLanes; ++i) all = fmaxf(all, mls[i].x);
  all = all == -INFINITY ? 0.0f : all;
  v = f32x4{0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < kLanes; ++i) {
    const float f = fast_exp2(mls[i].x - all);
    v += vs[i * kThreads + threadIdx.x] * f;
    total += mls[i].y * f;
  }
  const float by = total == 0.0f ? 0.0f : 1.0f / total;
  const RowSource dst = a.o.of(head);
  T out[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) out[j] = (T)(v[j] * by);
  *reinterpret_cast<u32x2*>(const_cast<unsigned char*>(dst.base) + token * dst.stride + d * 2) = __builtin_bit_cast(u32x2, out);
}

}  // namespace spg
