// Attention over a planned mask, forward.
//
// A workgroup of four waves has 128 queries of a head, a wave 32 of them: its queries stay in registers as the right operand, keys and values
// come through LDS in tiles of 64, one tile ahead.  The scores of a tile leave the first product with one query a lane (both halves of the wave
// hold half of its keys each), so maximum and sum of a row are the lane's own but for one exchange between the halves, and the
// probabilities are the second product's right operand as they are (attn_common.hpp).  One pass: out = sum_j 2^(x_j - m) v_j with the running
// maximum m; sums and maxima in 32 bits, probabilities rounded to 16 bits once, as an operand.  The accumulators are brought to a
// new maximum only where some row's grew by more than 2^8 since (the sum is in the same units, so nothing is approximated).
//
// Measured (bfloat16, 128 channels): two documents of 8192 tokens together, 16 heads on 8, capped, 199 us, 0.69 PFLOP/s (call after call without a trace 176, 0.78); 5003 queries over 11 147 keys through a
// pattern, 32 heads on 8, with distances, 165 us, 0.68 (144, 0.78).  Vector instructions issue in 59 % of the cycles (51 in the second), eight an entry with a cap,
// three of them powers and reciprocals; matrix instructions run in 39 % (39), LDS in 19 %: what vector and matrix instructions take
// together bounds it, for two waves a SIMD, as many as the registers allow, hardly overlap.  Tiles of 32 keys for three waves, products of the next tile beside
// the powers of this one (in the order of the code or by hints to the scheduler) and priorities were all slower.  Short rows (documents of a few
// hundred tokens) are bound by the chain of their tiles, 2 us each.
#pragma once
#include "attn_common.hpp"

namespace spg {

constexpr float kLazyMax = 8.0f;   // probabilities stay below 2^8 times the running maximum's

struct HeadTensor {       // rows of a packed tensor with heads: token t of head h begins at base + t * stride + h * head (bytes)
  unsigned char* base;
  int64_t stride, head;
  __device__ __forceinline__ RowSource of(int h) const { return {base + (int64_t)h * head, stride}; }
};

// Long rows may be shared by several workgroups, each with a stretch of the tiles; their sums are joined, in order, by a kernel of their own (joined by the
// last workgroup to finish, the fences that takes cost every workgroup more than the launch: 18 + 8 | 49 us).  A workgroup leaves the registers of its
// accumulators as they are: float4 [piece][workgroup][4 D / 32][256], and for rows maximum and sum.  2003 tokens, 8 heads: forward 33 | 17 us and 5 to join.
struct Split {
  int most;               // pieces that the grid has places for (1: nothing is shared)
  int slots;              // workgroups that the card holds at once
  f32x4* sums;
  float2* tops;           // [piece][workgroup][128]: maximum in units of log 2, sum
};

// How many pieces n tiles are cut into.  A piece is half as long again as the average of what the card's `slots` places have to do (total: what
// all workgroups have), and at least kLeastTiles: shorter ones cost more in joining than they save (gradients of documents of 4096 tokens, pieces
// of 1, 1.25, 1.5 and 2 averages: 98, 88, 86, 103 us).  So all together are cut into at most 2/3 slots more than they are.
constexpr int kLeastTiles = 4;
__device__ __forceinline__ int pieces_of(int n, int slots, unsigned long long total) {
  const float even = fminf((float)total * 1.5f / (float)slots, (float)n);   // (a large number in 24 bits: less than one tile off)
  const int per = max((int)even + 1, kLeastTiles);
  return n > 2 * kLeastTiles ? ceil_div_d(n, per) : 1;
}
// The stretch of n tiles that a piece has.
struct Share { int first, last, pieces; };
__device__ __forceinline__ Share share_of(int n, int pieces, int piece) {
  const int per = ceil_div_d(n, pieces);
  return {uniform(min(piece * per, n)), uniform(min((piece + 1) * per, n)), uniform(pieces)};
}
__device__ __forceinline__ Share share_of(const Split& sp, int n, unsigned long long total, int piece) {
  if (sp.most == 1) return {0, n, 1};
  return share_of(n, uniform(min(pieces_of(n, sp.slots, total), sp.most)), piece);
}

struct AttnArgs {
  HeadTensor q, k, v, o;
  float* lse;             // [heads][q_len], natural logarithm
  int q_len, k_len, heads, group, bytes, q_tiles;
  PlanView plan;
  ScoreShape score;
  Split split;
};

// What the gradients need to know of 64 rows of a head: what their exponents add to s * mul (ScoreFactors; -inf for a row that sees nothing or
// does not exist), minus the sums of dO * O, and their bounds.
struct RowFacts {
  float base[kQueryTile], less[kQueryTile];
  int lo[kQueryTile], hi[kQueryTile], diag[kQueryTile];
};

struct Counts { int keys, cut_keys, queries, cut_queries; };
struct AttnGrads {
  HeadTensor d_o, dq, dk, dv;
  // in the workspace:
  RowFacts* facts;        // [heads][ceil(q_len / 128) * 2]
  int4 *k_list, *q_list;  // work, most first: tile, what it reaches from y to before z, pieces of it + 65536 * this piece; for every (key) head
  Counts* counts;         // entries of both lists, and how many of them, all in front, are pieces of cut tiles
  f32x4* sums;            // [pieces and heads of keys, then of queries][4 D / 32][256]
  int more;               // entries that a list can hold beside its tiles
  int slots;              // workgroups that the card holds at once; 0: nothing is cut
};

// Which head and tile a workgroup has, and what the tile reaches.  Workgroups go to the eight dies in turn: heads that share keys stay on one, whose
// L2 cache then holds them once.  The tiles with the most to do come first.
struct Place { int head, tile, lo, hi, piece; };
__device__ __forceinline__ Place place_of(int n, int heads, const int4* order) {
  int head, rank;
  if (heads % 8 == 0) {
    const int per = heads / 8, j = n / 8;
    head = n % 8 * per + j % per;
    rank = j / per;
  } else {
    head = n % heads;
    rank = n / heads;
  }
  const int4 o = load_uniform(order + uniform(rank));
  return {uniform(head), o.x, o.y, o.z, o.w};
}

// The first tile of 64 keys (queries) at or behind c, before end, whose flag is set; two of them share a flag.
static_assert(kPatTile == 2 * kKeyTile && kPatTile == 2 * kQueryTile, "tiles of a flag");
__device__ __forceinline__ int next_tile(const unsigned* flags, int c, int end) {
  if (!flags) return c;
  while (c < end) {
    const int b = c >> 1;
    const unsigned w = load_uniform(flags + (b >> 5)) >> (b & 31);
    if (w & 1) return c;
    c = uniform(w ? (b + __ffs(w) - 1) << 1 : ((b >> 5) + 1) << 6);
  }
  return end;
}

// Factors of a head's scores, and how what shape_scores leaves becomes an exponent: x = s * mul + add.
struct ScoreFactors { float scale2, cap2, slope2, mul, add; };
template <bool CAP, bool BIAS>
__device__ __forceinline__ ScoreFactors score_factors(const ScoreShape& sh, int head) {
  ScoreFactors f;
  f.scale2 = CAP ? sh.scale / sh.cap * (2.0f * kLog2e) : sh.scale * kLog2e;
  f.cap2 = sh.cap * kLog2e;
  f.slope2 = BIAS ? load_uniform(sh.slopes + head) * kLog2e : 0.0f;
  f.mul = BIAS ? 1.0f : CAP ? -2.0f * f.cap2 : f.scale2;
  f.add = CAP && !BIAS ? f.cap2 : 0.0f;
  return f;
}

// A score from a product s, `d` = slope2 |diag - j|.  Without a cap: x = scale2 s - d, in units of log 2 (s itself where there is no distance
// either).  With one: r = 1 / (1 + e^2y), where y is the score by the cap, so that tanh y = 1 - 2r and 1 - tanh^2 y = 4 (r - r^2) (`back` is a
// quarter of that); without distances r itself is left, which spares two operations an entry: x = cap2 - 2 cap2 r falls with r.
template <bool CAP, bool BIAS>
__device__ __forceinline__ float shaped(float s, const ScoreFactors& f, float d, float* back) {
  if constexpr (CAP) {
    s = fast_rcp(fast_exp2(s * f.scale2) + 1.0f);
    if (back) *back = __builtin_fmaf(-s, s, s);
    if constexpr (BIAS) s = __builtin_fmaf(s, -2.0f * f.cap2, f.cap2 - d);
  } else if constexpr (BIAS) {
    s = __builtin_fmaf(s, f.scale2, -d);
  }
  return s;
}

// The bounds of a wave's rows.
__device__ __forceinline__ GroupBound wave_bound(const AttnArgs& a, int tile, int wave) {
  const int g = tile * (kPatTile / kRowGroup) + wave;
  return g < ceil_div_d(a.q_len, kRowGroup) ? load_uniform(a.plan.groups + g) : GroupBound{0, 0, 0, 0};
}

// A row's output from its lanes' accumulators, N channels from c0 on; with its logarithm.
template <typename T, int N>
__device__ __forceinline__ void store_rows(const HeadTensor& to, int head, int row, int half, int c0, int bytes, const f32x16* acc, float by) {
  unsigned char* out = to.base + (int64_t)head * to.head + (int64_t)row * to.stride;
#pragma unroll
  for (int i = 0; i < N / 32; ++i)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int byte = (c0 + 32 * i + 8 * r + 4 * half) * 2;
      T v[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = (T)(acc[i][4 * r + j] * by);
      if (byte < bytes) *reinterpret_cast<u32x2*>(out + byte) = __builtin_bit_cast(u32x2, v);
    }
}
template <typename T, int N>
__device__ __forceinline__ void finish_rows(const AttnArgs& a, int head, int row, int half, int c0, const f32x16* acc, float m, float l) {
  if (row >= a.q_len) return;
  if (half == 0 && c0 == 0) a.lse[(int64_t)head * a.q_len + row] = l == 0.0f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
  store_rows<T, N>(a.o, head, row, half, c0, a.bytes, acc, l == 0.0f ? 0.0f : 1.0f / l);
}

template <int D>
__device__ __forceinline__ void leave_sums(f32x4* sums, int64_t cell, const f32x16* acc) {
  f32x4* to = sums + cell * (D / 8 * 256) + threadIdx.x;
#pragma unroll
  for (int i = 0; i < D / 32; ++i)
#pragma unroll
    for (int r = 0; r < 4; ++r) to[(4 * i + r) * 256] = f32x4{acc[i][4 * r], acc[i][4 * r + 1], acc[i][4 * r + 2], acc[i][4 * r + 3]};
}
// Adds the 32 channels from c0 on of a piece.
template <int D>
__device__ __forceinline__ void add_sums(const f32x4* sums, int64_t cell, int c0, float by, f32x16& acc) {
  const f32x4* from = sums + cell * (D / 8 * 256) + c0 / 8 * 256 + threadIdx.x;
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const f32x4 x = from[r * 256];
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[4 * r + j] = __builtin_fmaf(x[j], by, acc[4 * r + j]);
  }
}

// With a cap and no distances |x| <= cap2, so that a fixed maximum will do: none is looked for, exchanged or raised (BOUNDED: 8192 tokens 216 -> 201 us).
// It is cap2, less what keeps the smallest power at 2^-120; the largest is then 2^(2 cap2 - 120), for which float and bfloat16 have room up to a cap2
// of 76 (2^32, times 2^30 keys, times values up to 2^65); float16 has none.
constexpr float kBoundedCap2 = 76.0f;
__device__ __forceinline__ float fixed_maximum(float cap2) { return cap2 - fmaxf(0.0f, 2.0f * cap2 - 120.0f); }

template <typename T, int D, bool CAP, bool BIAS, bool BOUNDED>
__global__ void __launch_bounds__(256, 2) k_attn_fwd(AttnArgs a) {
  static_assert(!BOUNDED || (CAP && !BIAS), "bounded scores");
  using S = TileShape<D>;
  __shared__ __align__(16) unsigned char k_even[kKeyTile * D * 2], v_even[kKeyTile * D * 2], k_odd[kKeyTile * D * 2], v_odd[kKeyTile * D * 2];
  const Place at = place_of(blockIdx.x, a.heads, a.plan.q_order);
  const int head = at.head, qt = at.tile, lo = at.lo, hi = at.hi;
  const int lane = lane_id(), half = lane >> 5, wave = uniform(threadIdx.x / kWave);
  const int row_base = S::row_base(lane), across_base = S::across_base(lane);
  const int row = qt * kPatTile + wave * kRowGroup + (lane & 31);
  const GroupBound mine = wave_bound(a, qt, wave);
  const ScoreFactors f = score_factors<CAP, BIAS>(a.score, head);
  const RowBound rb = row < a.q_len ? a.plan.rows[row] : RowBound{0, 0, 0, 0};
  vec8<T> q[D / 16];
  load_row<T, D>(a.q.of(head), row, row < a.q_len, a.bytes, half, q);
  const int kv = uniform(head / a.group);
  const RowSource ks = a.k.of(kv), vs = a.v.of(kv);
  const TileLoader<D, kKeyTile, 256> load_k(ks.stride, lane), load_v(vs.stride, lane);
  f32x16 acc[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) acc[i] = f32x16{};
  float m = BOUNDED ? fixed_maximum(f.cap2) : -INFINITY, l = 0.0f;

  const unsigned* flags = a.plan.seen_words ? a.plan.seen + (int64_t)qt * a.plan.seen_words : nullptr;
  const int begin = lo / kKeyTile;
  const Share share = share_of(a.split, ceil_div_d(hi, kKeyTile) - begin, a.split.most > 1 ? load_uniform(a.plan.totals) * a.heads : 0, blockIdx.y);
  if ((int)blockIdx.y >= share.pieces) return;
  const int end = begin + share.last;

  float key_part[16];                                // slope2 times a key's place among a lane's
  int least_diag = 0;                                // of the wave's rows
  if constexpr (BIAS && !CAP) {
#pragma unroll
    for (int i = 0; i < 16; ++i) key_part[i] = f.slope2 * (float)(8 * (i / 4) + i % 4);
    least_diag = row < a.q_len ? rb.diag : 0x7fffffff;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) least_diag = min(least_diag, __shfl_xor(least_diag, d));
    least_diag = uniform(least_diag);
  }
  constexpr bool kFalls = CAP && !BIAS;              // the smallest s is the largest score
  const float hidden = kFalls ? INFINITY : -INFINITY;
  auto compute = [&](const unsigned char* kt, const unsigned char* vt, int k0) {
    if (mine.lo >= k0 + kKeyTile || mine.hi <= k0) return;
    const bool whole = mine.all_lo <= k0 && mine.all_hi >= k0 + kKeyTile;
    f32x16 s[kKeyTile / 32];
#pragma unroll
    for (int t = 0; t < kKeyTile / 32; ++t) s[t] = f32x16{};
#pragma unroll
    for (int j = 0; j < kKeyTile / 32 * (D / 16); ++j) {   // (both halves in turn where a cap follows, 8192 tokens 176 us, one after the other 180; without one 146 | 144)
      const int t = CAP ? j % 2 : j / (D / 16), i = CAP ? j / 2 : j % (D / 16);
      s[t] = mma(S::template row<T>(kt, row_base, 32 * t, i), q[i], s[t]);
    }
    // Where every key of a tile is at or before every row, a distance is a row's part less a key's: the key's goes into the product's scaling, the row's
    // into the exponent, and an entry costs two operations less (5003 queries through a pattern: 174 -> 169.5 us).
    float row_part[kKeyTile / 32] = {};
    if (BIAS && !CAP && whole && k0 + kKeyTile - 1 <= least_diag) {
#pragma unroll
      for (int t = 0; t < kKeyTile / 32; ++t) {
        row_part[t] = f.slope2 * (float)(k0 + 4 * half + 32 * t - rb.diag);
#pragma unroll
        for (int i = 0; i < 16; ++i) s[t][i] = __builtin_fmaf(s[t][i], f.scale2, key_part[i]);
      }
    } else if constexpr (CAP || BIAS) {
      const float away = (float)(rb.diag - k0 - 4 * half);
#pragma unroll
      for (int t = 0; t < kKeyTile / 32; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[t][i] = shaped<CAP, BIAS>(s[t][i], f, f.slope2 * fabsf(away - (float)(32 * t + 8 * (i / 4) + i % 4)), nullptr);
    }
    if (!whole) {
      const unsigned span = rb.hi > rb.lo ? rb.hi - rb.lo : 0;
      const int off = k0 + 4 * half - rb.lo;
#pragma unroll
      for (int t = 0; t < kKeyTile / 32; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[t][i] = (unsigned)(off + 32 * t + 8 * (i / 4) + i % 4) < span ? s[t][i] : hidden;
    }
    if constexpr (!BOUNDED) {
      float tops[kKeyTile / 32];
#pragma unroll
      for (int t = 0; t < kKeyTile / 32; ++t) {
        tops[t] = hidden;
#pragma unroll
        for (int i = 0; i < 16; i += 2) tops[t] = kFalls ? min3(tops[t], s[t][i], s[t][i + 1]) : max3(tops[t], s[t][i], s[t][i + 1]);
        tops[t] = __builtin_fmaf(tops[t], f.mul, f.add + row_part[t]);
      }
      const float top = max_halves(fmaxf(tops[0], tops[1]));
      if (__any(top > m + kLazyMax)) {
        const float now = fmaxf(m, top);
        const float by = m == now ? 1.0f : fast_exp2(m - now);
        m = now;
        l *= by;
#pragma unroll
        for (int i = 0; i < D / 32; ++i) acc[i] *= by;
      }
    }
    const float base = f.add - (m == -INFINITY ? 0.0f : m);
    float sum = 0.0f;
#pragma unroll
    for (int t = 0; t < kKeyTile / 32; ++t) {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        s[t][i] = fast_exp2(__builtin_fmaf(s[t][i], f.mul, base + row_part[t]));
        sum += s[t][i];
      }
      vec8<T> p[2];
      to_operand<T>(s[t], p);
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < D / 32; ++i) acc[i] = mma(S::template across<T>(vt, across_base, 32 * t + 16 * u, i), p[u], acc[i]);
    }
    l += sum;
  };
  auto load = [&](unsigned char* kt, unsigned char* vt, int k0) {
    load_tiles(load_k, ks.base, kt, load_v, vs.base, vt, k0, lo, hi, a.bytes);
  };

  int c = next_tile(flags, begin + share.first, end);
  if (c < end) load(k_even, v_even, c * kKeyTile);
  while (c < end) {
    int next = next_tile(flags, c + 1, end);
    tiles_ready();                                  // the tile is there, and nobody reads the other one any more
    if (next < end) load(k_odd, v_odd, next * kKeyTile);
    compute(k_even, v_even, c * kKeyTile);
    c = next;
    if (c >= end) break;
    next = next_tile(flags, c + 1, end);
    tiles_ready();
    if (next < end) load(k_even, v_even, next * kKeyTile);
    compute(k_odd, v_odd, c * kKeyTile);
    c = next;
  }

  l = add_halves(l);
  if (share.pieces > 1) {
    const int64_t cell = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    leave_sums<D>(a.split.sums, cell, acc);
    if (half == 0) a.split.tops[cell * kPatTile + wave * kRowGroup + lane] = make_float2(m, l);
    return;
  }
  finish_rows<T, D>(a, head, row, half, 0, acc, m, l);
}

// A workgroup has 32 channels of a tile's rows.  2003 tokens, 8 heads of 64 channels: 5 us.
template <typename T, int D>
__global__ void __launch_bounds__(256) k_attn_join(AttnArgs a) {
  const Place at = place_of(blockIdx.x, a.heads, a.plan.q_order);
  const Share share = share_of(a.split, ceil_div_d(at.hi, kKeyTile) - at.lo / kKeyTile, load_uniform(a.plan.totals) * a.heads, 0);
  if (share.pieces == 1) return;
  const int lane = lane_id(), row = threadIdx.x / kWave * kRowGroup + (lane & 31), c0 = blockIdx.y * 32;
  const float2* tops = a.split.tops + (int64_t)blockIdx.x * kPatTile + row;
  const int64_t step = (int64_t)gridDim.x * kPatTile;
  f32x16 acc = {};
  float m = -INFINITY, l = 0.0f;
#pragma unroll 4
  for (int p = 0; p < share.pieces; ++p) m = fmaxf(m, tops[p * step].x);
  const float base = m == -INFINITY ? 0.0f : m;
#pragma unroll 4
  for (int p = 0; p < share.pieces; ++p) {
    const float2 top = tops[p * step];
    const float by = fast_exp2(top.x - base);
    l = __builtin_fmaf(top.y, by, l);
    add_sums<D>(a.split.sums, (int64_t)p * gridDim.x + blockIdx.x, c0, by, acc);
  }
  finish_rows<T, 32>(a, at.head, at.tile * kPatTile + row, lane >> 5, c0, &acc, m, l);
}

}  // namespace spg
