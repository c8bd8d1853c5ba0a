// Attention over a planned mask, forward.
//
// A workgroup of four waves has 128 queries of a head, a wave 32 of them: its queries stay in registers as the right operand, keys and values
// come through LDS in tiles of 64, one tile ahead.  The scores of a tile leave the first product with one query a lane (both halves of the wave
// hold half of its keys each), so maximum and sum of a row are the lane's own but for one exchange between the halves, and the
// probabilities are the second product's right operand as they are (attn_common.hpp).  One pass: out = sum_j 2^(x_j - m) v_j with the running
// maximum m; sums and maxima in 32 bits, probabilities rounded to 16 bits once, as an operand.  The accumulators are brought to a
// new maximum only where some row's grew by more than 2^8 since (the sum is in the same units, so nothing is approximated).
#pragma once
#include "attn_common.hpp"

namespace spg {

constexpr float kLazyMax = 8.0f;   // probabilities stay below 2^8 times the running maximum's

struct HeadTensor {       // rows of a packed tensor with heads: token t of head h begins at base + t * stride + h * head (bytes)
  unsigned char* base;
  int64_t stride, head;
  __device__ __forceinline__ RowSource of(int h) const { return {base + (int64_t)h * head, stride}; }
};

struct AttnArgs {
  HeadTensor q, k, v, o;
  float* lse;             // [heads][q_len], natural logarithm
  int q_len, k_len, heads, group, bytes, q_tiles;
  PlanView plan;
  ScoreShape score;
};

struct AttnGrads {
  HeadTensor d_o, dq, dk, dv;
  float* lse2;            // workspace [heads][q_len]: the rows' logarithms in units of log 2, +inf for a row that sees nothing
  float* delta;           // workspace [heads][q_len]: the sum of dO * O
};

// Which head and tile of rows a workgroup has.  Workgroups go to the eight dies in turn: heads that share keys stay on one, whose L2 cache then
// holds them once.  Last rows first: under a causal mask they are the longest.
__device__ __forceinline__ void head_and_tile(int n, int heads, int tiles, int* head, int* tile) {
  if (heads % 8 == 0) {
    const int per = heads / 8, j = n / 8;
    *head = uniform(n % 8 * per + j % per);
    *tile = uniform(tiles - 1 - j / per);
  } else {
    *head = uniform(n % heads);
    *tile = uniform(tiles - 1 - n / heads);
  }
}

// The first tile at or behind c, before end, whose flag is set; 1 << shift tiles share a flag.
__device__ __forceinline__ int next_tile(const unsigned* flags, int c, int end, int shift) {
  if (!flags) return c;
  while (c < end) {
    const int b = c >> shift;
    const unsigned w = load_uniform(flags + (b >> 5)) >> (b & 31);
    if (w & 1) return c;
    c = uniform(w ? (b + __ffs(w) - 1) << shift : ((b >> 5) + 1) << (5 + shift));
  }
  return end;
}

// Scores of 32 keys by the lane's query in units of log 2.  `away`: diag - (the lane's first key); for a masked pair -inf.
// keep: tanh of the capped score, for the gradient.
template <bool CAP, bool BIAS, bool KEEP>
__device__ __forceinline__ void shape_scores(f32x16& s, float scale2, float cap2, float slope2, float away, f32x16* keep) {
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    float x;
    if constexpr (CAP) {
      const float t = tanh_of(s[i] * scale2);
      if constexpr (KEEP) (*keep)[i] = t;
      x = t * cap2;
    } else {
      x = s[i] * scale2;
    }
    if constexpr (BIAS) x -= slope2 * fabsf(away - (float)(8 * (i / 4) + i % 4));
    s[i] = x;
  }
}

// scale2, cap2, slope2 of shape_scores.
template <bool CAP, bool BIAS>
__device__ __forceinline__ void score_factors(const ScoreShape& sh, int head, float* scale2, float* cap2, float* slope2) {
  *scale2 = CAP ? sh.scale / sh.cap * (2.0f * kLog2e) : sh.scale * kLog2e;
  *cap2 = sh.cap * kLog2e;
  *slope2 = BIAS ? load_uniform(sh.slopes + head) * kLog2e : 0.0f;
}

template <typename T, int D, bool CAP, bool BIAS>
__global__ void __launch_bounds__(256, 2) k_attn_fwd(AttnArgs a) {
  using S = TileShape<D>;
  __shared__ __align__(16) unsigned char k_even[kKeyTile * D * 2], v_even[kKeyTile * D * 2], k_odd[kKeyTile * D * 2], v_odd[kKeyTile * D * 2];
  int head, qt;
  head_and_tile(blockIdx.x, a.heads, a.q_tiles, &head, &qt);
  const int lane = lane_id(), half = lane >> 5, wave = uniform(threadIdx.x / kWave);
  const int row_base = S::row_base(lane), across_base = S::across_base(lane);
  const int row = qt * kPatTile + wave * kRowGroup + (lane & 31);
  const int groups = ceil_div_d(a.q_len, kRowGroup);
  int lo = 0x7fffffff, hi = 0;                       // keys that any query of the workgroup sees
  GroupBound mine{0, 0, 0, 0};
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const int g = qt * 4 + w;
    if (g >= groups) break;
    const GroupBound b = load_uniform(a.plan.groups + g);
    if (b.hi > b.lo) { lo = min(lo, b.lo); hi = max(hi, b.hi); }
    if (w == wave) mine = b;
  }
  lo = uniform(lo);
  hi = uniform(hi);
  mine = {uniform(mine.lo), uniform(mine.hi), uniform(mine.all_lo), uniform(mine.all_hi)};
  float scale2, cap2, slope2;
  score_factors<CAP, BIAS>(a.score, head, &scale2, &cap2, &slope2);
  const RowBound rb = row < a.q_len ? a.plan.rows[row] : RowBound{0, 0, 0, 0};
  vec8<T> q[D / 16];
  load_row<T, D>(a.q.of(head), row, row < a.q_len, a.bytes, half, q);
  const int kv = uniform(head / a.group);
  const RowSource ks = a.k.of(kv), vs = a.v.of(kv);
  f32x16 acc[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) acc[i] = f32x16{};
  float m = -INFINITY, l = 0.0f;

  const unsigned* flags = a.plan.seen_words ? a.plan.seen + (int64_t)qt * a.plan.seen_words : nullptr;
  const int end = hi > lo ? ceil_div_d(hi, kKeyTile) : 0;

  auto compute = [&](const unsigned char* kt, const unsigned char* vt, int k0) {
    if (mine.lo >= k0 + kKeyTile || mine.hi <= k0) return;
    const bool whole = mine.all_lo <= k0 && mine.all_hi >= k0 + kKeyTile;
    const int at_row = in_loop(row_base), at_across = in_loop(across_base);
    f32x16 s[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      s[t] = f32x16{};
#pragma unroll
      for (int i = 0; i < D / 16; ++i) s[t] = mma(S::template row<T>(kt, at_row, 32 * t, i), q[i], s[t]);
    }
    if constexpr (CAP || BIAS) {
      shape_scores<CAP, BIAS, false>(s[0], scale2, cap2, slope2, (float)(rb.diag - k0 - 4 * half), nullptr);
      shape_scores<CAP, BIAS, false>(s[1], scale2, cap2, slope2, (float)(rb.diag - k0 - 4 * half - 32), nullptr);
    }
    const float c = CAP || BIAS ? 1.0f : scale2;
    if (!whole) {
      const unsigned span = rb.hi > rb.lo ? rb.hi - rb.lo : 0;
      const int off = k0 + 4 * half - rb.lo;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[t][i] = (unsigned)(off + 32 * t + 8 * (i / 4) + i % 4) < span ? s[t][i] : -INFINITY;
    }
    float top = fmaxf(s[0][0], s[1][0]);
#pragma unroll
    for (int i = 1; i < 16; ++i) top = fmaxf(top, fmaxf(s[0][i], s[1][i]));
    top = max_halves(top) * c;
    if (__any(top > m + kLazyMax)) {
      const float now = fmaxf(m, top);
      const float by = m == now ? 1.0f : fast_exp2(m - now);
      m = now;
      l *= by;
#pragma unroll
      for (int i = 0; i < D / 32; ++i) acc[i] *= by;
    }
    const float base = m == -INFINITY ? 0.0f : m;
    float sum = 0.0f;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        s[t][i] = fast_exp2(__builtin_fmaf(s[t][i], c, -base));
        sum += s[t][i];
      }
      vec8<T> p[2];
      to_operand<T>(s[t], p);
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < D / 32; ++i) acc[i] = mma(S::template across<T>(vt, at_across, 32 * t + 16 * u, i), p[u], acc[i]);
    }
    l += sum;
  };
  auto load = [&](unsigned char* kt, unsigned char* vt, int k0) {
    load_tile<D, kKeyTile, 256>(ks, kt, k0, lo, hi, a.bytes);
    load_tile<D, kKeyTile, 256>(vs, vt, k0, lo, hi, a.bytes);
  };

  int c = next_tile(flags, hi > lo ? lo / kKeyTile : 0, end, 1);
  if (c < end) load(k_even, v_even, c * kKeyTile);
  while (c < end) {
    int next = next_tile(flags, c + 1, end, 1);
    tiles_ready();                                  // the tile is there, and nobody reads the other one any more
    if (next < end) load(k_odd, v_odd, next * kKeyTile);
    compute(k_even, v_even, c * kKeyTile);
    c = next;
    if (c >= end) break;
    next = next_tile(flags, c + 1, end, 1);
    tiles_ready();
    if (next < end) load(k_even, v_even, next * kKeyTile);
    compute(k_odd, v_odd, c * kKeyTile);
    c = next;
  }

  if (row >= a.q_len) return;
  l = add_halves(l);
  const float by = l == 0.0f ? 0.0f : 1.0f / l;
  if (half == 0) a.lse[(int64_t)head * a.q_len + row] = l == 0.0f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
  const RowSource os = a.o.of(head);
  unsigned char* out = const_cast<unsigned char*>(os.base) + (int64_t)row * os.stride;
#pragma unroll
  for (int i = 0; i < D / 32; ++i)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int byte = (32 * i + 8 * r + 4 * half) * 2;
      T v[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = (T)(acc[i][4 * r + j] * by);
      if (byte < a.bytes) *reinterpret_cast<u32x2*>(out + byte) = __builtin_bit_cast(u32x2, v);
    }
}

}  // namespace spg
