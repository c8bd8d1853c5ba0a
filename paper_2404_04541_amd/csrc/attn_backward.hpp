// Attention over a planned mask, gradients.
//
// With P = 2^(x - lse2) (x: the shaped scores in units of log 2, lse2 the row's logarithm from the forward pass), dP = dO V^T and
// delta_i = sum_d dO_id O_id:  dV = P^T dO,  dS = P (dP - delta) (1 - tanh^2),  dQ = scale dS K,  dK = scale dS^T Q.
// Two kernels, each with a fixed order of its sums (no atomics: the same inputs give the same bits): k_attn_dq goes over the keys of 128
// queries as the forward kernel does and leaves -delta and what exponents begin with for k_attn_dkv, which goes over the queries, of all heads that share
// them, of 128 keys.  That computes S and dP twice, seven products where five would do with atomics on dQ in 32 bits.
// P, dS are rounded to 16 bits once, as operands; all sums are held in 32 bits.
#pragma once
#include "attn_forward.hpp"

namespace spg {

template <typename T, int D, bool CAP, bool BIAS>
__global__ void __launch_bounds__(256, 2) k_attn_dq(AttnArgs a, AttnGrads g) {
  using S = TileShape<D>;
  __shared__ __align__(16) unsigned char k_even[kKeyTile * D * 2], v_even[kKeyTile * D * 2], k_odd[kKeyTile * D * 2], v_odd[kKeyTile * D * 2];
  int head, qt;
  head_and_tile(blockIdx.x, a.heads, a.plan.q_order, &head, &qt);
  const int lane = lane_id(), half = lane >> 5, wave = uniform(threadIdx.x / kWave);
  const int row_base = S::row_base(lane), across_base = S::across_base(lane);
  const int row = qt * kPatTile + wave * kRowGroup + (lane & 31);
  const int groups = ceil_div_d(a.q_len, kRowGroup);
  int lo = 0x7fffffff, hi = 0;
  GroupBound mine{0, 0, 0, 0};
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const int n = qt * 4 + w;
    if (n >= groups) break;
    const GroupBound b = load_uniform(a.plan.groups + n);
    if (b.hi > b.lo) { lo = min(lo, b.lo); hi = max(hi, b.hi); }
    if (w == wave) mine = b;
  }
  lo = uniform(lo);
  hi = uniform(hi);
  mine = {uniform(mine.lo), uniform(mine.hi), uniform(mine.all_lo), uniform(mine.all_hi)};
  const ScoreFactors f = score_factors<CAP, BIAS>(a.score, head);
  const bool real = row < a.q_len;
  const RowBound rb = real ? a.plan.rows[row] : RowBound{0, 0, 0, 0};
  vec8<T> q[D / 16], d_o[D / 16];
  load_row<T, D>(g.d_o.of(head), row, real, a.bytes, half, d_o);
  float delta = 0.0f, lse2 = INFINITY;   // (a row that sees nothing: every power is 0)
  {
    load_row<T, D>(a.o.of(head), row, real, a.bytes, half, q);   // (O for the moment)
#pragma unroll
    for (int i = 0; i < D / 16; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) delta = __builtin_fmaf((float)d_o[i][j], (float)q[i][j], delta);
    delta = add_halves(delta);
  }
  if (real) {
    const int64_t at = (int64_t)head * a.q_len + row;
    const float v = a.lse[at];
    lse2 = v == -INFINITY ? INFINITY : v * kLog2e;
    if (half == 0) { g.base[at] = f.add - lse2; g.less[at] = -delta; }
  }
  const float base = f.add - lse2;
  load_row<T, D>(a.q.of(head), row, real, a.bytes, half, q);
  const int kv = uniform(head / a.group);
  const RowSource ks = a.k.of(kv), vs = a.v.of(kv);
  const TileLoader<D, kKeyTile, 256> load_k(ks.stride, lane), load_v(vs.stride, lane);
  f32x16 acc[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) acc[i] = f32x16{};

  const unsigned* flags = a.plan.seen_words ? a.plan.seen + (int64_t)qt * a.plan.seen_words : nullptr;
  const int end = hi > lo ? ceil_div_d(hi, kKeyTile) : 0;

  auto compute = [&](const unsigned char* kt, const unsigned char* vt, int k0) {
    if (mine.lo >= k0 + kKeyTile || mine.hi <= k0) return;
    const bool whole = mine.all_lo <= k0 && mine.all_hi >= k0 + kKeyTile;
    const int at_row = in_loop(row_base), at_across = in_loop(across_base);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      f32x16 s = {}, dp = {};
#pragma unroll
      for (int i = 0; i < D / 16; ++i) s = mma(S::template row<T>(kt, at_row, 32 * t, i), q[i], s);
#pragma unroll
      for (int i = 0; i < D / 16; ++i) dp = mma(S::template row<T>(vt, at_row, 32 * t, i), d_o[i], dp);
      const float away = (float)(rb.diag - k0 - 4 * half - 32 * t);
      const unsigned span = rb.hi > rb.lo ? rb.hi - rb.lo : 0;
      const int off = k0 + 4 * half + 32 * t - rb.lo;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        float back;
        const float x = shaped<CAP, BIAS>(s[i], f, f.slope2 * fabsf(away - (float)(8 * (i / 4) + i % 4)), &back);
        s[i] = fast_exp2(__builtin_fmaf(x, f.mul, base)) * (dp[i] - delta);
        if constexpr (CAP) s[i] *= back;
      }
      if (!whole) {
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = (unsigned)(off + 8 * (i / 4) + i % 4) < span ? s[i] : 0.0f;
      }
      vec8<T> p[2];
      to_operand<T>(s, p);
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < D / 32; ++i) acc[i] = mma(S::template across<T>(kt, at_across, 32 * t + 16 * u, i), p[u], acc[i]);
    }
  };
  auto load = [&](unsigned char* kt, unsigned char* vt, int k0) {
    load_tile(load_k, ks.base, kt, k0, lo, hi, a.bytes);
    load_tile(load_v, vs.base, vt, k0, lo, hi, a.bytes);
  };

  int c = next_tile(flags, hi > lo ? lo / kKeyTile : 0, end, 1);
  if (c < end) load(k_even, v_even, c * kKeyTile);
  while (c < end) {
    int next = next_tile(flags, c + 1, end, 1);
    tiles_ready();
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

  if (!real) return;
  const float by = CAP ? 4.0f * a.score.scale : a.score.scale;
  const RowSource os = g.dq.of(head);
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

// A workgroup has 64 keys of a key head and goes over their queries in tiles of 64 rows, head by head.  Wave w has keys 32 (w % 2) .. and of every
// tile the rows 32 (w / 2) ..; keys and values stay in registers as right operands, queries and dO come through LDS with what their exponents and dP
// begin with and their bounds, one tile ahead.  At the end the two waves of the same keys exchange sums: one adds up dK, the other dV.
constexpr int kQueryTile = 64;

template <int D>
struct QueryTile {
  unsigned char q[kQueryTile * D * 2], d_o[kQueryTile * D * 2];
  float base[kQueryTile], less[kQueryTile];
  RowBound rows[kQueryTile];
};

template <typename T, int D, bool CAP, bool BIAS>
__global__ void __launch_bounds__(256, 2) k_attn_dkv(AttnArgs a, AttnGrads g) {
  using S = TileShape<D>;
  __shared__ __align__(16) QueryTile<D> even, odd;
  int kv, kt;
  head_and_tile(blockIdx.x, a.heads / a.group, a.plan.k_order, &kv, &kt);
  const int lane = lane_id(), half = lane >> 5, wave = uniform(threadIdx.x / kWave), part = wave >> 1;
  const int row_base = S::row_base(lane), across_base = S::across_base(lane);
  const int k0 = kt * kKeyTile + (wave & 1) * 32, key = k0 + (lane & 31);
  const bool real = key < a.k_len;
  vec8<T> k[D / 16], v[D / 16];
  load_row<T, D>(a.k.of(kv), key, real, a.bytes, half, k);
  load_row<T, D>(a.v.of(kv), key, real, a.bytes, half, v);
  f32x16 dk[D / 32], dv[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) { dk[i] = f32x16{}; dv[i] = f32x16{}; }

  const int2 span = load_uniform(a.plan.cols + kt);
  const int lo = uniform(span.x), hi = uniform(span.y);
  const unsigned* flags = a.plan.seen_by_words ? a.plan.seen_by + (int64_t)(kt * kKeyTile / kPatTile) * a.plan.seen_by_words : nullptr;
  const int end = hi > lo ? ceil_div_d(hi, kQueryTile) : 0;
  const int begin = next_tile(flags, hi > lo ? lo / kQueryTile : 0, end, 1);

  auto load = [&](QueryTile<D>& t, int head, int tile) {
    const int first = tile * kQueryTile;
    const TileLoader<D, kQueryTile, 256> load_q(a.q.stride, in_loop(lane)), load_do(g.d_o.stride, in_loop(lane));   // (made anew: registers are short)
    load_tile(load_q, a.q.of(head).base, t.q, first, lo, hi, a.bytes);
    load_tile(load_do, g.d_o.of(head).base, t.d_o, first, lo, hi, a.bytes);
    const int64_t at = (int64_t)head * a.q_len + first;
    const unsigned rows = a.q_len - first < kQueryTile ? a.q_len - first : kQueryTile;
    if (wave == 0) {
      const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc((void*)(g.base + at), 0, rows * 4, 0x00027000);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void*)t.base, 4, in_loop(lane) * 4, 0, 0, 0);
    } else if (wave == 1) {
      const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc((void*)(g.less + at), 0, rows * 4, 0x00027000);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void*)t.less, 4, in_loop(lane) * 4, 0, 0, 0);
    } else if (wave == 2) {
      const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc((void*)(a.plan.rows + first), 0, rows * 16, 0x00027000);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void*)t.rows, 16, in_loop(lane) * 16, 0, 0, 0);
    }
  };
  ScoreFactors f;
  auto compute = [&](const QueryTile<D>& t, int tile) {
    const int group = tile * (kQueryTile / kRowGroup) + part;
    if (group * kRowGroup >= a.q_len) return;
    const GroupBound b = load_uniform(a.plan.groups + group);
    if (b.lo >= k0 + 32 || b.hi <= k0) return;
    const bool whole = b.all_lo <= k0 && b.all_hi >= k0 + 32 && (group + 1) * kRowGroup <= a.q_len;
    const unsigned char *tq = t.q + part * (kRowGroup * D * 2), *to = t.d_o + part * (kRowGroup * D * 2);
    const int at_row = in_loop(row_base), at_across = in_loop(across_base), r0 = part * kRowGroup + 4 * half;
    f32x16 s = {}, dp;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) s = mma(S::template row<T>(tq, at_row, 0, i), k[i], s);
#pragma unroll
    for (int r = 0; r < 4; ++r) {                // dP - delta
      const f32x4 x = *reinterpret_cast<const f32x4*>(&t.less[r0 + 8 * r]);
#pragma unroll
      for (int j = 0; j < 4; ++j) dp[4 * r + j] = x[j];
    }
#pragma unroll
    for (int i = 0; i < D / 16; ++i) dp = mma(S::template row<T>(to, at_row, 0, i), v[i], dp);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      __builtin_amdgcn_sched_barrier(0);      // (all of them at once would cost 16 registers)
      const f32x4 base = *reinterpret_cast<const f32x4*>(&t.base[r0 + 8 * r]);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int i = 4 * r + j;
        float back, d = 0.0f;
        if constexpr (BIAS) d = f.slope2 * fabsf((float)(t.rows[r0 + 8 * r + j].diag - key));
        const float x = shaped<CAP, BIAS>(s[i], f, d, &back);
        s[i] = fast_exp2(__builtin_fmaf(x, f.mul, base[j]));
        dp[i] *= s[i];
        if constexpr (CAP) dp[i] *= back;
      }
    }
    if (!whole) {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int2 rb = *reinterpret_cast<const int2*>(&t.rows[r0 + 8 * (i / 4) + i % 4]);   // lo, hi
        const bool sees = (key >= rb.x) & (key < rb.y);
        s[i] = sees ? s[i] : 0.0f;
        dp[i] = sees ? dp[i] : 0.0f;
      }
    }
    vec8<T> p[2];
    to_operand<T>(s, p);
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < D / 32; ++i) dv[i] = mma(S::template across<T>(to, at_across, 16 * u, i), p[u], dv[i]);
    to_operand<T>(dp, p);
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < D / 32; ++i) dk[i] = mma(S::template across<T>(tq, at_across, 16 * u, i), p[u], dk[i]);
  };

  // head by head, tile by tile, in pairs of buffers
  int head = kv * a.group, c = begin;
  const int last = head + a.group;
  auto step = [&](int* h, int* tile) {
    *tile = next_tile(flags, *tile + 1, end, 1);
    if (*tile >= end) { *tile = begin; ++*h; }
  };
  if (begin < end) {
    load(even, head, c);
    while (head < last) {
      int h2 = head, c2 = c;
      step(&h2, &c2);
      tiles_ready();
      if (h2 < last) load(odd, h2, c2);
      f = score_factors<CAP, BIAS>(a.score, head);
      compute(even, c);
      head = h2; c = c2;
      if (head >= last) break;
      step(&h2, &c2);
      tiles_ready();
      if (h2 < last) load(even, h2, c2);
      f = score_factors<CAP, BIAS>(a.score, head);
      compute(odd, c);
      head = h2; c = c2;
    }
  }

  // wave (keys, part 0) takes over the other's dK, wave (keys, part 1) its dV
  __syncthreads();
  f32x4* room = reinterpret_cast<f32x4*>((wave & 1) ? odd.q : even.q) + part * (D / 8 * kWave) + lane;
  static_assert(2 * (D / 8) * kWave * 16 <= 2 * kQueryTile * D * 2, "both waves' sums fit a buffer's queries and dO");
  const f32x4* other = reinterpret_cast<const f32x4*>((wave & 1) ? odd.q : even.q) + (1 - part) * (D / 8 * kWave) + lane;
#pragma unroll
  for (int i = 0; i < D / 32; ++i)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      f32x4 x;
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = part ? dk[i][4 * r + j] : dv[i][4 * r + j];
      room[(4 * i + r) * kWave] = x;
    }
  __syncthreads();
  if (!real) return;
  const RowSource to = (part ? g.dv : g.dk).of(kv);
  const float by = part ? 1.0f : CAP ? 4.0f * a.score.scale : a.score.scale;
  unsigned char* out = const_cast<unsigned char*>(to.base) + (int64_t)key * to.stride;
#pragma unroll
  for (int i = 0; i < D / 32; ++i)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int byte = (32 * i + 8 * r + 4 * half) * 2;
      const f32x4 x = other[(4 * i + r) * kWave];
      T y[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) y[j] = (T)(((part ? dv[i][4 * r + j] : dk[i][4 * r + j]) + x[j]) * by);
      if (byte < a.bytes) *reinterpret_cast<u32x2*>(out + byte) = __builtin_bit_cast(u32x2, y);
    }
}

}  // namespace spg
