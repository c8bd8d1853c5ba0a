// Attention over a planned mask, gradients.
//
// With P = 2^(x - lse2) (x: the shaped scores in units of log 2, lse2 the row's logarithm from the forward pass), dP = dO V^T and
// delta_i = sum_d dO_id O_id:  dV = P^T dO,  dS = P (dP - delta) (1 - tanh^2),  dQ = scale dS K,  dK = scale dS^T Q.
// k_attn_facts sums up what the rows' exponents begin with and -delta; after it workgroups of two kinds run in one launch, each with a fixed order of its
// sums (no atomics: the same inputs give the same bits): for dQ they go over the keys of 128 queries as the forward kernel does, for dK and dV over
// the queries, of all heads that share them, of 64 keys.  That computes S and dP twice, seven products where five would do with atomics on dQ in 32 bits.
// P, dS are rounded to 16 bits once, as operands; all sums are held in 32 bits.  In float16, whose smallest step is 2^-24, both are held 2^15 times as large, and
// dS less where a row (for dQ) or a key (for dK) would pass 2^15: so neither the length of the rows nor the size of dO costs digits (Lift).
//
// Measured (bfloat16, 128 channels, capped): two documents of 8192 tokens together, 16 heads on 8, 639 us, 0.76 PFLOP/s for the seven products (call after call without a trace 567 with the rows' sums; vector instructions issue in
// 55 % of the cycles, matrix instructions run in 42 %, LDS in 24 %: as the forward kernel); eleven documents of 4096 tokens, 16 heads on 4, 80 us and 5.2 to join, where two launches, one after
// the other, took 126 and 8.6: the long chains of one kind fill the places that the other leaves.
#pragma once
#include "attn_forward.hpp"
#include "attn_plan_kernels.hpp"

namespace spg {

// What an operand made of P is multiplied by: P is at most 1, so 2^15 times P fits float16, and probabilities down to 2^-29 keep all digits.  bfloat16
// has float's exponents.
template <typename T> constexpr bool kLifted = std::is_same<T, f16_t>::value;
template <typename T> constexpr float kLift = kLifted<T> ? 15.0f : 0.0f;   // in units of log 2
constexpr float kLiftMost = 32768.0f;

// dS of a lane's row (key) goes to sums that are in units of 2^-15 / lower, lower a power of two.  Where an entry would pass 2^15, entries, sums and `lower` go down
// so far that the largest is below it; never up again, so that what the sums hold is exact.  Both halves of a wave have the same row (key).  us without | with: 2003 tokens,
// 8 heads of 64 channels 23.6 | 25, 8192 tokens, 16 heads on 8 of 128, capped, 650 | 666.
// What comes later is lowered through `base`, which is added to its exponents, where there is one.
template <int N>
__device__ __forceinline__ void lift_step(f32x16& ds, f32x16* sums, float& lower, float* base) {
  float top = fabsf(ds[0]);
#pragma unroll
  for (int i = 1; i < 15; i += 2) top = max3(top, fabsf(ds[i]), fabsf(ds[i + 1]));
  top = max_halves(fmaxf(top, fabsf(ds[15])));
  if (__any(top >= kLiftMost)) {
    const int down = top >= kLiftMost ? (int)(__float_as_uint(top) >> 23) - 127 - 14 : 0;
    const float by = __uint_as_float((unsigned)(127 - down) << 23);
    lower *= by;
    if (base) *base -= (float)down;
    ds *= by;
#pragma unroll
    for (int i = 0; i < N; ++i) sums[i] *= by;
  }
}

// The work of n tiles as a list, most first, by one workgroup of 256 threads; up to 256 tiles are cut into pieces where there are places for them.  More
// are not, whatever the places: with one key head their chains are then the time.  counts: the list's length, and how many of its entries belong to cut tiles: they come first.
template <typename F, typename W>
__device__ __forceinline__ void list_work(int n, F reach, W tiles, unsigned long long total, const AttnGrads& g, int4* list, int* counts) {
  if (n > 256) {
    order_by_work(n, reach, list);
    if (threadIdx.x == 0) { counts[0] = n; counts[1] = 0; }
    return;
  }
  __shared__ int2 of[256];                       // tiles, pieces
  const int i = threadIdx.x;
  const int2 r = i < n ? reach(i) : make_int2(0, 0);
  const int mine = tiles(r), cut = i < n && g.slots ? pieces_of(mine, g.slots, total) : 1;
  of[i] = i < n ? make_int2(mine, cut) : make_int2(0, 0);
  __syncthreads();
  int place = 0, all = 0, front = 0;
#pragma unroll 16
  for (int k = 0; k < ceil_div_d(n, 16) * 16; ++k) {
    const int2 x = of[k];
    place += (x.x > mine) | ((x.x == mine) & (k < i)) ? x.y : 0;
    all += x.y;
    front += x.y > 1 ? x.y : 0;
  }
  if (i < n)
    for (int p = 0; p < cut && place + p < n + g.more; ++p) list[place + p] = make_int4(i, r.x, r.y, cut + 65536 * p);
  if (i == 0) { counts[0] = min(all, n + g.more); counts[1] = min(front, n + g.more); }
}

// A workgroup has 64 rows of a head: D / 8 lanes a row, 16 bytes of O and dO each.  The first two make the lists of work meanwhile.
// Memory bounds it: 8192 tokens, 16 heads of 128 channels 14.8 us, 4.5 TB/s; 4096 tokens, with lists of cut work, 9.3.
template <typename T, int D>
__global__ void __launch_bounds__(256) k_attn_facts(AttnArgs a, AttnGrads g) {
  constexpr int kLanes = D / 8, kStep = 256 / kLanes;
  if (blockIdx.x < 2) {
    if (blockIdx.y > 0) return;
    const unsigned long long total = (load_uniform(a.plan.totals) + load_uniform(a.plan.totals + 1)) * a.heads;
    if (blockIdx.x == 0)
      list_work(ceil_div_d(a.k_len, kKeyTile), [&](int i) { return a.plan.cols[i]; }, [&](int2 r) { return (int)query_tiles(r) * a.group; }, total, g, g.k_list, &g.counts->keys);
    else
      list_work(a.q_tiles, [&](int i) { return query_tile_reach(a.plan, a.q_len, i); }, [](int2 r) { return (int)key_tiles(r); }, total, g, g.q_list, &g.counts->queries);
    return;
  }
  const int n = blockIdx.x - 2, head = blockIdx.y, chunk = threadIdx.x % kLanes, mine = threadIdx.x / kLanes;
  const HeadTensor &o = a.o, &d_o = g.d_o;
  __shared__ float deltas[kQueryTile];
  u32x4 x[kQueryTile / kStep], y[kQueryTile / kStep];
#pragma unroll
  for (int i = 0; i < kQueryTile / kStep; ++i) {
    const int64_t row = (int64_t)n * kQueryTile + i * kStep + mine;
    x[i] = y[i] = u32x4{0, 0, 0, 0};
    if (row < a.q_len && chunk * 16 < a.bytes) {
      x[i] = *reinterpret_cast<const u32x4*>(o.of(head).base + row * o.stride + chunk * 16);
      y[i] = *reinterpret_cast<const u32x4*>(d_o.of(head).base + row * d_o.stride + chunk * 16);
    }
  }
#pragma unroll
  for (int i = 0; i < kQueryTile / kStep; ++i) {
    const vec8<T> u = __builtin_bit_cast(vec8<T>, x[i]), v = __builtin_bit_cast(vec8<T>, y[i]);
    float sum = 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j) sum = __builtin_fmaf((float)u[j], (float)v[j], sum);
#pragma unroll
    for (int d = 1; d < kLanes; d *= 2) sum += __shfl_xor(sum, d);
    if (chunk == 0) deltas[i * kStep + mine] = sum;
  }
  __syncthreads();
  if (threadIdx.x >= kQueryTile) return;
  const int i = threadIdx.x, row = n * kQueryTile + i;
  const bool real = row < a.q_len;
  const RowBound rb = real ? a.plan.rows[row] : RowBound{0, 0, 0, 0};
  const float lse = real ? a.lse[(int64_t)head * a.q_len + row] : -INFINITY;
  RowFacts& facts = g.facts[(int64_t)head * a.q_tiles * (kPatTile / kQueryTile) + n];
  facts.base[i] = lse == -INFINITY ? -INFINITY : (a.score.cap > 0.0f && !a.score.slopes ? a.score.cap * kLog2e : 0.0f) - lse * kLog2e + kLift<T>;   // (a row that sees nothing: every power is 0)
  facts.less[i] = -deltas[i];
  facts.lo[i] = rb.lo;
  facts.hi[i] = rb.hi;
  facts.diag[i] = rb.diag;
}

// k_attn_back's arguments, read where they are wanted: the compiler loads all arguments of a kernel at its begin, and with those of both kinds of work the scalar
// registers did not do (70 of them kept in lanes of vector registers; 8192 tokens 682 -> 647 us).
struct BackArgs { AttnArgs a; AttnGrads g; };
__device__ __forceinline__ BackArgs back_args() {
  typedef const __attribute__((address_space(4))) BackArgs Memory;
  Memory* p = (Memory*)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  return *(const BackArgs*)p;
}

template <typename T, int D, bool CAP, bool BIAS>
__device__ __forceinline__ void dq_tile(unsigned char* lds, int n) {
  const BackArgs args = back_args();
  const AttnArgs& a = args.a;
  const AttnGrads& g = args.g;
  using S = TileShape<D>;
  constexpr int kTile = kKeyTile * D * 2;
  unsigned char *k_even = lds, *v_even = lds + kTile, *k_odd = lds + 2 * kTile, *v_odd = lds + 3 * kTile;
  const Place at = place_of(n, a.heads, g.q_list);
  const int head = at.head, qt = at.tile, lo = at.lo, hi = at.hi;
  const int lane = lane_id(), half = lane >> 5, wave = uniform(threadIdx.x / kWave);
  const int row_base = S::row_base(lane), across_base = S::across_base(lane);
  const int row = qt * kPatTile + wave * kRowGroup + (lane & 31);
  const GroupBound mine = wave_bound(a, qt, wave);
  const int begin = lo / kKeyTile;
  const Share share = share_of(ceil_div_d(hi, kKeyTile) - begin, at.piece & 0xffff, at.piece >> 16);
  const ScoreFactors f = score_factors<CAP, BIAS>(a.score, head);
  const bool real = row < a.q_len;
  const RowBound rb = real ? a.plan.rows[row] : RowBound{0, 0, 0, 0};
  const RowFacts& facts = g.facts[((int64_t)head * a.q_tiles + qt) * (kPatTile / kQueryTile) + wave / 2];
  float base = facts.base[row % kQueryTile], lower = 1.0f;
  const float less = facts.less[row % kQueryTile];
  vec8<T> q[D / 16], d_o[D / 16];
  load_row<T, D>(a.q.of(head), row, real, a.bytes, half, q);
  load_row<T, D>(g.d_o.of(head), row, real, a.bytes, half, d_o);
  const int kv = uniform(head / a.group);
  const RowSource ks = a.k.of(kv), vs = a.v.of(kv);
  const TileLoader<D, kKeyTile, 256> load_k(ks.stride, lane), load_v(vs.stride, lane);
  f32x16 acc[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) acc[i] = f32x16{};

  const unsigned* flags = a.plan.seen_words ? a.plan.seen + (int64_t)qt * a.plan.seen_words : nullptr;
  const int end = begin + share.last;

  auto compute = [&](const unsigned char* kt, const unsigned char* vt, int k0) {
    if (mine.lo >= k0 + kKeyTile || mine.hi <= k0) return;
    const bool whole = mine.all_lo <= k0 && mine.all_hi >= k0 + kKeyTile;
    const int at_row = in_loop(row_base), at_across = in_loop(across_base);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      f32x16 s = {}, dp = {};
#pragma unroll
      for (int i = 0; i < D / 16; ++i) {
        s = mma(S::template row<T>(kt, at_row, 32 * t, i), q[i], s);
        dp = mma(S::template row<T>(vt, at_row, 32 * t, i), d_o[i], dp);
      }
      const float away = (float)(rb.diag - k0 - 4 * half - 32 * t);
      const unsigned span = rb.hi > rb.lo ? rb.hi - rb.lo : 0;
      const int off = k0 + 4 * half + 32 * t - rb.lo;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        float back;
        const float x = shaped<CAP, BIAS>(s[i], f, f.slope2 * fabsf(away - (float)(8 * (i / 4) + i % 4)), &back);
        s[i] = fast_exp2(__builtin_fmaf(x, f.mul, base)) * (dp[i] + less);
        if constexpr (CAP) s[i] *= back;
      }
      if (!whole) {
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = (unsigned)(off + 8 * (i / 4) + i % 4) < span ? s[i] : 0.0f;
      }
      if constexpr (kLifted<T>) lift_step<D / 32>(s, acc, lower, &base);
      vec8<T> p[2];
      to_operand<T>(s, p);
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < D / 32; ++i) acc[i] = mma(S::template across<T>(kt, at_across, 32 * t + 16 * u, i), p[u], acc[i]);
    }
  };
  auto load = [&](unsigned char* kt, unsigned char* vt, int k0) {
    load_tiles(load_k, ks.base, kt, load_v, vs.base, vt, k0, lo, hi, a.bytes);
  };

  int c = next_tile(flags, begin + share.first, end);
  if (c < end) load(k_even, v_even, c * kKeyTile);
  while (c < end) {
    int next = next_tile(flags, c + 1, end);
    tiles_ready();
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

  if constexpr (kLifted<T>) {
#pragma unroll
    for (int i = 0; i < D / 32; ++i) acc[i] *= 1.0f / (kLiftMost * lower);
  }
  const BackArgs end_args = back_args();
  if (share.pieces > 1) leave_sums<D>(end_args.g.sums, load_uniform(&end_args.g.counts->cut_keys) * (end_args.a.heads / end_args.a.group) + n, acc);
  else if (row < end_args.a.q_len) store_rows<T, D>(end_args.g.dq, head, row, half, 0, end_args.a.bytes, acc, (CAP ? 4.0f : 1.0f) * end_args.a.score.scale);
}

// A workgroup has 64 keys of a key head and goes over their queries in tiles of 64 rows, head by head.  Wave w has keys 32 (w % 2) .. and of every
// tile the rows 32 (w / 2) ..; keys and values stay in registers as right operands, queries and dO come through LDS with what their exponents and dP
// begin with and their bounds, one tile ahead.  At the end the two waves of the same keys exchange sums: one adds up dK, the other dV.
template <int D>
struct QueryTile {
  unsigned char q[kQueryTile * D * 2], d_o[kQueryTile * D * 2];
  RowFacts facts;
};

template <typename T, int D, bool CAP, bool BIAS>
__device__ __forceinline__ void dkv_tile(unsigned char* lds, int n) {
  const BackArgs args = back_args();
  const AttnArgs& a = args.a;
  const AttnGrads& g = args.g;
  using S = TileShape<D>;
  QueryTile<D>&even = reinterpret_cast<QueryTile<D>*>(lds)[0], &odd = reinterpret_cast<QueryTile<D>*>(lds)[1];
  const Place at = place_of(n, a.heads / a.group, g.k_list);
  const int kv = at.head, kt = at.tile, lo = at.lo, hi = at.hi;
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

  const unsigned* flags = a.plan.seen_by_words ? a.plan.seen_by + (int64_t)(kt * kKeyTile / kPatTile) * a.plan.seen_by_words : nullptr;
  const int low = hi > lo ? lo / kQueryTile : 0, end = hi > lo ? ceil_div_d(hi, kQueryTile) : 0, tiles = end - low;
  const int begin = next_tile(flags, low, end);
  // the work is a list: all tiles of one head, then of the next
  const Share share = share_of(tiles * a.group, at.piece & 0xffff, at.piece >> 16);

  auto load = [&](QueryTile<D>& t, int head, int tile) {
    const int first = tile * kQueryTile;
    const TileLoader<D, kQueryTile, 256> load_q(a.q.stride, in_loop(lane)), load_do(g.d_o.stride, in_loop(lane));   // (made anew: registers are short)
    load_tiles(load_q, a.q.of(head).base, t.q, load_do, g.d_o.of(head).base, t.d_o, first, lo, hi, a.bytes);
    const RowFacts* from = g.facts + (int64_t)head * a.q_tiles * (kPatTile / kQueryTile) + tile;
    const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc((void*)from, 0, sizeof(RowFacts), 0x00027000);
    if (wave == 0) __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void*)&t.facts, 16, in_loop(lane) * 16, 0, 0, 0);
    if (BIAS && wave == 1) __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void*)t.facts.diag, 4, in_loop(lane) * 4 + 1024, 0, 0, 0);
  };
  static_assert(sizeof(RowFacts) == 5 * 256 && offsetof(RowFacts, diag) == 1024, "one load of 16 bytes a lane for all but the diagonals");
  const int groups = ceil_div_d(a.q_len, kRowGroup);
  // bounds of the rows that this wave has of a tile
  auto bounds = [&](int tile) {
    const int group = tile * (kQueryTile / kRowGroup) + part;
    return group < groups ? load_uniform(a.plan.groups + group) : GroupBound{0, 0, 0, 0};
  };
  ScoreFactors f = score_factors<CAP, BIAS>(a.score, kv * a.group);
  float lower = 1.0f;
  auto compute = [&](const QueryTile<D>& t, const GroupBound& b) {
    if ((b.lo >= k0 + 32) | (b.hi <= k0)) return;
    const bool whole = (b.all_lo <= k0) & (b.all_hi >= k0 + 32);
    const unsigned char *tq = t.q + part * (kRowGroup * D * 2), *to = t.d_o + part * (kRowGroup * D * 2);
    const int at_row = in_loop(row_base), at_across = in_loop(across_base), r0 = part * kRowGroup + 4 * half;
    f32x16 s = {}, dp;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) s = mma(S::template row<T>(tq, at_row, 0, i), k[i], s);
#pragma unroll
    for (int r = 0; r < 4; ++r) {                // dP - delta
      const f32x4 x = *reinterpret_cast<const f32x4*>(&t.facts.less[r0 + 8 * r]);
#pragma unroll
      for (int j = 0; j < 4; ++j) dp[4 * r + j] = x[j];
    }
#pragma unroll
    for (int i = 0; i < D / 16; ++i) dp = mma(S::template row<T>(to, at_row, 0, i), v[i], dp);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      __builtin_amdgcn_sched_barrier(0);      // (all of them at once would cost 16 registers)
      const f32x4 base = *reinterpret_cast<const f32x4*>(&t.facts.base[r0 + 8 * r]);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int i = 4 * r + j;
        float back, d = 0.0f;
        if constexpr (BIAS) d = f.slope2 * fabsf((float)(t.facts.diag[r0 + 8 * r + j] - key));
        const float x = shaped<CAP, BIAS>(s[i], f, d, &back);
        s[i] = fast_exp2(__builtin_fmaf(x, f.mul, base[j]));
        dp[i] *= s[i];
        if constexpr (CAP) dp[i] *= back;
      }
    }
    if (!whole) {
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        typedef int i32x4 __attribute__((ext_vector_type(4)));
        const i32x4 from = *reinterpret_cast<const i32x4*>(&t.facts.lo[r0 + 8 * r]), until = *reinterpret_cast<const i32x4*>(&t.facts.hi[r0 + 8 * r]);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const bool sees = (key >= from[j]) & (key < until[j]);
          s[4 * r + j] = sees ? s[4 * r + j] : 0.0f;
          dp[4 * r + j] = sees ? dp[4 * r + j] : 0.0f;
        }
      }
    }
    vec8<T> p[2];
    to_operand<T>(s, p);
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < D / 32; ++i) dv[i] = mma(S::template across<T>(to, at_across, 16 * u, i), p[u], dv[i]);
    if constexpr (kLifted<T>) {
      dp *= lower;                              // (a branch around it where lower is 1 costs 40 scalar registers)
      lift_step<D / 32>(dp, dk, lower, nullptr);
    }
    to_operand<T>(dp, p);
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < D / 32; ++i) dk[i] = mma(S::template across<T>(tq, at_across, 16 * u, i), p[u], dk[i]);
  };

  // head by head, tile by tile, in pairs of buffers
  const int head0 = kv * a.group;
  auto place = [&](int h, int tile) { return (h - head0) * tiles + tile - low; };
  auto settle = [&](int* h, int* tile) {              // the next tile that the pattern holds, of this head or the next one
    *tile = next_tile(flags, *tile, end);
    if (*tile >= end) { *tile = begin; ++*h; }
  };
  if (begin < end && share.first < share.last) {
    int head = uniform(head0 + share.first / tiles), c = uniform(low + share.first % tiles);
    settle(&head, &c);
    bool more = place(head, c) < share.last;
    if (more) load(even, head, c);
    GroupBound here = bounds(c), there{0, 0, 0, 0};
    auto next_one = [&](QueryTile<D>& t) {            // begins the next tile's loads; its bounds are there when its turn comes
      int h2 = head, c2 = c + 1;
      settle(&h2, &c2);
      more = place(h2, c2) < share.last;
      tiles_ready();
      if (more) {
        load(t, h2, c2);
        there = bounds(c2);
      }
      if constexpr (BIAS) f.slope2 = load_uniform(a.score.slopes + head) * kLog2e;
      head = h2;
      c = c2;
    };
    while (more) {
      next_one(odd);
      compute(even, here);
      here = there;
      if (!more) break;
      next_one(even);
      compute(odd, here);
      here = there;
    }
  }

  // wave (keys, part 0) takes over the other's dK, wave (keys, part 1) its dV
  if constexpr (kLifted<T>) {
#pragma unroll
    for (int i = 0; i < D / 32; ++i) { dk[i] *= 1.0f / (kLiftMost * lower); dv[i] *= 1.0f / kLiftMost; }
  }
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
  f32x16 sum[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const f32x4 x = other[(4 * i + r) * kWave];
#pragma unroll
      for (int j = 0; j < 4; ++j) sum[i][4 * r + j] = (part ? dv[i][4 * r + j] : dk[i][4 * r + j]) + x[j];
    }
  const BackArgs end_args = back_args();
  if (share.pieces > 1) leave_sums<D>(end_args.g.sums, n, sum);
  else if (key < end_args.a.k_len)
    store_rows<T, D>(part ? end_args.g.dv : end_args.g.dk, kv, key, half, 0, end_args.a.bytes, sum, part ? 1.0f : (CAP ? 4.0f : 1.0f) * end_args.a.score.scale);
}

// Keys' workgroups come first, for their chains are the longer ones.  How many there are only the lists know: the last ones have nothing.
template <typename T, int D, bool CAP, bool BIAS>
__global__ void __launch_bounds__(256, 2) k_attn_back(BackArgs) {
  static_assert(sizeof(QueryTile<D>) >= 2 * kKeyTile * D * 2, "both kinds fit");
  __shared__ __align__(16) unsigned char lds[2 * sizeof(QueryTile<D>)];
  const BackArgs args = back_args();
  const Counts c = load_uniform(args.g.counts);
  const int n = blockIdx.x, keys = uniform(c.keys * (args.a.heads / args.a.group)), queries = uniform(c.queries * args.a.heads);
  if (n < keys) dkv_tile<T, D, CAP, BIAS>(lds, n);
  else if (n - keys < queries) dq_tile<T, D, CAP, BIAS>(lds, n - keys);
}

// A workgroup has 32 channels of a tile's rows (keys).
template <typename T, int D, bool CAP>
__global__ void __launch_bounds__(256) k_attn_back_join(AttnArgs a, AttnGrads g) {
  const Counts c = load_uniform(g.counts);
  const int kv_heads = a.heads / a.group, keys = c.cut_keys * kv_heads, n = blockIdx.x;
  if (n >= keys + c.cut_queries * a.heads) return;
  const bool of_keys = n < keys;
  const int heads = of_keys ? kv_heads : a.heads;
  const Place at = place_of(of_keys ? n : n - keys, heads, of_keys ? g.k_list : g.q_list);
  if (at.piece >> 16) return;
  const int c0 = blockIdx.y * 32, lane = lane_id(), wave = uniform(threadIdx.x / kWave);
  const float by = CAP ? 4.0f * a.score.scale : a.score.scale;
  f32x16 sum = {};
#pragma unroll 4
  for (int p = 0; p < (at.piece & 0xffff); ++p) add_sums<D>(g.sums, n + (int64_t)p * heads, c0, 1.0f, sum);   // (a head's next piece is so many places on)
  if (of_keys) {
    const int part = wave >> 1, key = at.tile * kKeyTile + (wave & 1) * 32 + (lane & 31);
    if (key < a.k_len) store_rows<T, 32>(part ? g.dv : g.dk, at.head, key, lane >> 5, c0, a.bytes, &sum, part ? 1.0f : by);
  } else {
    const int row = at.tile * kPatTile + wave * kRowGroup + (lane & 31);
    if (row < a.q_len) store_rows<T, 32>(g.dq, at.head, row, lane >> 5, c0, a.bytes, &sum, by);
  }
}

}  // namespace spg
