// Attention over a paged cache held in 8 bits, and what fills the cache.
//
// A page holds 64 tokens of one sequence, in e4m3 with a scale (a power of two) for each page and key head: keys as [token][channel], values as
// [channel][token], which is how the two products read them: both as left operands, 8 neighbouring bytes along the contraction.  A
// wave has 16 query rows (the heads that share a key head, for every new token) as right operands and takes a page in four
// products of 16 keys; row 4g + i of product t is key 16 g + 4 t + i, so that the lanes with quarter g of the probabilities have
// the 16 neighbouring keys whose 16 bytes of a value's channel are one load, and nothing moves between lanes.  Pages go from memory to registers.
#pragma once
#include "attn_forward.hpp"
#include "page_need.hpp"

namespace spg {

constexpr int kRows = 16;             // query rows of a workgroup
constexpr float kMost8 = 448.0f;      // the largest e4m3 value

struct CacheView {        // one layer
  unsigned char *k, *v;   // [pages][heads][64][room], [pages][heads][room][64]
  float *k_scale, *v_scale;   // [pages][heads]
  int64_t pages;
  int heads, bytes8;      // key heads; channels of a head, a multiple of 8
};

struct TableView {        // pages of sequence s: page[ptr[s]] .. page[ptr[s + 1] - 1]
  const int64_t* ptr;
  const int32_t* page;
  const int32_t* lens;    // tokens of each sequence
  int seqs;
  int64_t nnz;
};

// The last s with base(s) <= slot, base ascending; 0 where there is none.  By the whole wave: 64 places are looked at together, so that a table of 4096
// sequences takes two dependent loads, not twelve.
template <typename F>
__device__ __forceinline__ int find_seq(int seqs, int64_t slot, F base) {
  const int n = wave_count_below(seqs, slot + 1, base);
  return n > 0 ? n - 1 : 0;
}

// ---- append -----------------------------------------------------------------------------------

struct AppendArgs {
  CacheView c;
  TableView t;
  const int64_t* new_ptr;   // tokens new_ptr[s] .. new_ptr[s + 1] - 1 of k and v are the last ones of sequence s
  HeadTensor k, v;
  int64_t tokens;
};

// 2^e with the least e for which most * 2^-e <= 448 = 1.75 * 2^8.
__device__ __forceinline__ float scale_for(float most) {
  const unsigned u = __float_as_uint(most);
  int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffff) > 0x600000 ? 1 : 0);
  e = most == 0.0f || e < -100 ? -100 : e > 120 ? 120 : e;
  return __uint_as_float((unsigned)(e + 127) << 23);
}

// To 8 bits, nearest, ties to even; beyond the largest value the largest; NaN stays NaN.
__device__ __forceinline__ unsigned to8(float a, float b, float c, float d) {
  auto fit = [](float x) { return x != x ? x : fminf(fmaxf(x, -kMost8), kMost8); };
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(fit(a), fit(b), 0, false);
  return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(fit(c), fit(d), w, true);
}
__device__ __forceinline__ unsigned rescale8(unsigned w, float by) {
  return to8(__builtin_amdgcn_cvt_f32_fp8(w, 0) * by, __builtin_amdgcn_cvt_f32_fp8(w, 1) * by, __builtin_amdgcn_cvt_f32_fp8(w, 2) * by,
             __builtin_amdgcn_cvt_f32_fp8(w, 3) * by);
}

// A workgroup has a page that new tokens fall into, and a head.  How many pages those are the host does not know: sequence s has places
// new_ptr[s] / 64 + 2 s and on, which hold the pages that new_ptr[s + 1] - new_ptr[s] tokens can touch, and those that it does not need end at once.
// Rows are read twice, first for the scale, which the caches hold; values are turned in LDS, so that a channel's tokens are written as words.  A prompt of 32 768 tokens, 8 heads of
// 128 channels: 54 us, 3.7 TB/s read and written; 4096 tokens 12.3 us; one token of a sequence 5.3 us, of 128 sequences 10: a chain of dependent loads (table, page, scale).
template <typename T, int R>
__global__ void __launch_bounds__(256) k_cache_append(AppendArgs a) {
  const int head = blockIdx.y, tid = threadIdx.x;
  const int64_t slot = blockIdx.x;
  auto begin_of = [&](int s) { const int64_t v = a.new_ptr[s]; return v < 0 ? 0 : v > a.tokens ? a.tokens : v; };
  const int s = find_seq(a.t.seqs, slot, [&](int i) { return begin_of(i) / kPage + 2 * (int64_t)i; });
  const int64_t first = begin_of(s), count = begin_of(s + 1) - first;
  const int64_t len = a.t.lens[s], start = len - count;
  if (count <= 0 || start < 0) return;
  const int64_t n = start / kPage + (slot - (first / kPage + 2 * (int64_t)s));      // the page's place in the sequence
  if (n < start / kPage || n * kPage >= len) return;
  const int64_t at = a.t.ptr[s] + n;
  if (at < 0 || at >= a.t.ptr[s + 1] || at >= a.t.nnz) return;
  const int64_t page = a.t.page[at];
  if (page < 0 || page >= a.c.pages) return;
  const int from = start > n * kPage ? (int)(start - n * kPage) : 0;                // new tokens of the page: from .. to - 1
  const int to = len < (n + 1) * kPage ? (int)(len - n * kPage) : kPage;
  const int64_t token0 = first + (n * kPage + from - start);                        // ... the first of them
  const int64_t ph = page * a.c.heads + head;
  const RowSource ks = a.k.of(head), vs = a.v.of(head);
  constexpr int kChunks = R / 8;

  __shared__ float tops[2][4];
  __shared__ __align__(16) unsigned char fresh[R][kPage + 4];                       // new values by channel and token
  float top[2] = {0.0f, 0.0f};
  auto fetch = [&](const RowSource& src, int o, int chunk) {
    vec8<T> x = {};
    if (chunk * 8 < a.c.bytes8) x = *reinterpret_cast<const vec8<T>*>(src.base + (token0 + o - from) * src.stride + chunk * 16);
    return x;
  };
  for (int i = tid; i < (to - from) * kChunks; i += 256) {
    const vec8<T> x = fetch(ks, from + i / kChunks, i % kChunks), y = fetch(vs, from + i / kChunks, i % kChunks);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float p = fabsf((float)x[j]), q = fabsf((float)y[j]);
      top[0] = p < INFINITY ? fmaxf(top[0], p) : top[0];
      top[1] = q < INFINITY ? fmaxf(top[1], q) : top[1];
    }
  }
#pragma unroll
  for (int j = 0; j < 2; ++j) {
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) top[j] = fmaxf(top[j], __shfl_xor(top[j], d));
    if (lane_id() == 0) tops[j][tid / kWave] = top[j];
  }
  __syncthreads();
  float scale[2], by[2];
  bool grows[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const float need = scale_for(fmaxf(fmaxf(tops[j][0], tops[j][1]), fmaxf(tops[j][2], tops[j][3])));
    const float old = from ? (j ? a.c.v_scale : a.c.k_scale)[ph] : 0.0f;
    scale[j] = fmaxf(old, need);
    grows[j] = from && need > old;
    by[j] = old / scale[j];
  }
  __syncthreads();                                                                  // (everybody has the old scales)
  if (tid == 0) { a.c.k_scale[ph] = scale[0]; a.c.v_scale[ph] = scale[1]; }

  unsigned char* kp = a.c.k + ph * (kPage * R);
  unsigned char* vp = a.c.v + ph * (kPage * R);
  if (grows[0])
    for (int i = tid; i < from * R / 4; i += 256) reinterpret_cast<unsigned*>(kp)[i] = rescale8(reinterpret_cast<unsigned*>(kp)[i], by[0]);
  const float inv[2] = {1.0f / scale[0], 1.0f / scale[1]};                          // (powers of two: exact)
  for (int i = tid; i < (to - from) * kChunks; i += 256) {
    const int o = from + i / kChunks, chunk = i % kChunks;
    const vec8<T> x = fetch(ks, o, chunk), y = fetch(vs, o, chunk);
    float f[8], e[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) { f[j] = (float)x[j] * inv[0]; e[j] = (float)y[j] * inv[1]; }
    u32x2 w = {to8(f[0], f[1], f[2], f[3]), to8(f[4], f[5], f[6], f[7])};
    *reinterpret_cast<u32x2*>(kp + o * R + chunk * 8) = w;
    w = u32x2{to8(e[0], e[1], e[2], e[3]), to8(e[4], e[5], e[6], e[7])};
#pragma unroll
    for (int j = 0; j < 8; ++j) fresh[chunk * 8 + j][o] = (unsigned char)(w[j / 4] >> (8 * (j % 4)));
  }
  __syncthreads();
  // values: words of four tokens of a channel; the tokens before are kept (rounded again where the scale has grown), and so is what lies behind
  const int w0 = grows[1] ? 0 : from / 4, words = (to + 3) / 4 - w0;
  for (int i = tid; i < words * R; i += 256) {
    const int d = i / words, o = (w0 + i % words) * 4;
    unsigned* p = reinterpret_cast<unsigned*>(vp + d * kPage + o);
    unsigned old = 0, keep = 0;
    if (o < from || o + 4 > to) {
      old = *p;
      unsigned before = 0, behind = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        before |= o + j < from ? 0xffu << (8 * j) : 0u;
        behind |= o + j >= to ? 0xffu << (8 * j) : 0u;
      }
      keep = before | behind;
      if (grows[1]) old = (rescale8(old, by[1]) & before) | (old & behind);
    }
    const unsigned now = *reinterpret_cast<const unsigned*>(&fresh[d][o]);
    *p = (now & ~keep) | (old & keep);
  }
}

// ---- attend -----------------------------------------------------------------------------------

struct AttendArgs {
  CacheView c;
  TableView t;
  HeadTensor q, o;          // row i of sequence s: token s * q_len + i
  int q_len, heads, group, tiles, window;
  int chunk;                // pages of a workgroup
  ScoreShape score;
  float* part;              // [slots][key heads][tiles][16 rows][R]: sums of what the workgroups saw, not divided
  float2* part_ml;          // [slots][key heads][tiles][16 rows]: maximum (units of log 2) and sum
};

// Sequence s: its tokens, and the pages first .. last - 1 that its queries see.
struct SeqPages { int64_t at; int len, lo, first, last; };
__device__ __forceinline__ int64_t first_page(const AttendArgs& a, int s) {
  const int64_t b = a.t.ptr[s];
  return b < 0 ? 0 : b > a.t.nnz ? a.t.nnz : b;
}
__device__ __forceinline__ SeqPages seq_pages(const AttendArgs& a, int s) {
  const int64_t b = first_page(a, s);
  int64_t e = first_page(a, s + 1);
  e = e < b ? b : e;
  const int64_t most = (e - b) * kPage;
  const int64_t len = a.t.lens[s];
  SeqPages r;
  r.at = b;
  r.len = len < 0 ? 0 : (int)(len < most ? len : most);
  r.lo = a.window && r.len - a.q_len - a.window + 1 > 0 ? r.len - a.q_len - a.window + 1 : 0;
  r.first = r.lo / kPage;
  r.last = ceil_div_d(r.len, kPage);
  return r;
}

__device__ __forceinline__ vec8<bf16_t> widen(u32x2 w, bf16_t) {
  typedef bf16_t pair __attribute__((ext_vector_type(2)));
  union { pair p[4]; vec8<bf16_t> v; } u;
  u.p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[0], 1.0f, false);
  u.p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[0], 1.0f, true);
  u.p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[1], 1.0f, false);
  u.p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[1], 1.0f, true);
  return u.v;
}
__device__ __forceinline__ vec8<f16_t> widen(u32x2 w, f16_t) {
  typedef f16_t pair __attribute__((ext_vector_type(2)));
  union { pair p[4]; vec8<f16_t> v; } u;
  u.p[0] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[0], 1.0f, false);
  u.p[1] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[0], 1.0f, true);
  u.p[2] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[1], 1.0f, false);
  u.p[3] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[1], 1.0f, true);
  return u.v;
}

__device__ __forceinline__ float max_quarters(float v) {
  v = max_halves(v);
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float add_quarters(float v) {
  v = add_halves(v);
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// A workgroup has `chunk` pages of a sequence, a key head and 16 query rows; its four waves take the pages in turn and are joined in LDS.
// Places of chunks: sequence s has ptr[s] / chunk + s and on (as many as its pages can need, found without knowing the lengths on the host).
// Memory bounds it: four sequences of 100 000 to 131 071 tokens, 32 heads on 8 of 128 channels 175 us, 5.5 TB/s (a copy reaches 4.9); 128 sequences of 3 to 8192 tokens 46 us where a
// last-level cache holds a part of them, 4.0 TB/s and up without; one of 2001 tokens 7.6 us, of which most is the chain to the first page.
template <typename T, int R, bool CAP, bool BIAS>
__global__ void __launch_bounds__(256, R == 128 ? 3 : 4) k_cache_attend(AttendArgs a) {
  constexpr int kSteps = R / 32, kOut = R / 16, kLoads = R / 64;
  const int64_t slot = blockIdx.x;
  const int kv = blockIdx.y, tile = blockIdx.z;
  const int lane = lane_id(), quarter = lane >> 4, col = lane & 15, wave = uniform(threadIdx.x / kWave);
  const int s = uniform(find_seq(a.t.seqs, slot, [&](int i) { return first_page(a, i) / a.chunk + i; }));
  const SeqPages sp = seq_pages(a, s);
  const int64_t piece = slot - (sp.at / a.chunk + s);
  if (piece < 0 || piece * a.chunk >= sp.last) return;
  const int begin = uniform(max(sp.first, (int)piece * a.chunk)), end = uniform(min(sp.last, (int)(piece + 1) * a.chunk));
  if (begin >= end) return;
  const bool alone = sp.first / a.chunk == (sp.last - 1) / a.chunk;    // nothing to join with

  const int r = tile * kRows + col, token = r / a.group, head = kv * a.group + r % a.group;
  const bool real = token < a.q_len;
  const int diag = sp.len - a.q_len + token;
  vec8<T> q[kSteps];
  {
    const RowSource src = a.q.of(real ? head : 0);
    const unsigned char* p = src.base + ((int64_t)s * a.q_len + (real ? token : 0)) * src.stride;
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      const int d = (R / 4) * quarter + 8 * i;
      u32x4 w = {0, 0, 0, 0};
      if (real && d < a.c.bytes8) w = *reinterpret_cast<const u32x4*>(p + d * 2);
      q[i] = __builtin_bit_cast(vec8<T>, w);
    }
  }
  const float scale2 = CAP ? a.score.scale / a.score.cap * (2.0f * kLog2e) : a.score.scale * kLog2e, cap2 = a.score.cap * kLog2e;
  const float slope2 = BIAS && real ? a.score.slopes[head] * kLog2e : 0.0f;
  // which keys of a page the lane's row sees: lo <= key <= diag
  const int row_lo = a.window ? diag - a.window + 1 : 0;
  const int first_diag = sp.len - a.q_len + (tile * kRows) / a.group;            // of the tile's first row: the least
  int last_token = (tile * kRows + kRows - 1) / a.group;
  last_token = last_token < a.q_len ? last_token : a.q_len - 1;
  const int last_lo = a.window ? sp.len - a.q_len + last_token - a.window + 1 : 0;

  f32x4 acc[kOut];
#pragma unroll
  for (int i = 0; i < kOut; ++i) acc[i] = f32x4{0, 0, 0, 0};
  float m = -INFINITY, l = 0.0f;
  int unit = 127, most = 0;                        // acc is in units of 2^(unit - 127); the largest exponent of a scale of values so far
  u32x4 kw[4][kLoads], vw[kOut];

  auto page_of = [&](int n) {
    const int64_t p = load_uniform(a.t.page + sp.at + n);
    return p >= 0 && p < a.c.pages ? p : (int64_t)-1;
  };
  auto load_k = [&](int64_t page) {
    const unsigned char* p = a.c.k + (page * a.c.heads + kv) * (kPage * R) + (16 * (col / 4) + col % 4) * R + (R / 4) * quarter;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int i = 0; i < kLoads; ++i) kw[t][i] = *reinterpret_cast<const u32x4*>(p + 4 * t * R + 16 * i);
  };
  auto load_v = [&](int64_t page) {
    const unsigned char* p = a.c.v + (page * a.c.heads + kv) * (kPage * R) + col * kPage + 16 * quarter;
#pragma unroll
    for (int i = 0; i < kOut; ++i) vw[i] = *reinterpret_cast<const u32x4*>(p + 16 * i * kPage);
  };

  int n = begin + wave;
  int64_t page = n < end ? page_of(n) : -1;
  if (page >= 0) { load_k(page); load_v(page); }
  while (n < end) {
    const int next = n + 4;
    const int64_t next_page = next < end ? page_of(next) : -1;
    if (page >= 0) {
      const float ks = load_uniform(a.c.k_scale + page * a.c.heads + kv), vs = load_uniform(a.c.v_scale + page * a.c.heads + kv);
      if (a.c.bytes8 < R) {                        // channels behind the head's may hold anything, and 0 times NaN is NaN
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
          const unsigned keep = (R / 4) * quarter + 8 * i < a.c.bytes8 ? ~0u : 0u;
#pragma unroll
          for (int t = 0; t < 4; ++t) { kw[t][i / 2][2 * (i % 2)] &= keep; kw[t][i / 2][2 * (i % 2) + 1] &= keep; }
        }
      }
      f32x4 x[4];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        x[t] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < kSteps; ++i) x[t] = mma(widen(u32x2{kw[t][i / 2][2 * (i % 2)], kw[t][i / 2][2 * (i % 2) + 1]}, T()), q[i], x[t]);
      }
      if (next_page >= 0) load_k(next_page);
      const int k0 = n * kPage;
      const float c = scale2 * ks;
      const float away = (float)(diag - k0 - 16 * quarter);
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float y = x[t][i] * c;
          if constexpr (CAP) y = tanh_of(y) * cap2;
          if constexpr (BIAS) y -= slope2 * fabsf(away - (float)(4 * t + i));
          x[t][i] = y;
        }
      const bool whole = k0 + kPage - 1 <= first_diag && k0 >= last_lo;
      if (!whole) {
        const int off = k0 + 16 * quarter;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) x[t][i] = off + 4 * t + i <= diag && off + 4 * t + i >= row_lo ? x[t][i] : -INFINITY;
        // what no row of the sequence sees may hold anything: as values it becomes zero
        const int dead = sp.lo - off, live = sp.len - off;       // keys below dead and from live on
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          unsigned mask = 0;
#pragma unroll
          for (int b = 0; b < 4; ++b) mask |= 4 * w + b >= dead && 4 * w + b < live ? 0xffu << (8 * b) : 0u;
#pragma unroll
          for (int i = 0; i < kOut; ++i) vw[i][w] &= mask;
        }
      }
      float top = -INFINITY;
#pragma unroll
      for (int t = 0; t < 4; ++t) top = fmaxf(top, fmaxf(fmaxf(x[t][0], x[t][1]), fmaxf(x[t][2], x[t][3])));
      top = max_quarters(top);
      const float now = fmaxf(m, top), base = now == -INFINITY ? 0.0f : now;
      const float by = m == now ? 1.0f : fast_exp2(m - now);
      // acc goes to units of the page's scale, which costs nothing beside the new maximum; but not further down than 2^-64 of the largest scale so far: a page
      // of zeros has the scale 2^-100, next to which sums of large values would overflow (448 * 2^31 tokens * 2^64 is finite).  A page below that has its
      // probabilities scaled instead: what float16 has no room for there is less than 2^-63 of the largest value of the cache.
      const int exponent = uniform((int)(__float_as_uint(vs) >> 23));
      most = max(most, exponent);
      const int new_unit = max(exponent, most - 64), shift = unit - new_unit;
      m = now;
      unit = new_unit;
      l *= by;
#pragma unroll
      for (int i = 0; i < kOut; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = __builtin_amdgcn_ldexpf(acc[i][j] * by, shift);
      vec8<T> p[2];
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          x[t][i] = fast_exp2(x[t][i] - base);
          l += x[t][i];
        }
      if (exponent != unit) {
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) x[t][i] = __builtin_amdgcn_ldexpf(x[t][i], exponent - unit);
      }
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) p[t / 2][4 * (t % 2) + i] = (T)x[t][i];
#pragma unroll
      for (int i = 0; i < kOut; ++i) {
        acc[i] = mma(widen(u32x2{vw[i][0], vw[i][1]}, T()), p[0], acc[i]);
        acc[i] = mma(widen(u32x2{vw[i][2], vw[i][3]}, T()), p[1], acc[i]);
      }
      if (next_page >= 0) load_v(next_page);
    } else if (next_page >= 0) {
      load_k(next_page);
      load_v(next_page);
    }
    n = next;
    page = next_page;
  }
  l = add_quarters(l);

  // join the waves: rows by their maxima
  __shared__ float ms[4][kRows], ls[4][kRows];
  __shared__ __align__(16) float sums[4][kRows][R + 4];
  if (quarter == 0) { ms[wave][col] = m; ls[wave][col] = l; }
#pragma unroll
  for (int i = 0; i < kOut; ++i) *reinterpret_cast<f32x4*>(&sums[wave][col][16 * i + 4 * quarter]) = acc[i] * __uint_as_float((unsigned)unit << 23);
  __syncthreads();
  const int64_t cell = (slot * gridDim.y + kv) * gridDim.z + tile;
  for (int i = threadIdx.x; i < kRows * R / 4; i += 256) {
    const int row = i / (R / 4), d = i % (R / 4) * 4;
    const int rr = tile * kRows + row, tok = rr / a.group;
    if (tok >= a.q_len) continue;
    const float top = fmaxf(fmaxf(ms[0][row], ms[1][row]), fmaxf(ms[2][row], ms[3][row])), base = top == -INFINITY ? 0.0f : top;
    f32x4 v = {0, 0, 0, 0};
    float sum = 0.0f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float f = fast_exp2(ms[w][row] - base);
      v += *reinterpret_cast<const f32x4*>(&sums[w][row][d]) * f;
      sum += ls[w][row] * f;
    }
    if (alone) {
      if (d < a.c.bytes8) {
        const float by = sum == 0.0f ? 0.0f : 1.0f / sum;
        const RowSource dst = a.o.of(kv * a.group + rr % a.group);
        T out[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) out[j] = (T)(v[j] * by);
        *reinterpret_cast<u32x2*>(const_cast<unsigned char*>(dst.base) + ((int64_t)s * a.q_len + tok) * dst.stride + d * 2) = __builtin_bit_cast(u32x2, out);
      }
    } else {
      *reinterpret_cast<f32x4*>(a.part + (cell * kRows + row) * R + d) = v;
      if (d == 0) a.part_ml[cell * kRows + row] = make_float2(top, sum);
    }
  }
}

// Joins a row's chunks; rows that no chunk has (no tokens) become zero.  A workgroup has a row of a sequence: R / 4 threads go over every
// (1024 / R)-th chunk, four channels each, and their sums are joined in order.  4 x 32 rows of up to 52 chunks 6 us, 128 x 32 rows of one to 11 7.7 us.
template <typename T, int R>
__global__ void __launch_bounds__(256) k_cache_join(AttendArgs a) {
  constexpr int kThreads = R / 4, kLanes = 256 / kThreads;
  const int s = blockIdx.x, tok = blockIdx.y / a.heads, head = blockIdx.y % a.heads, kv = head / a.group;
  const SeqPages sp = seq_pages(a, s);
  const bool none = sp.first >= sp.last;
  const int c0 = none ? 0 : sp.first / a.chunk, c1 = none ? 0 : (sp.last - 1) / a.chunk + 1;
  if (c1 - c0 == 1) return;
  const int rr = tok * a.group + head % a.group, d = threadIdx.x % kThreads * 4, mine = threadIdx.x / kThreads;
  const int64_t slot = sp.at / a.chunk + s, kv_heads = a.heads / a.group;
  float top = -INFINITY, sum = 0.0f;
  f32x4 v = {0, 0, 0, 0};
#pragma unroll 4
  for (int c = c0 + mine; c < c1; c += kLanes) {
    const int64_t row = (((slot + c) * kv_heads + kv) * a.tiles + rr / kRows) * kRows + rr % kRows;
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
  *reinterpret_cast<u32x2*>(const_cast<unsigned char*>(dst.base) + ((int64_t)s * a.q_len + tok) * dst.stride + d * 2) = __builtin_bit_cast(u32x2, out);
}

}  // namespace spg
