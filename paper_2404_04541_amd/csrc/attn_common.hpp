// Shared pieces of the attention kernels: 16-bit types, matrix instructions, tiles in LDS, the mask's rows.
//
// Every product of these kernels has the 32 x 32 x 16 form: a lane of the left operand holds 8 elements of row lane % 32, one of
// the right operand 8 elements of column lane % 32 (elements 8 * (lane / 32) and on along the contraction), and lane l of the
// result holds, of column l % 32, the rows 8 * (i / 4) + 4 * (l / 32) + i % 4, i = 0 .. 15.  So the probabilities of a tile leave
// the first product in the lanes that need them as the right operand of the second, if that contracts over its rows in the order
// in which they come: half h of the wave has rows 4h .. 4h + 3 and 8 + 4h .. 8 + 4h + 3 of every 16.  The left operand of the second
// product is a tile read across its rows, four rows at a time (ds_read_b64_tr_b16), in that order; nothing moves between lanes.
#pragma once
#include "common.hpp"

namespace spg {

typedef __bf16 bf16_t;
typedef _Float16 f16_t;
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef short i16x4 __attribute__((ext_vector_type(4)));

template <typename T> struct Vec8;
template <> struct Vec8<bf16_t> { typedef bf16_t type __attribute__((ext_vector_type(8))); };
template <> struct Vec8<f16_t> { typedef f16_t type __attribute__((ext_vector_type(8))); };
template <typename T> using vec8 = typename Vec8<T>::type;

__device__ __forceinline__ f32x16 mma(vec8<bf16_t> a, vec8<bf16_t> b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16 mma(vec8<f16_t> a, vec8<f16_t> b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 mma(vec8<bf16_t> a, vec8<bf16_t> b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 mma(vec8<f16_t> a, vec8<f16_t> b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

__host__ __device__ constexpr int ceil_div_d(int a, int b) { return a / b + (a % b != 0); }

constexpr int kPatTile = 128;    // rows and columns of a pattern's tiles; queries of a workgroup (forward, dQ)
constexpr int kKeyTile = 64;     // keys that come through LDS together (forward, dQ), or that a workgroup has (dK, dV)
constexpr int kQueryTile = 64;   // queries that come through LDS together (dK, dV)
constexpr int kRowGroup = 32;    // rows whose bounds the plan sums up: a wave's queries
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// Row i of a mask sees the keys lo <= j < hi and is at distance 0 from key diag.
struct RowBound { int lo, hi, diag, pad; };
// Of kRowGroup rows: the keys that any of them sees lie in [lo, hi); all rows see [all_lo, all_hi).
struct GroupBound { int lo, hi, all_lo, all_hi; };

// The plan in device memory; what a pattern adds is null without one.  A tile of kPatTile queries (keys) has a row of flags, a bit for
// every tile of keys (queries), in `seen` (`seen_by`).
struct PlanView {
  RowBound* rows;          // q_len
  GroupBound* groups;      // ceil(q_len / kRowGroup)
  int2* cols;              // per kKeyTile keys: the queries that can see any of them
  int4* q_order;           // tiles of kPatTile queries, the ones with the most to do first: the tile, and the keys from y to before z that its queries see
  unsigned long long* totals;   // tiles of kKeyTile keys that the tiles of queries go over, tiles of kQueryTile queries that those of keys go over
  unsigned* seen;          // ceil(q_len / kPatTile) rows of seen_words
  unsigned* seen_by;       // ceil(k_len / kPatTile) rows of seen_by_words
  int* error;
  int seen_words, seen_by_words;
};

// What a score is made of: s = cap tanh(scale q.k / cap) - slope |diag - j|, in units of log 2 (so that the softmax takes exp2 as it is).
struct ScoreShape {
  float scale, cap;        // cap 0: none
  const float* slopes;     // per query head, or null
};

// exp2 by the hardware's instruction (subnormal results become 0: a probability below 2^-126).
__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float fast_rcp(float x) { return __builtin_amdgcn_rcpf(x); }

// tanh(x), given x * 2 log2(e): 1 - 2 / (exp(2x) + 1).  Off by at most about 2e-7 in absolute terms, which is what a capped score needs.
__device__ __forceinline__ float tanh_of(float x2) { return 1.0f - 2.0f * fast_rcp(fast_exp2(x2) + 1.0f); }

// The largest and the smallest of three, as one instruction each; NaN comes through (a row with a score of NaN has no other result).  By builtins, for the
// compiler places the waits behind a matrix instruction, whose results arrive cycles later, only in front of instructions that it knows: between
// the last product and an instruction in inline assembly there was none.  (fmaxf and fminf would first bring what might be a signalling NaN into order.)
__device__ __forceinline__ float max3(float a, float b, float c) { return __builtin_elementwise_maximum(__builtin_elementwise_maximum(a, b), c); }
__device__ __forceinline__ float min3(float a, float b, float c) { return __builtin_elementwise_minimum(__builtin_elementwise_minimum(a, b), c); }

// A value that all lanes have, in a scalar register: descriptors and addresses that depend on it then need no loop over the lanes.
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// What no kernel that is running writes, at an address that all lanes have: through the scalar cache, so that it does not wait behind loads of tiles.
template <typename E>
__device__ __forceinline__ E load_uniform(const E* p) {
  static_assert(sizeof(E) % 4 == 0, "whole words");
  typedef const __attribute__((address_space(4))) int const_int;
  const_int* w = (const_int*)(uintptr_t)p;
  struct Words { int v[sizeof(E) / 4]; } words;
#pragma unroll
  for (int i = 0; i < (int)(sizeof(E) / 4); ++i) words.v[i] = w[i];
  return __builtin_bit_cast(E, words);
}

// The larger of both halves' values, in both halves.
__device__ __forceinline__ float max_halves(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float add_halves(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(3))) i16x4 lds_i16x4;

// A tile of rows of D 16-bit elements in LDS, in chunks of 16 bytes.  A chunk's place in its row is exclusive-ored with bits of the row's
// number, so that both ways in which tiles are read spread over all banks: 16 rows at one chunk (row operands) and four rows at 64 neighbouring
// bytes (reads across rows, half a wave at a time).  Rows of 256 bytes: chunk ^ 4 (r % 4) ^ (r / 4 % 4); of 128 bytes two rows share the banks.
// (With reads across rows taken to be of eight rows and 32 bytes, each took twice as long: 8192 tokens, forward 203 -> 200 us, backward 641 -> 631.)
template <int D>
struct TileShape {
  static constexpr int kChunks = D / 8;
  static constexpr int kRowBytes = D * 2;
  __device__ static __forceinline__ int swizzle(int row) {
    if constexpr (D == 128) return ((row & 3) << 2) ^ ((row >> 2) & 3);
    else return ((row & 2) << 1) ^ ((row >> 2) & 3);
  }
  // Where a lane reads, in bytes.  The bits of a chunk's number lie below a row's, so the chunks of a row are found by an exclusive or with
  // a constant, and rows that are a multiple of 16 away by a constant distance.
  // Row operand of step i: elements 16 i + 8 (lane / 32) .. of row lane % 32.
  __device__ static __forceinline__ int row_base(int lane) { return (lane & 31) * kRowBytes + (((lane >> 5) ^ swizzle(lane & 31)) << 4); }
  template <typename T>
  __device__ static __forceinline__ vec8<T> row(const unsigned char* tile, int base, int r0, int i) {
    return *reinterpret_cast<const vec8<T>*>(tile + r0 * kRowBytes + (base ^ (32 * i)));
  }
  // The operand across rows: of column 32 i + lane % 32 the rows r0 + 4h .. + 3 and r0 + 8 + 4h .. + 3, h = lane / 32, r0 a multiple of 16.  Lane j of
  // 16 fetches 8 bytes, columns 4 (j % 4) .. of row j / 4; the instruction hands lane j the four rows of column j.
  __device__ static __forceinline__ int across_base(int lane) {
    const int r = ((lane >> 5) << 2) + ((lane >> 2) & 3), byte = ((lane & 16) + ((lane & 3) << 2)) * 2;
    return r * kRowBytes + (((byte >> 4) ^ swizzle(r)) << 4) + (byte & 15);
  }
  template <typename T>
  __device__ static __forceinline__ vec8<T> across(const unsigned char* tile, int base, int r0, int i) {
    union { i16x4 part[2]; vec8<T> all; } u;
    u.part[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(tile + r0 * kRowBytes + (base ^ (64 * i))));
    u.part[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(tile + (r0 + 8) * kRowBytes + (base ^ 32 ^ (64 * i))));   // (eight rows on, bit 1 of the swizzle differs)
    return u.all;
  }
};

// Keeps what is computed from v inside the loop that it stands in: an exclusive or per read costs less than a register for each of the addresses.
__device__ __forceinline__ int in_loop(int v) {
  asm volatile("" : "+v"(v));
  return v;
}

// Loads to LDS are outstanding until the wave waits for them; the barrier then makes them everybody's.
__device__ __forceinline__ void tiles_ready() {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
}

// Rows of a packed tensor: token t of one head begins at base + t * stride (bytes).
struct RowSource {
  const unsigned char* base;
  int64_t stride;
};

// Brings rows first .. first + ROWS - 1 into a tile, from global memory straight to LDS: each lane asks for the chunk that belongs where its 16
// bytes land (lane l of an instruction writes 16 l bytes behind a common address).  Rows outside [lo, hi) and chunks behind the head's `bytes` become
// zero: their lanes' offsets lie outside the buffer that the resource describes.  Most tiles have neither: two operations a load.
template <int D, int ROWS, int THREADS>
struct TileLoader {
  using S = TileShape<D>;
  static constexpr int kLoads = ROWS * S::kChunks / THREADS, kStep = kWave / S::kChunks;   // instructions a wave; rows of one
  static_assert(kLoads * THREADS == ROWS * S::kChunks && 16 % kStep == 0, "whole instructions");
  int wave, row0, chunk;      // of the first instruction; the swizzle is linear, so those of the others follow without carries
  unsigned stride, at0;
  __device__ __forceinline__ TileLoader(int64_t stride_, int lane) : wave(uniform(threadIdx.x / kWave)), stride((unsigned)stride_) {
    row0 = wave * (kLoads * kStep) + lane / S::kChunks;
    chunk = ((lane % S::kChunks) ^ S::swizzle(row0)) * 16;
    at0 = (unsigned)row0 * stride;
  }
};

template <int D, int ROWS, int THREADS>
__device__ __forceinline__ void load_tile(const TileLoader<D, ROWS, THREADS>& l, const unsigned char* base, unsigned char* tile, int first, int lo, int hi, int bytes, bool inside) {
  using L = TileLoader<D, ROWS, THREADS>;
  const unsigned limit = (ROWS - 1) * l.stride + (unsigned)bytes;
  const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)(base + (uint64_t)(unsigned)first * l.stride), 0, limit, 0x00027000);
#pragma unroll
  for (int i = 0; i < L::kLoads; ++i) {
    const int row = first + l.row0 + i * L::kStep, c = l.chunk ^ (L::S::swizzle(i * L::kStep) * 16);
    unsigned at = l.at0 + (unsigned)(i * L::kStep) * l.stride + (unsigned)c;
    if (!inside) at = (row >= lo) & (row < hi) & (c < bytes) ? at : 0x80000000u;
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_void*)(tile + (l.wave * L::kLoads + i) * (kWave * 16)), 16, (int)at, 0, 0, 0);
  }
}

// Two tensors' tiles of the same rows: most are whole, and their loads cost two operations each.
template <int D, int ROWS, int THREADS>
__device__ __forceinline__ void load_tiles(const TileLoader<D, ROWS, THREADS>& la, const unsigned char* a, unsigned char* tile_a, const TileLoader<D, ROWS, THREADS>& lb,
                                           const unsigned char* b, unsigned char* tile_b, int first, int lo, int hi, int bytes) {
  if ((first >= lo) & (first + ROWS <= hi) & (bytes == 2 * D)) {
    load_tile(la, a, tile_a, first, lo, hi, bytes, true);
    load_tile(lb, b, tile_b, first, lo, hi, bytes, true);
  } else {
    load_tile(la, a, tile_a, first, lo, hi, bytes, false);
    load_tile(lb, b, tile_b, first, lo, hi, bytes, false);
  }
}

// A lane's operand of one row that stays in registers: 8 elements at 16 * step + 8 * half for every step; zero outside the head and where !ok.
template <typename T, int D>
__device__ __forceinline__ void load_row(const RowSource& src, int64_t row, bool ok, int bytes, int half, vec8<T>* out) {
  const unsigned char* p = src.base + row * src.stride;
#pragma unroll
  for (int s = 0; s < D / 16; ++s) {
    const int byte = (16 * s + 8 * half) * 2;
    u32x4 v = {0, 0, 0, 0};
    if (ok && byte < bytes) v = *reinterpret_cast<const u32x4*>(p + byte);
    out[s] = __builtin_bit_cast(vec8<T>, v);
  }
}

// 16 numbers of a result as two right operands.
template <typename T>
__device__ __forceinline__ void to_operand(const f32x16& v, vec8<T>* out) {
#pragma unroll
  for (int i = 0; i < 8; ++i) { out[0][i] = (T)v[i]; out[1][i] = (T)v[8 + i]; }
}

// How many of n ascending numbers at(0) .. at(n - 1) lie below `limit`, by the whole wave: 64 of them are looked at together.
template <typename F>
__device__ __forceinline__ int wave_count_below(int n, int64_t limit, F at) {
  int a = 0;                                     // at(i) < limit for i < a
  while (n - a > 0) {
    const int step = ceil_div_d(n - a, kWave);   // lane l looks at the last of its share
    const int i = a + (lane_id() + 1) * step - 1;
    const bool below = (int64_t)a + (int64_t)(lane_id() + 1) * step - 1 < n && at(i) < limit;
    const int shares = __popcll(__ballot(below));
    a += shares * step;
    if (step == 1) return a;
    n = (int64_t)a + step < n ? a + step : n;    // the next share's last number is not below
  }
  return a;
}

}  // namespace spg
