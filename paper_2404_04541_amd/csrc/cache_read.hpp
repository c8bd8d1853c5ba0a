// Tokens back out of the paged cache, as rows of 16 bits.
#pragma once
#include "cache_kernels.hpp"

namespace spg {

struct ReadArgs {
  CacheView c;
  TableView t;
  const int64_t* ptr;       // rows ptr[s] .. ptr[s + 1] - 1 of k and v become the last tokens of sequence s
  HeadTensor k, v;
  int64_t tokens;
};

// A workgroup has a page that rows lie in, and a head; places of pages as in k_cache_append.  Keys are rows already; values are turned in LDS, two channels a word.
// Rows of tokens before the sequence's first, or in pages that its table lacks, become zero.  Memory bounds it: 64 sequences of 30 to 16 384 tokens, 8 heads of 128 channels, 137 us, 4.9 TB/s read and written, which is
// what a copy reaches; one of 2001 tokens 6.6 us.
template <typename T, int R>
__global__ void __launch_bounds__(256) k_cache_read(ReadArgs a) {
  const int head = blockIdx.y, tid = threadIdx.x;
  const int64_t slot = blockIdx.x;
  auto begin_of = [&](int s) { const int64_t v = a.ptr[s]; return v < 0 ? 0 : v > a.tokens ? a.tokens : v; };
  const int s = find_seq(a.t.seqs, slot, [&](int i) { return begin_of(i) / kPage + 2 * (int64_t)i; });
  const int64_t first = begin_of(s), count = begin_of(s + 1) - first;
  const int64_t len = a.t.lens[s], start = len - count;
  if (count <= 0) return;
  const int64_t n = (start >> 6) + (slot - (first / kPage + 2 * (int64_t)s));       // the page's place in the sequence
  static_assert(kPage == 64, "a shift");
  if (n * kPage >= len) return;
  const int from = start > n * kPage ? (int)(start - n * kPage) : 0;                // tokens of the page: from .. to - 1
  const int to = len < (n + 1) * kPage ? (int)(len - n * kPage) : kPage;
  const int64_t row0 = first + (n * kPage + from - start);                          // the row of the first of them
  const int64_t at = a.t.ptr[s] + n;
  int64_t page = n >= 0 && at >= 0 && at < a.t.ptr[s + 1] && at < a.t.nnz ? a.t.page[at] : -1;
  if (page >= a.c.pages) page = -1;
  const RowSource ks = a.k.of(head), vs = a.v.of(head);
  const int chunks = a.c.bytes8 / 8;
  auto put = [&](const RowSource& dst, int o, int chunk, u32x4 v) {
    *reinterpret_cast<u32x4*>(const_cast<unsigned char*>(dst.base) + (row0 + o - from) * dst.stride + chunk * 16) = v;
  };
  if (page < 0) {
    for (int i = tid; i < (to - from) * chunks; i += 256) {
      put(ks, from + i / chunks, i % chunks, u32x4{0, 0, 0, 0});
      put(vs, from + i / chunks, i % chunks, u32x4{0, 0, 0, 0});
    }
    return;
  }
  const int64_t ph = page * a.c.heads + head;
  const float k_by = a.c.k_scale[ph], v_by = a.c.v_scale[ph];
  const unsigned char* kp = a.c.k + ph * (kPage * R);
  const unsigned char* vp = a.c.v + ph * (kPage * R);
  // values: a lane takes four tokens of two channels
  __shared__ __align__(16) unsigned turned[kPage][R / 2 + 4];
  for (int i = tid; i < kPage / 4 * (R / 2); i += 256) {
    const int o = i % (kPage / 4) * 4, d = i / (kPage / 4) * 2;
    const unsigned x = *reinterpret_cast<const unsigned*>(vp + d * kPage + o), y = *reinterpret_cast<const unsigned*>(vp + (d + 1) * kPage + o);
    const T lo[4] = {(T)(__builtin_amdgcn_cvt_f32_fp8(x, 0) * v_by), (T)(__builtin_amdgcn_cvt_f32_fp8(x, 1) * v_by), (T)(__builtin_amdgcn_cvt_f32_fp8(x, 2) * v_by),
                     (T)(__builtin_amdgcn_cvt_f32_fp8(x, 3) * v_by)};
    const T hi[4] = {(T)(__builtin_amdgcn_cvt_f32_fp8(y, 0) * v_by), (T)(__builtin_amdgcn_cvt_f32_fp8(y, 1) * v_by), (T)(__builtin_amdgcn_cvt_f32_fp8(y, 2) * v_by),
                     (T)(__builtin_amdgcn_cvt_f32_fp8(y, 3) * v_by)};
#pragma unroll
    for (int b = 0; b < 4; ++b)
      turned[o + b][d / 2] = (unsigned)__builtin_bit_cast(unsigned short, lo[b]) | (unsigned)__builtin_bit_cast(unsigned short, hi[b]) << 16;
  }
  for (int i = tid; i < (to - from) * chunks; i += 256) {
    const int o = from + i / chunks, chunk = i % chunks;
    const u32x2 w = *reinterpret_cast<const u32x2*>(kp + o * R + chunk * 8);
    T out[8];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      out[4 * j] = (T)(__builtin_amdgcn_cvt_f32_fp8(w[j], 0) * k_by);
      out[4 * j + 1] = (T)(__builtin_amdgcn_cvt_f32_fp8(w[j], 1) * k_by);
      out[4 * j + 2] = (T)(__builtin_amdgcn_cvt_f32_fp8(w[j], 2) * k_by);
      out[4 * j + 3] = (T)(__builtin_amdgcn_cvt_f32_fp8(w[j], 3) * k_by);
    }
    put(ks, o, chunk, __builtin_bit_cast(u32x4, out));
  }
  __syncthreads();
  for (int i = tid; i < (to - from) * chunks; i += 256) {
    const int o = from + i / chunks, chunk = i % chunks;
    put(vs, o, chunk, *reinterpret_cast<const u32x4*>(&turned[o][chunk * 4]));
  }
}

}  // namespace spg
