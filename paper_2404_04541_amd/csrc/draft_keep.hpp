// The nodes that stay move together: token start + way[i] of a sequence becomes token start + i, in all layers, keys and values.
//
// A wave has a sequence, a key head, a layer, and keys or values; the four of a workgroup share what they have to know of the sequence.  It goes over the pages that tokens come to, in order: way[i] >= i, so what
// a page's tokens are taken from lies in the page or behind it, and nothing that is still to be read has been written.  Only where tokens come from another page are they read twice, first for the scale.
// A token's values are a byte in each of its channels' rows, so every row of a page is read and written for any token that moves.  48 sequences, up to 60 nodes, 16 layers of 8 heads of 128 channels 30 to 40 us,
// about 100 MB of such rows; with a byte a lane and load instead of rows of 16 bytes through LDS 41 to 47.  One sequence in two layers 6 us: the chain of loads that leads there.
#pragma once
#include "draft_attend.hpp"

namespace spg {

struct KeepArgs {
  unsigned char* data[2];         // keys, values of all layers
  float* scale[2];
  int64_t pages;
  int layers, heads, bytes8;
  TableView t;
  TreeView trees;
  const int32_t *path, *kept;
  int32_t* new_lens;
};

constexpr int kKeepPlaces = kMostNodes / kPage + 2;       // pages that a tree's nodes can lie in, and one more

// What stays of a sequence's tree.
struct Way {
  int i[kMostNodes];              // ascending
  int count;
  int64_t page[kKeepPlaces];      // of places start / 64 and on; -1: none
};

// What the wave's lanes have put into LDS is there for the others.
__device__ __forceinline__ void in_wave_order() {
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_wave_barrier();
}

template <int R>
__global__ void __launch_bounds__(256) k_draft_keep(KeepArgs a) {
  __shared__ Way way;
  __shared__ unsigned tiles[2][R][kPage / 4 + 1];           // of the two waves that have values
  const int s = blockIdx.x, head = blockIdx.y, tid = threadIdx.x, lane = lane_id(), wave = uniform(tid / kWave), unit = blockIdx.z * 4 + wave;
  const int layer = unit / 2, values = unit % 2;
  const Tree tree = tree_of(a.trees, s);
  const int64_t len = a.t.lens[s], start = len - tree.n;
  const int asked = min(max(a.kept[s], 0), tree.n);
  if (tid == 0) way.count = asked;
  __syncthreads();
  if (tid < asked) {
    const int p = a.path[tree.first + tid];
    way.i[tid] = p;
    if (p >= tree.n || p <= (tid ? a.path[tree.first + tid - 1] : -1)) atomicMin(&way.count, tid);
  }
  const int place0 = (int)(start / kPage), places = (int)((len + kPage - 1) / kPage) - place0;
  bool lacks = tree.n == 0 || start < 0;
  if (!lacks && tid < places) {
    const int64_t at = a.t.ptr[s] + place0 + tid;
    const int64_t page = at >= 0 && at < a.t.ptr[s + 1] && at < a.t.nnz ? a.t.page[at] : -1;
    lacks = page < 0 || page >= a.pages;
    way.page[tid] = page;
  }
  lacks = __syncthreads_or(lacks);
  const int count = uniform(way.count);
  if (head == 0 && blockIdx.z == 0 && tid == 0) a.new_lens[s] = (int)(lacks ? len : start + count);
  if (lacks || count == 0 || layer >= a.layers || uniform(way.i[count - 1]) == count - 1) return;      // nothing moves

  const int64_t layer0 = (int64_t)layer * a.pages;
  unsigned char* const data = a.data[values];
  float* const scale = a.scale[values];
  auto cell = [&](int place) { return (layer0 + way.page[place]) * a.heads + head; };
  const int start0 = (int)(start - (int64_t)place0 * kPage);                         // the tree's first token, counted from the first page's first one, as all tokens are from here on
  for (int place = 0; place * kPage < start0 + count; ++place) {
    const int t0 = place * kPage, begin = max(start0 - t0, 0), until = min(start0 + count - t0, kPage);
    const int i0 = t0 + begin - start0, last = i0 + until - begin - 1;
    if (uniform(way.i[last]) == last) continue;
    auto source = [&](int o) { return start0 + way.i[t0 + o - start0]; };            // of the page's token o
    const int64_t mine = cell(place);
    const float old = scale[mine];
    float now = old;
    if (source(until - 1) / kPage != place) {
      // what comes from other pages: its largest magnitude (2^-9 times it, for 256 times the largest scale is 2^128; the smallest code times the smallest scale is 2^-109)
      float top = 0.0f;
      auto measure = [&](float code, float by) { const float v = fabsf(code) * (by * 0x1p-9f); top = v < INFINITY ? fmaxf(top, v) : top; };
      for (int o = begin; o < until; ++o) {
        const int from = uniform(source(o));
        if (from / kPage == place) continue;
        const int64_t c = cell(from / kPage);
        const float by = scale[c];
        if (!values) {
          if (4 * lane < a.bytes8) {
            const unsigned code = *reinterpret_cast<const unsigned*>(data + c * (kPage * R) + from % kPage * R + 4 * lane);
            measure(__builtin_amdgcn_cvt_f32_fp8(code, 0), by);
            measure(__builtin_amdgcn_cvt_f32_fp8(code, 1), by);
            measure(__builtin_amdgcn_cvt_f32_fp8(code, 2), by);
            measure(__builtin_amdgcn_cvt_f32_fp8(code, 3), by);
          }
        } else {
          for (int d = lane; d < a.bytes8; d += kWave) measure(__builtin_amdgcn_cvt_f32_fp8(data[c * (kPage * R) + d * kPage + from % kPage], 0), by);
        }
      }
#pragma unroll
      for (int d = 1; d < kWave; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
      now = fmaxf(old, scale_for(top * 0x1p9f));      // (of infinity the largest scale)
    }
    const bool grows = now > old;
    if (grows && lane == 0) scale[mine] = now;
    // (A code that is not 0 has made the page's scale grow; zeros of a page of large scale have not, and infinity times 0 would be NaN.)
    auto by_of = [&](int from) { return from / kPage == place ? old / now : fminf(scale[cell(from / kPage)] / now, 0x1p126f); };
    unsigned char* const to = data + mine * (kPage * R);
    if (!values) {
      // 16 tokens on their way together; a token is R / 4 words
      constexpr int kWords = R / 4, kTokens = kWave / kWords, kLoads = 16 / kTokens;
      const int w = lane % kWords;
      for (int o0 = begin; o0 < until; o0 += 16) {
        unsigned code[kLoads];
        float by[kLoads];
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
          const int o = o0 + i * kTokens + lane / kWords;
          by[i] = 1.0f;
          if (o < until) {
            const int from = source(o);
            code[i] = *reinterpret_cast<const unsigned*>(data + cell(from / kPage) * (kPage * R) + from % kPage * R + 4 * w);
            by[i] = by_of(from);
          }
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");      // (the tokens are there before others take their places)
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
          const int o = o0 + i * kTokens + lane / kWords;
          if (o < until) *reinterpret_cast<unsigned*>(to + o * R + 4 * w) = by[i] == 1.0f ? code[i] : rescale8(code[i], by[i]);
        }
      }
      if (grows)
        for (int n = lane; n < begin * kWords; n += kWave) reinterpret_cast<unsigned*>(to)[n] = rescale8(reinterpret_cast<unsigned*>(to)[n], old / now);
    } else {
      // the page's values come to LDS as rows of 16 bytes and go back so, a row of 64 tokens to a channel; in between a lane has R / 64 channels
      constexpr int kChannels = R / kWave, kRows = kWave / 4, kPitch = kPage / 4 + 1;      // words of a row in LDS: no two of 64 rows begin in the same bank
      unsigned(&tile)[R][kPitch] = tiles[wave / 2];
      const int w0 = grows ? 0 : begin / 4, w1 = (until + 3) / 4;
      u32x4 chunk[R / kRows];
#pragma unroll
      for (int i = 0; i < R / kRows; ++i) chunk[i] = *reinterpret_cast<const u32x4*>(to + (lane / 4 + i * kRows) * kPage + lane % 4 * 16);
#pragma unroll
      for (int i = 0; i < R / kRows; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) tile[lane / 4 + i * kRows][lane % 4 * 4 + j] = chunk[i][j];
      in_wave_order();
      for (int w = w0; w < w1; ++w) {
        unsigned word[kChannels];
#pragma unroll
        for (int c = 0; c < kChannels; ++c) word[c] = tile[lane + c * kWave][w];
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          const int o = 4 * w + b;
          if (o >= until) break;
          const int from = o < begin ? t0 + o : uniform(source(o));
          const float by = by_of(from);
          if (from == t0 + o && by == 1.0f) continue;
#pragma unroll
          for (int c = 0; c < kChannels; ++c) {
            unsigned x;
            if (from / kPage == place) x = reinterpret_cast<const unsigned char*>(tile[lane + c * kWave])[from % kPage];
            else x = data[cell(from / kPage) * (kPage * R) + (lane + c * kWave) * kPage + from % kPage];
            if (by != 1.0f) x = to8(__builtin_amdgcn_cvt_f32_fp8(x, 0) * by, 0.0f, 0.0f, 0.0f) & 0xffu;
            word[c] = (word[c] & ~(0xffu << (8 * b))) | x << (8 * b);
          }
        }
#pragma unroll
        for (int c = 0; c < kChannels; ++c) tile[lane + c * kWave][w] = word[c];      // (what a later token is taken from lies behind)
      }
      in_wave_order();
      if (lane % 4 >= w0 / 4 && lane % 4 <= (w1 - 1) / 4)
#pragma unroll
        for (int i = 0; i < R / kRows; ++i) {
          u32x4 v;
#pragma unroll
          for (int j = 0; j < 4; ++j) v[j] = tile[lane / 4 + i * kRows][lane % 4 * 4 + j];
          *reinterpret_cast<u32x4*>(to + (lane / 4 + i * kRows) * kPage + lane % 4 * 16) = v;
        }
      in_wave_order();
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  }
}

}  // namespace spg
