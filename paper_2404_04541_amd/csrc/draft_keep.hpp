// The nodes that stay move together: token start + way[i] of a sequence becomes token start + i, in all layers, keys and values.
//
// A workgroup has a sequence, a key head, a layer, and keys or values.  It goes over the pages that tokens come to, in order: way[i] >= i, so what a page's tokens are taken from lies in the page or
// behind it, and nothing that is still to be read has been written.  A page's tokens are gathered in LDS first, with the largest magnitude that comes from other pages; then the scale is known.
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

template <int R>
__global__ void __launch_bounds__(256) k_draft_keep(KeepArgs a) {
  __shared__ Way way;
  __shared__ __align__(16) unsigned char codes[R * (kPage + 4)];      // keys: [token][R], values: [channel][64 + 4]
  __shared__ float tops[4];
  const int s = blockIdx.x, head = blockIdx.y, layer = blockIdx.z / 2, values = blockIdx.z % 2, tid = threadIdx.x;
  const Tree tree = tree_of(a.trees, s);
  const int64_t len = a.t.lens[s], start = len - tree.n;
  const bool first = head == 0 && blockIdx.z == 0 && tid == 0;
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
  const int count = way.count;
  if (first) a.new_lens[s] = (int)(lacks ? len : start + count);
  if (lacks || count == 0 || way.i[count - 1] == count - 1) return;      // nothing moves

  const int64_t layer0 = (int64_t)layer * a.pages;
  unsigned char* const data = a.data[values];
  float* const scale = a.scale[values];
  auto cell = [&](int place) { return (layer0 + way.page[place]) * a.heads + head; };
  for (int place = 0; place * kPage + (int64_t)place0 * kPage < start + count; ++place) {
    const int64_t t0 = (int64_t)(place0 + place) * kPage;                              // the page's first token
    const int begin = (int)(start > t0 ? start - t0 : 0), until = (int)(start + count - t0 < kPage ? start + count - t0 : kPage);
    const int i0 = (int)(t0 + begin - start), moves = until - begin;
    if (way.i[i0 + moves - 1] == i0 + moves - 1) continue;
    const int64_t mine = cell(place);
    const float old = scale[mine];
    auto source = [&](int i) { return start + way.i[i0 + i] - (int64_t)place0 * kPage; };   // counted from the first page's first token
    float top = 0.0f;
    auto measure = [&](float code, float by) { const float v = fabsf(code) * by; top = v < INFINITY ? fmaxf(top, v) : top; };
    if (!values) {
      for (int n = tid; n < moves * (R / 4); n += 256) {
        const int i = n / (R / 4), w = n % (R / 4), from = (int)source(i);
        const int64_t c = cell(from / kPage);
        const unsigned code = *reinterpret_cast<const unsigned*>(data + c * (kPage * R) + from % kPage * R + 4 * w);
        *reinterpret_cast<unsigned*>(codes + i * R + 4 * w) = code;
        if (from / kPage != place && 4 * w < a.bytes8) {
          const float by = scale[c];
          measure(__builtin_amdgcn_cvt_f32_fp8(code, 0), by);
          measure(__builtin_amdgcn_cvt_f32_fp8(code, 1), by);
          measure(__builtin_amdgcn_cvt_f32_fp8(code, 2), by);
          measure(__builtin_amdgcn_cvt_f32_fp8(code, 3), by);
        }
      }
    } else {
      for (int n = tid; n < moves * R; n += 256) {
        const int i = n / R, d = n % R, from = (int)source(i);
        const int64_t c = cell(from / kPage);
        const unsigned code = data[c * (kPage * R) + d * kPage + from % kPage];
        codes[d * (kPage + 4) + begin + i] = (unsigned char)code;
        if (from / kPage != place && d < a.bytes8) measure(__builtin_amdgcn_cvt_f32_fp8(code, 0), scale[c]);
      }
    }
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
    if (lane_id() == 0) tops[tid / kWave] = top;
    __syncthreads();
    const float now = fmaxf(old, scale_for(fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]))));
    const bool grows = now > old;
    if (tid == 0 && grows) scale[mine] = now;                // (everybody has the old one)
    auto by_of = [&](int i) { const int from = (int)source(i) / kPage; return from == place ? old / now : scale[cell(from)] / now; };
    unsigned char* const to = data + mine * (kPage * R);
    if (!values) {
      for (int n = tid; n < moves * (R / 4); n += 256) {
        const int i = n / (R / 4), w = n % (R / 4);
        const float by = by_of(i);
        const unsigned code = *reinterpret_cast<const unsigned*>(codes + i * R + 4 * w);
        *reinterpret_cast<unsigned*>(to + (begin + i) * R + 4 * w) = by == 1.0f ? code : rescale8(code, by);
      }
      if (grows)
        for (int n = tid; n < begin * (R / 4); n += 256) reinterpret_cast<unsigned*>(to)[n] = rescale8(reinterpret_cast<unsigned*>(to)[n], old / now);
    } else {
      const int w0 = grows ? 0 : begin / 4, words = (until + 3) / 4 - w0;
      for (int n = tid; n < words * R; n += 256) {
        const int d = n / words, o = (w0 + n % words) * 4;
        unsigned* p = reinterpret_cast<unsigned*>(to + d * kPage + o);
        const unsigned was = *p, again = grows ? rescale8(was, old / now) : was;
        unsigned word = 0;
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          unsigned byte = (o + b < begin ? again : was) >> (8 * b) & 0xffu;
          if (o + b >= begin && o + b < until) {
            byte = codes[d * (kPage + 4) + o + b];
            const float by = by_of(o + b - begin);
            if (by != 1.0f) byte = to8(__builtin_amdgcn_cvt_f32_fp8(byte, 0) * by, 0.0f, 0.0f, 0.0f) & 0xffu;
          }
          word |= byte << (8 * b);
        }
        *p = word;
      }
    }
    __syncthreads();
  }
}

}  // namespace spg
