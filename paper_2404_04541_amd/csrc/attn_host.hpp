// What the entry points of attention, of the paged cache and of drafted tokens share on the host: argument checks, scratch memory, views of the
// caller's structures, the choice of a kernel's variant.
#pragma once
#include "../../include/spattn.h"

#include <cmath>
#include <exception>
#include <type_traits>

#include "cache_kernels.hpp"
#include "context.hpp"

namespace spg {

constexpr int64_t kMaxTokens = int64_t(1) << 30;
constexpr int64_t kMaxStride = int64_t(1) << 23;    // elements: 128 rows stay within 31 bits of bytes

// Nothing leaves a C entry but a status: an exception (a string that finds no memory) becomes one.
template <typename F>
inline int guarded(spgemm_context* h, F f) {
  if (!h) return SPGEMM_INVALID_ARG;
  try {
    return f();
  } catch (const std::exception&) {
    return SPGEMM_ALLOC_FAILED;
  }
}

inline int launched(spgemm_context* h) {
  HIP_TRY(h, hipGetLastError());
  return SPGEMM_OK;
}

// The handle's scratch memory, at least so many bytes: grown where a call needs more than any before it.  A captured call leaves the block's address in the
// graph, whose replays use it for as long as the handle lives; so a block that was captured, or is outgrown while a capture goes on (which cannot wait for the
// stream), stays, and the next is at least twice as large, so that all that stay together are smaller than the last.  Any other is released.
inline int scratch(spgemm_context* h, size_t bytes, void** out) {
  hipStreamCaptureStatus status = hipStreamCaptureStatusNone;
  if (hipStreamIsCapturing(h->stream, &status) != hipSuccess) (void)hipGetLastError();
  const bool captures = status != hipStreamCaptureStatusNone;
  if (bytes > h->work_bytes) {
    size_t want = bytes;
    if (h->work && (h->work_captured || captures)) {
      want = bytes > 2 * h->work_bytes ? bytes : 2 * h->work_bytes;
      h->outgrown.push_back(h->work);
    } else if (h->work) {
      HIP_TRY(h, hipStreamSynchronize(h->stream));
      dev_free(h, h->work);
    }
    h->work = nullptr;
    h->work_bytes = 0;
    h->work_captured = false;
    void* p = dev_alloc(h, want);
    if (!p && want > bytes) p = dev_alloc(h, want = bytes);
    if (!p) return fail(h, SPGEMM_ALLOC_FAILED, "scratch memory");
    h->work = p;
    h->work_bytes = want;
  }
  h->work_captured |= captures;
  *out = h->work;
  return SPGEMM_OK;
}

// Pieces of one block of memory, in order.
struct Carve {
  unsigned char* base;
  size_t used = 0;
  template <typename E>
  E* take(int64_t n) {
    E* p = reinterpret_cast<E*>(base + used);
    used += align_up((size_t)n * sizeof(E));
    return p;
  }
};

// Waits for what kernels left in device memory.
template <typename E>
inline int fetch(spgemm_context* h, const void* from, E* to) {
  PinnedLease lease(h->stream);
  if (!lease.p) return fail(h, SPGEMM_ALLOC_FAILED, "pinned memory");
  static_assert(sizeof(E) <= sizeof(Control), "fits a pinned block");
  lease.written();
  HIP_TRY(h, hipMemcpyAsync(lease.p, from, sizeof(E), hipMemcpyDeviceToHost, h->stream));
  HIP_TRY(h, hipStreamSynchronize(h->stream));
  lease.waited();
  std::memcpy(to, lease.p, sizeof(E));
  return SPGEMM_OK;
}

inline int check_tensor(spgemm_context* h, const spattn_tensor& t, int64_t tokens, const char* name) {
  if (tokens == 0) return SPGEMM_OK;
  if (!t.data) return fail(h, SPGEMM_INVALID_ARG, std::string(name) + " is null");
  if (t.token_stride < 0 || t.head_stride < 0) return fail(h, SPGEMM_INVALID_ARG, std::string(name) + ": negative stride");
  if (reinterpret_cast<uintptr_t>(t.data) % 16 || t.token_stride % 8 || t.head_stride % 8)
    return fail(h, SPGEMM_UNSUPPORTED, std::string(name) + ": base and strides must be multiples of 16 bytes");
  if (t.token_stride >= kMaxStride) return fail(h, SPGEMM_UNSUPPORTED, std::string(name) + ": a token stride must be below 2^23 elements");
  return SPGEMM_OK;
}

inline HeadTensor view(const spattn_tensor& t) { return {static_cast<unsigned char*>(t.data), t.token_stride * 2, t.head_stride * 2}; }

inline int check_shape(spgemm_context* h, int32_t dtype, int32_t heads, int32_t kv_heads, int32_t head_dim, float scale, float cap) {
  if (dtype != SPATTN_F16 && dtype != SPATTN_BF16) return fail(h, SPGEMM_INVALID_ARG, "unknown dtype");
  if (heads <= 0 || kv_heads <= 0 || heads % kv_heads) return fail(h, SPGEMM_INVALID_ARG, "heads must be a positive multiple of kv_heads");
  if (heads > 65535) return fail(h, SPGEMM_UNSUPPORTED, "more than 65535 heads");
  if (head_dim <= 0) return fail(h, SPGEMM_INVALID_ARG, "head_dim must be positive");
  if (head_dim % 8 || head_dim > 128) return fail(h, SPGEMM_UNSUPPORTED, "head_dim must be a multiple of 8, at most 128");
  if (!(scale > 0.0f) || !std::isfinite(scale)) return fail(h, SPGEMM_INVALID_ARG, "scale must be positive and finite");
  if (!(cap >= 0.0f) || !std::isfinite(cap)) return fail(h, SPGEMM_INVALID_ARG, "cap must be 0 or positive and finite");
  if (cap > 0.0f && !std::isfinite(4.0f * scale / cap)) return fail(h, SPGEMM_INVALID_ARG, "cap is too small for scale");
  return SPGEMM_OK;
}

// Calls f.template operator()<type, padded head, cap, bias>() for what the arguments say.
template <typename F>
inline void dispatch(int32_t dtype, int head_dim, bool cap, bool bias, F f) {
  auto scores = [&](auto type, auto dim) {
    if (cap && bias) f(type, dim, std::true_type{}, std::true_type{});
    else if (cap) f(type, dim, std::true_type{}, std::false_type{});
    else if (bias) f(type, dim, std::false_type{}, std::true_type{});
    else f(type, dim, std::false_type{}, std::false_type{});
  };
  auto dims = [&](auto type) {
    if (head_dim <= 64) scores(type, std::integral_constant<int, 64>{});
    else scores(type, std::integral_constant<int, 128>{});
  };
  if (dtype == SPATTN_BF16) dims(bf16_t{});
  else dims(f16_t{});
}

inline int check_cache(spgemm_context* h, const spcache* c) {
  if (!c) return fail(h, SPGEMM_INVALID_ARG, "cache is null");
  if (c->layers <= 0 || c->pages < 0 || c->kv_heads <= 0 || c->head_dim <= 0) return fail(h, SPGEMM_INVALID_ARG, "cache: sizes must be positive");
  if (c->head_dim % 8 || c->head_dim > 128) return fail(h, SPGEMM_UNSUPPORTED, "cache: head_dim must be a multiple of 8, at most 128");
  if (c->pages >= kMaxPages || c->kv_heads > 65535 || c->layers > 65535) return fail(h, SPGEMM_UNSUPPORTED, "cache: too many pages, heads or layers");
  if (c->pages > 0 && (!c->k || !c->v || !c->k_scale || !c->v_scale)) return fail(h, SPGEMM_INVALID_ARG, "cache: null array");
  if (reinterpret_cast<uintptr_t>(c->k) % 16 || reinterpret_cast<uintptr_t>(c->v) % 16) return fail(h, SPGEMM_UNSUPPORTED, "cache: k and v must be 16-byte aligned");
  return SPGEMM_OK;
}

inline int check_table(spgemm_context* h, const spcache* c, const spgemm_csr* t, const int32_t* lens) {
  if (!t) return fail(h, SPGEMM_INVALID_ARG, "table is null");
  if (t->rows < 0 || t->nnz < 0 || !t->rowptr || (t->nnz > 0 && !t->colidx)) return fail(h, SPGEMM_INVALID_ARG, "table: null array or negative size");
  if (t->cols != c->pages) return fail(h, SPGEMM_DIM_MISMATCH, "table: cols is not the number of the cache's pages");
  if (t->rows > 0x3fffffff || t->nnz >= (int64_t(1) << 40)) return fail(h, SPGEMM_UNSUPPORTED, "table: too many rows or entries");
  if (t->rows > 0 && !lens) return fail(h, SPGEMM_INVALID_ARG, "lens is null");
  return SPGEMM_OK;
}

inline int check_layer(spgemm_context* h, const spcache* c, int64_t layer) {
  return layer < 0 || layer >= c->layers ? fail(h, SPGEMM_INVALID_ARG, "no such layer") : SPGEMM_OK;
}

inline int room_of(const spcache* c) { return c->head_dim <= 64 ? 64 : 128; }

inline CacheView view(const spcache* c, int64_t layer) {
  const int64_t cells = c->pages * c->kv_heads;
  const int64_t bytes = cells * SPCACHE_PAGE * room_of(c);
  return {static_cast<unsigned char*>(c->k) + layer * bytes, static_cast<unsigned char*>(c->v) + layer * bytes, c->k_scale + layer * cells,
          c->v_scale + layer * cells, c->pages, c->kv_heads, c->head_dim};
}

inline TableView view(const spgemm_csr* t, const int32_t* lens) { return {t->rowptr, t->colidx, lens, (int)t->rows, t->nnz}; }

}  // namespace spg
