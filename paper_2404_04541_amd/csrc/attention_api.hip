// C ABI of attention and the paged cache (see include/spattn.h): argument checks, scratch memory, launches.  All device work is in the
// attn_*, cache_ and page_kernels headers beside this file.
#include "attn_host.hpp"
#include "attn_plan_kernels.hpp"
#include "attn_backward.hpp"
#include "cache_read.hpp"
#include "page_kernels.hpp"

using namespace spg;

static_assert(kPage == SPCACHE_PAGE, "the header's page");

namespace {

int check_mask(spgemm_context* h, const spattn_mask* m) {
  if (!m) return fail(h, SPGEMM_INVALID_ARG, "mask is null");
  if (m->q_len < 0 || m->k_len < 0 || m->docs < 0 || m->window < 0) return fail(h, SPGEMM_INVALID_ARG, "mask: negative size");
  if (m->causal != 0 && m->causal != 1) return fail(h, SPGEMM_INVALID_ARG, "mask: causal takes 0 or 1");
  if (m->q_len >= kMaxTokens || m->k_len >= kMaxTokens || m->docs >= kMaxTokens) return fail(h, SPGEMM_UNSUPPORTED, "mask: sizes must be below 2^30");
  if (m->docs > 0 && (!m->q_ptr || !m->k_ptr)) return fail(h, SPGEMM_INVALID_ARG, "mask: row pointers are null");
  if (m->docs == 0 && (m->q_ptr || m->k_ptr)) return fail(h, SPGEMM_INVALID_ARG, "mask: row pointers without documents");
  if (m->tiles) {
    const spgemm_csr* t = m->tiles;
    if (t->nnz < 0 || !t->rowptr || (t->nnz > 0 && !t->colidx)) return fail(h, SPGEMM_INVALID_ARG, "pattern: null array or negative size");
    if (t->rows != ceil_div(m->q_len, kPatTile) || t->cols != ceil_div(m->k_len, kPatTile))
      return fail(h, SPGEMM_DIM_MISMATCH, "pattern: rows and cols are not those of the mask's tiles");
  }
  return SPGEMM_OK;
}

PlanView carve_plan(const spattn_mask* m, void* mem, size_t* bytes) {
  const int64_t q_tiles = ceil_div(m->q_len, kPatTile), k_tiles = ceil_div(m->k_len, kPatTile);
  Carve c{static_cast<unsigned char*>(mem)};
  PlanView p{};
  p.error = c.take<int>(1);
  p.totals = c.take<unsigned long long>(2);
  p.rows = c.take<RowBound>(m->q_len);
  p.groups = c.take<GroupBound>(ceil_div(m->q_len, kRowGroup));
  p.cols = c.take<int2>(ceil_div(m->k_len, kKeyTile));
  p.q_order = c.take<int4>(q_tiles);
  if (m->tiles) {
    p.seen_words = (int)ceil_div(k_tiles > 0 ? k_tiles : 1, 32);
    p.seen_by_words = (int)ceil_div(q_tiles > 0 ? q_tiles : 1, 32);
    p.seen = c.take<unsigned>(q_tiles * p.seen_words);
    p.seen_by = c.take<unsigned>(k_tiles * p.seen_by_words);
  }
  *bytes = c.used;
  return p;
}

int check_args(spgemm_context* h, const spattn_args* a) {
  if (!a) return fail(h, SPGEMM_INVALID_ARG, "args is null");
  int rc = check_mask(h, a->mask);
  if (rc) return rc;
  if (!a->plan_mem) return fail(h, SPGEMM_INVALID_ARG, "plan_mem is null");
  if ((rc = check_shape(h, a->dtype, a->heads, a->kv_heads, a->head_dim, a->scale, a->cap))) return rc;
  if ((rc = check_tensor(h, a->q, a->mask->q_len, "q"))) return rc;
  if ((rc = check_tensor(h, a->k, a->mask->k_len, "k"))) return rc;
  if ((rc = check_tensor(h, a->v, a->mask->k_len, "v"))) return rc;
  if (ceil_div(a->mask->q_len, kPatTile) * a->heads + ceil_div(a->mask->k_len, kKeyTile) * a->kv_heads > 0xffffff)   // (2^32 threads are a launch's limit)
    return fail(h, SPGEMM_UNSUPPORTED, "too many tiles");
  return SPGEMM_OK;
}

AttnArgs attn_args(const spattn_args* a, const spattn_tensor& o, const float* lse) {
  size_t bytes;
  AttnArgs g{};
  g.q = view(a->q); g.k = view(a->k); g.v = view(a->v); g.o = view(o);
  g.lse = const_cast<float*>(lse);
  g.q_len = (int)a->mask->q_len; g.k_len = (int)a->mask->k_len;
  g.heads = a->heads; g.group = a->heads / a->kv_heads; g.bytes = a->head_dim * 2;
  g.q_tiles = (int)ceil_div(a->mask->q_len, kPatTile);
  g.plan = carve_plan(a->mask, const_cast<void*>(a->plan_mem), &bytes);
  g.score = {a->scale, a->cap, a->slopes};
  return g;
}

// How many pieces the forward pass's rows may be cut into, with at most `tiles` tiles each: the card holds `resident` workgroups a compute unit; where `blocks` fill it
// nothing is cut (eleven documents, 4096 tokens, 512 workgroups for 512 places, us whole | cut: 38 | 37 and 7 to join), nor where the longest is
// short, else there are places for pieces until it is filled twice.
int split_pieces(spgemm_context* h, int64_t blocks, int64_t tiles, int resident) {
  const int64_t slots = (int64_t)h->num_cus * resident;
  if (blocks == 0 || blocks >= slots || tiles <= 2 * kLeastTiles) return 1;
  const int64_t most = ceil_div(2 * slots, blocks) + 1;
  return (int)(most < 64 ? most : 64);
}
size_t split_bytes(int64_t blocks, int most, int room) {
  return most == 1 ? 0 : align_up((size_t)blocks * most * 128 * room * sizeof(float)) + align_up((size_t)blocks * most * kPatTile * sizeof(float2));
}
Split split_of(spgemm_context* h, int64_t blocks, int most, int resident, int room, void* mem) {
  Carve c{static_cast<unsigned char*>(mem)};
  Split s{most, h->num_cus * resident, nullptr, nullptr};
  if (most > 1) {
    s.sums = c.take<f32x4>(blocks * most * 32 * room);
    s.tops = c.take<float2>(blocks * most * kPatTile);
  }
  return s;
}

CopyArgs copy_args(const spcache* c) {
  CopyArgs a{};
  a.k = static_cast<unsigned char*>(c->k); a.v = static_cast<unsigned char*>(c->v);
  a.k_scale = c->k_scale; a.v_scale = c->v_scale;
  a.pages = c->pages; a.layers = (int)c->layers; a.heads = c->kv_heads;
  a.page_bytes = (int64_t)c->kv_heads * SPCACHE_PAGE * room_of(c);
  return a;
}

// Workgroups that copy at most so many pages: as many as there are pieces, up to eight a compute unit, which is enough to keep the memory busy.
unsigned copy_grid(spgemm_context* h, const CopyArgs& a, int64_t most) {
  const int64_t units = most * a.layers * 2 * ceil_div(a.page_bytes, kCopyPiece), cap = (int64_t)h->num_cus * 8;
  return (unsigned)(units < 1 ? 1 : units < cap ? units : cap);
}

// The copies, at most so many pages; with `out` their kernel also leaves for the host what the ones before it found, and the call waits.
int copy_and_report(spgemm_context* h, CopyArgs& g, int64_t most, PageMoves* out) {
  static_assert(sizeof(PageMoves) <= sizeof(Control), "fits a pinned block");
  const dim3 grid(copy_grid(h, g, most));
  if (!out) {
    k_page_copy<<<grid, dim3(256), 0, h->stream>>>(g);
    return launched(h);
  }
  PinnedLease lease(h->stream);
  if (!lease.p) return fail(h, SPGEMM_ALLOC_FAILED, "pinned memory");
  g.report = reinterpret_cast<PageMoves*>(lease.p);
  lease.written();
  k_page_copy<<<grid, dim3(256), 0, h->stream>>>(g);
  int rc = launched(h);
  if (rc) return rc;
  HIP_TRY(h, hipStreamSynchronize(h->stream));
  lease.waited();
  std::memcpy(out, lease.p, sizeof(PageMoves));
  return SPGEMM_OK;
}

}  // namespace

extern "C" {

size_t spattn_plan_bytes(const spattn_mask* mask) {
  try {
    if (check_mask(nullptr, mask) != SPGEMM_OK) return 0;
  } catch (const std::exception&) {
    return 0;
  }
  size_t bytes;
  carve_plan(mask, nullptr, &bytes);
  return bytes;
}

int spattn_symbolic(spgemm_handle h, const spattn_mask* mask, void* plan_mem, size_t plan_bytes, int32_t* checked) {
  return guarded(h, [&]() -> int {
    int rc = check_mask(h, mask);
    if (rc) return rc;
    size_t need;
    const PlanView p = carve_plan(mask, plan_mem, &need);
    if (!plan_mem) return fail(h, SPGEMM_INVALID_ARG, "plan_mem is null");
    if (plan_bytes < need) return fail(h, SPGEMM_INVALID_ARG, "plan_mem is smaller than spattn_plan_bytes");
    if (reinterpret_cast<uintptr_t>(plan_mem) % 256) return fail(h, SPGEMM_INVALID_ARG, "plan_mem must be 256-byte aligned");
    if ((rc = ensure_device(h))) return rc;
    MaskView m{};
    m.q_len = (int)mask->q_len; m.k_len = (int)mask->k_len; m.docs = (int)mask->docs; m.causal = mask->causal;
    m.window = (int)(mask->window < kMaxTokens ? mask->window : 0);   // (a window of 2^30 hides nothing)
    m.q_ptr = mask->q_ptr; m.k_ptr = mask->k_ptr; m.prefix = mask->prefix;
    if (mask->tiles) { m.pat_ptr = mask->tiles->rowptr; m.pat_col = mask->tiles->colidx; m.pat_nnz = mask->tiles->nnz; }
    const int64_t flag_blocks = mask->tiles ? ceil_div(ceil_div(mask->q_len, kPatTile), 4) : 0;
    if (mask->q_len <= kSmallMask && mask->k_len <= kSmallMask) {
      k_plan_small<<<dim3(1), dim3(kSmallMask), 0, h->stream>>>(m, p);
      if (flag_blocks) k_plan_pattern<<<dim3((unsigned)flag_blocks), dim3(256), 0, h->stream>>>(m, p);
    } else {
      k_plan_rows<<<dim3((unsigned)ceil_div(mask->q_len > 0 ? mask->q_len : 1, 256)), dim3(256), 0, h->stream>>>(m, p);
      k_plan_cols<<<dim3((unsigned)(ceil_div(ceil_div(mask->k_len, kKeyTile), 4) + flag_blocks + 1)), dim3(256), 0, h->stream>>>(m, p);
    }
    if ((rc = launched(h))) return rc;
    if (!checked) return SPGEMM_OK;
    int32_t error = 0;
    if ((rc = fetch(h, p.error, &error))) return rc;
    *checked = error ? 0 : 1;
    return error ? fail(h, SPGEMM_INVALID_INPUT, "mask: documents or pattern out of range or not ascending") : SPGEMM_OK;
  });
}

int spattn_forward(spgemm_handle h, const spattn_args* a, spattn_tensor o, float* lse) {
  return guarded(h, [&]() -> int {
    int rc = check_args(h, a);
    if (rc) return rc;
    if ((rc = check_tensor(h, o, a->mask->q_len, "o"))) return rc;
    if (a->mask->q_len == 0) return SPGEMM_OK;
    if (!lse) return fail(h, SPGEMM_INVALID_ARG, "lse is null");
    if ((rc = ensure_device(h))) return rc;
    AttnArgs g = attn_args(a, o, lse);
    const int64_t blocks = (int64_t)g.q_tiles * g.heads;
    const int room = a->head_dim <= 64 ? 64 : 128, resident = room == 64 ? 4 : 2;
    const int most = split_pieces(h, blocks, ceil_div(a->mask->k_len, kKeyTile), resident);
    void* mem = nullptr;
    if (most > 1 && (rc = scratch(h, split_bytes(blocks, most, room), &mem))) return rc;
    g.split = split_of(h, blocks, most, resident, room, mem);
    const dim3 grid((unsigned)blocks, (unsigned)most);
    dispatch(a->dtype, a->head_dim, a->cap > 0, a->slopes != nullptr, [&](auto type, auto dim, auto cap, auto bias) {
      using T = decltype(type);
      if constexpr (cap() && !bias() && std::is_same<T, bf16_t>::value) {
        if (a->cap * kLog2e <= kBoundedCap2) {
          k_attn_fwd<T, dim(), true, false, true><<<grid, dim3(256), 0, h->stream>>>(g);
          return;
        }
      }
      k_attn_fwd<T, dim(), cap(), bias(), false><<<grid, dim3(256), 0, h->stream>>>(g);
    });
    if (most > 1)
      dispatch(a->dtype, a->head_dim, false, false, [&](auto type, auto dim, auto, auto) {
        k_attn_join<decltype(type), dim()><<<dim3((unsigned)blocks, dim() / 32), dim3(256), 0, h->stream>>>(g);
      });
    return launched(h);
  });
}

int spattn_backward(spgemm_handle h, const spattn_args* a, spattn_tensor o, const float* lse, spattn_tensor d_o, spattn_tensor dq,
                    spattn_tensor dk, spattn_tensor dv) {
  return guarded(h, [&]() -> int {
    int rc = check_args(h, a);
    if (rc) return rc;
    const int64_t q_len = a->mask->q_len, k_len = a->mask->k_len;
    if ((rc = check_tensor(h, o, q_len, "o")) || (rc = check_tensor(h, d_o, q_len, "d_o")) || (rc = check_tensor(h, dq, q_len, "dq")) ||
        (rc = check_tensor(h, dk, k_len, "dk")) || (rc = check_tensor(h, dv, k_len, "dv")))
      return rc;
    if (q_len > 0 && !lse) return fail(h, SPGEMM_INVALID_ARG, "lse is null");
    if ((rc = ensure_device(h))) return rc;
    const int64_t q_tiles = ceil_div(q_len, kPatTile), k_tiles = ceil_div(k_len, kKeyTile), both = q_tiles * a->heads + k_tiles * a->kv_heads;
    if (both == 0) return SPGEMM_OK;
    const int room = a->head_dim <= 64 ? 64 : 128, resident = room == 64 ? 3 : 2;
    // Where the card's places are filled less than four times, long tiles are cut: pieces_of bounds how many more workgroups that makes, and how many
    // pieces have to be joined.  us whole | cut, 16 heads on 4: 32 documents of 128 tokens and one of 4096 478 | 331, eleven of 4096 together 179 | 97; 16 heads on 16 of 64 channels,
    // 4096 tokens in two documents 107 | 111.
    int64_t slots = (int64_t)h->num_cus * resident;
    if (both >= 4 * slots || (ceil_div(q_len, kQueryTile) * (a->heads / a->kv_heads) <= 2 * kLeastTiles && ceil_div(k_len, kKeyTile) <= 2 * kLeastTiles)) slots = 0;
    const int64_t more = 2 * slots / 3 + 1, cells = slots ? 2 * more : 0;
    Carve c{nullptr};
    AttnGrads r{view(d_o), view(dq), view(dk), view(dv)};
    auto carve = [&] {
      r.facts = c.take<RowFacts>(a->heads * q_tiles * (kPatTile / kQueryTile));
      r.k_list = c.take<int4>(k_tiles + more);
      r.q_list = c.take<int4>(q_tiles + more);
      r.counts = c.take<Counts>(1);
      r.sums = c.take<f32x4>(cells * 32 * room);
    };
    carve();
    void* mem = nullptr;
    if ((rc = scratch(h, c.used, &mem))) return rc;
    c = Carve{static_cast<unsigned char*>(mem)};
    carve();
    r.slots = (int)slots;
    r.more = (int)more;
    AttnArgs g = attn_args(a, o, lse);
    auto launch = [&](auto type, auto dim, auto cap, auto bias) {
      using T = decltype(type);
      k_attn_facts<T, dim()><<<dim3((unsigned)g.q_tiles * (kPatTile / kQueryTile) + 2, (unsigned)a->heads), dim3(256), 0, h->stream>>>(g, r);
      k_attn_back<T, dim(), cap(), bias()><<<dim3((unsigned)(slots ? both + more : both)), dim3(256), 0, h->stream>>>(BackArgs{g, r});
      if (slots) k_attn_back_join<T, dim(), cap()><<<dim3((unsigned)cells, dim() / 32), dim3(256), 0, h->stream>>>(g, r);
    };
    dispatch(a->dtype, a->head_dim, a->cap > 0, a->slopes != nullptr, launch);
    return launched(h);
  });
}

int spcache_append(spgemm_handle h, const spcache* c, int64_t layer, const spgemm_csr* table, const int32_t* lens, const int64_t* new_ptr,
                   int64_t tokens, int32_t dtype, spattn_tensor k, spattn_tensor v) {
  return guarded(h, [&]() -> int {
    int rc = check_cache(h, c);
    if (rc) return rc;
    if ((rc = check_table(h, c, table, lens)) || (rc = check_layer(h, c, layer))) return rc;
    if (dtype != SPATTN_F16 && dtype != SPATTN_BF16) return fail(h, SPGEMM_INVALID_ARG, "unknown dtype");
    if (tokens < 0) return fail(h, SPGEMM_INVALID_ARG, "negative number of tokens");
    if (tokens >= kMaxTokens) return fail(h, SPGEMM_UNSUPPORTED, "tokens must be below 2^30");
    if ((rc = check_tensor(h, k, tokens, "k")) || (rc = check_tensor(h, v, tokens, "v"))) return rc;
    if (tokens == 0 || table->rows == 0) return SPGEMM_OK;
    if (!new_ptr) return fail(h, SPGEMM_INVALID_ARG, "new_ptr is null");
    const int64_t slots = tokens / SPCACHE_PAGE + 2 * table->rows;
    if (slots > 0xffffff) return fail(h, SPGEMM_UNSUPPORTED, "too many sequences");   // (2^32 threads are a launch's limit)
    if ((rc = ensure_device(h))) return rc;
    const AppendArgs a{view(c, layer), view(table, lens), new_ptr, view(k), view(v), tokens};
    const dim3 grid((unsigned)slots, (unsigned)c->kv_heads);
    dispatch(dtype, c->head_dim, false, false, [&](auto type, auto dim, auto, auto) {
      k_cache_append<decltype(type), dim()><<<grid, dim3(256), 0, h->stream>>>(a);
    });
    return launched(h);
  });
}

int spcache_read(spgemm_handle h, const spcache* c, int64_t layer, const spgemm_csr* table, const int32_t* lens, const int64_t* ptr, int64_t tokens, int32_t dtype,
                 spattn_tensor k, spattn_tensor v) {
  return guarded(h, [&]() -> int {
    int rc = check_cache(h, c);
    if (rc) return rc;
    if ((rc = check_table(h, c, table, lens)) || (rc = check_layer(h, c, layer))) return rc;
    if (dtype != SPATTN_F16 && dtype != SPATTN_BF16) return fail(h, SPGEMM_INVALID_ARG, "unknown dtype");
    if (tokens < 0) return fail(h, SPGEMM_INVALID_ARG, "negative number of tokens");
    if (tokens >= kMaxTokens) return fail(h, SPGEMM_UNSUPPORTED, "tokens must be below 2^30");
    if ((rc = check_tensor(h, k, tokens, "k")) || (rc = check_tensor(h, v, tokens, "v"))) return rc;
    if (tokens == 0 || table->rows == 0) return SPGEMM_OK;
    if (!ptr) return fail(h, SPGEMM_INVALID_ARG, "ptr is null");
    const int64_t slots = tokens / SPCACHE_PAGE + 2 * table->rows;
    if (slots > 0xffffff) return fail(h, SPGEMM_UNSUPPORTED, "too many sequences");   // (2^32 threads are a launch's limit)
    if ((rc = ensure_device(h))) return rc;
    const ReadArgs a{view(c, layer), view(table, lens), ptr, view(k), view(v), tokens};
    const dim3 grid((unsigned)slots, (unsigned)c->kv_heads);
    dispatch(dtype, c->head_dim, false, false, [&](auto type, auto dim, auto, auto) {
      k_cache_read<decltype(type), dim()><<<grid, dim3(256), 0, h->stream>>>(a);
    });
    return launched(h);
  });
}

int spcache_attend(spgemm_handle h, const spcache* c, int64_t layer, const spgemm_csr* table, const int32_t* lens, int64_t q_len, int32_t heads,
                   int32_t dtype, float scale, float cap, const float* slopes, int64_t window, spattn_tensor q, spattn_tensor o) {
  return guarded(h, [&]() -> int {
    int rc = check_cache(h, c);
    if (rc) return rc;
    if ((rc = check_table(h, c, table, lens)) || (rc = check_layer(h, c, layer))) return rc;
    if ((rc = check_shape(h, dtype, heads, c->kv_heads, c->head_dim, scale, cap))) return rc;
    if (q_len < 0 || window < 0) return fail(h, SPGEMM_INVALID_ARG, "negative q_len or window");
    const int64_t n = table->rows;
    if (q_len >= kMaxTokens || n * q_len >= kMaxTokens) return fail(h, SPGEMM_UNSUPPORTED, "tokens must be below 2^30");
    if ((rc = check_tensor(h, q, n * q_len, "q")) || (rc = check_tensor(h, o, n * q_len, "o"))) return rc;
    const int64_t tiles = ceil_div(q_len * (heads / c->kv_heads), kRows);
    if (q_len * heads > 65535) return fail(h, SPGEMM_UNSUPPORTED, "too many query rows for a sequence");
    if (n * q_len == 0) return SPGEMM_OK;
    if ((rc = ensure_device(h))) return rc;
    AttendArgs a{};
    a.c = view(c, layer); a.t = view(table, lens); a.q = view(q); a.o = view(o);
    a.q_len = (int)q_len; a.heads = heads; a.group = heads / c->kv_heads;
    a.tiles = (int)tiles;
    a.window = (int)(window < kMaxTokens ? window : 0);
    a.score = {scale, cap, slopes};
    // Pages of a workgroup: so many that the workgroups fill the card twice (three are resident on a compute unit), at least one for every wave.  128
    // sequences of 3 to 8192 tokens, us filling it once | twice: 51 | 47 and 7 to join; four of 131 071: 172 | 176 and 6.
    const int64_t want = (int64_t)h->num_cus * 6;
    int64_t chunk = ceil_div(table->nnz * c->kv_heads * tiles, want);
    chunk = chunk < 4 ? 4 : ceil_div(chunk, 4) * 4;
    a.chunk = (int)chunk;
    const int64_t slots = table->nnz / chunk + n;
    if (slots > 0xffffff) return fail(h, SPGEMM_UNSUPPORTED, "too many pages");   // (2^32 threads are a launch's limit)
    const int64_t cells = slots * c->kv_heads * tiles;
    const int room = room_of(c);
    const size_t part = align_up((size_t)cells * kRows * room * sizeof(float)), ml = align_up((size_t)cells * kRows * sizeof(float2));
    void* mem = nullptr;
    if ((rc = scratch(h, part + ml, &mem))) return rc;
    a.part = static_cast<float*>(mem);
    a.part_ml = reinterpret_cast<float2*>(static_cast<unsigned char*>(mem) + part);
    const dim3 grid((unsigned)slots, (unsigned)c->kv_heads, (unsigned)tiles), join((unsigned)n, (unsigned)(q_len * heads));
    dispatch(dtype, c->head_dim, cap > 0, slopes != nullptr, [&](auto type, auto dim, auto capped, auto bias) {
      k_cache_attend<decltype(type), dim(), capped(), bias()><<<grid, dim3(256), 0, h->stream>>>(a);
    });
    dispatch(dtype, c->head_dim, false, false, [&](auto type, auto dim, auto, auto) {
      k_cache_join<decltype(type), dim()><<<join, dim3(256), 0, h->stream>>>(a);
    });
    return launched(h);
  });
}

int spcache_fork(spgemm_handle h, const spcache* c, const spgemm_csr* table, const int32_t* lens, int64_t n_out, const int32_t* parent,
                 const int32_t* new_lens, int64_t* out_rowptr, int32_t* out_pages, int64_t room, int32_t* refs, int64_t* nnz_out) {
  return guarded(h, [&]() -> int {
    int rc = check_cache(h, c);
    if (rc) return rc;
    if ((rc = check_table(h, c, table, lens))) return rc;
    if (n_out < 0 || room < 0) return fail(h, SPGEMM_INVALID_ARG, "negative size");
    if (n_out > 0x3fffffff) return fail(h, SPGEMM_UNSUPPORTED, "too many rows");
    if ((n_out > 0 && (!parent || !new_lens)) || !out_rowptr || (room > 0 && !out_pages) || (c->pages > 0 && !refs))
      return fail(h, SPGEMM_INVALID_ARG, "null array");
    if ((rc = ensure_device(h))) return rc;
    const int64_t blocks = ceil_div(c->pages, kPageBlock);
    ForkArgs a{};
    auto lay = [&](void* mem) {
      Carve w{static_cast<unsigned char*>(mem)};
      a.out = w.take<PageMoves>(1);
      a.owner = w.take<int32_t>(c->pages);
      a.fresh = w.take<int64_t>(n_out);
      a.src = w.take<int32_t>(n_out);
      a.dst = w.take<int32_t>(n_out);
      a.used.words = w.take<unsigned>(blocks * (kPageBlock / 32));
      a.used.counts = w.take<unsigned>(blocks);
      return w.used;
    };
    void* mem = nullptr;
    if ((rc = scratch(h, lay(nullptr), &mem))) return rc;
    lay(mem);
    a.t = view(table, lens);
    a.pages = a.used.pages = c->pages;
    a.parent = parent; a.new_lens = new_lens; a.rows = (int)n_out;
    a.ptr = out_rowptr; a.page = out_pages; a.room = room; a.refs = refs;
    const unsigned rows4 = (unsigned)ceil_div(n_out > 0 ? n_out : 1, 4);
    const int64_t clear = blocks < h->num_cus ? blocks : h->num_cus;
    k_fork_rows<<<dim3((unsigned)(1 + (clear > 0 ? clear : 1))), dim3(1024), 0, h->stream>>>(a);
    k_fork_gather<<<dim3(rows4), dim3(256), 0, h->stream>>>(a);
    k_fork_flags<<<dim3((unsigned)(blocks + 1)), dim3(1024), 0, h->stream>>>(a);
    k_fork_assign<<<dim3(rows4), dim3(256), 0, h->stream>>>(a);
    CopyArgs g = copy_args(c);
    g.src = a.src; g.dst = a.dst;
    g.in = a.out;
    PageMoves out{};
    if ((rc = copy_and_report(h, g, n_out, nnz_out ? &out : nullptr))) return rc;
    if (!nnz_out) return SPGEMM_OK;
    *nnz_out = out.nnz;
    if (out.error == kForkPages) return fail(h, SPGEMM_ALLOC_FAILED, "the cache has no page left");
    return out.error ? fail(h, SPGEMM_INVALID_INPUT, "a parent, length or page out of range, or too little room for the table") : SPGEMM_OK;
  });
}

int spcache_compact(spgemm_handle h, const spcache* c, const spgemm_csr* table, int32_t* out_pages, int64_t* live) {
  return guarded(h, [&]() -> int {
    int rc = check_cache(h, c);
    if (rc) return rc;
    static const int32_t none = 0;
    if ((rc = check_table(h, c, table, &none))) return rc;
    if (table->nnz > 0 && !out_pages) return fail(h, SPGEMM_INVALID_ARG, "out_pages is null");
    if ((rc = ensure_device(h))) return rc;
    const int64_t blocks = ceil_div(c->pages, kPageBlock);
    CompactArgs a{};
    auto lay = [&](void* mem) {
      Carve w{static_cast<unsigned char*>(mem)};
      a.out = w.take<PageMoves>(1);
      a.rank = w.take<int32_t>(c->pages);
      a.movers = w.take<int32_t>(c->pages / 2 + 1);
      a.holes = w.take<int32_t>(c->pages / 2 + 1);
      a.live.words = w.take<unsigned>(blocks * (kPageBlock / 32));
      a.live.counts = w.take<unsigned>(blocks);
      return w.used;
    };
    void* mem = nullptr;
    if ((rc = scratch(h, lay(nullptr), &mem))) return rc;
    lay(mem);
    a.t = view(table, nullptr);
    a.live.pages = c->pages;
    a.page = out_pages;
    const int64_t cap = (int64_t)h->num_cus * 8;
    auto grid = [&](int64_t n) { const int64_t g = ceil_div(n > 0 ? n : 1, 256); return dim3((unsigned)(g < cap ? g : cap)); };
    k_compact_clear<<<grid(blocks * (kPageBlock / 32)), dim3(256), 0, h->stream>>>(a);
    k_compact_mark<<<grid(table->nnz), dim3(256), 0, h->stream>>>(a);
    if (blocks > 0) {
      k_compact_count<<<dim3((unsigned)ceil_div(blocks, 4)), dim3(256), 0, h->stream>>>(a);
      k_compact_map<<<dim3((unsigned)blocks), dim3(kPageBlock), 0, h->stream>>>(a);
    }
    CopyArgs g = copy_args(c);
    g.src = a.movers; g.dst = a.holes;
    g.in = a.out;
    g.old_page = table->colidx; g.rank = a.rank; g.new_page = out_pages; g.nnz = table->nnz;
    PageMoves out{};
    if ((rc = copy_and_report(h, g, c->pages / 2, live ? &out : nullptr))) return rc;
    if (!live) return SPGEMM_OK;
    *live = out.live;
    return out.error ? fail(h, SPGEMM_INVALID_INPUT, "a page of the table is out of range") : SPGEMM_OK;
  });
}

int spcache_copy(spgemm_handle h, const spcache* c, int64_t n, const int32_t* src, const int32_t* dst) {
  return guarded(h, [&]() -> int {
    int rc = check_cache(h, c);
    if (rc) return rc;
    if (n < 0) return fail(h, SPGEMM_INVALID_ARG, "negative number of pages");
    if (n == 0) return SPGEMM_OK;
    if (!src || !dst) return fail(h, SPGEMM_INVALID_ARG, "null array");
    if (n >= kMaxPages) return fail(h, SPGEMM_UNSUPPORTED, "more pairs than a cache has pages");
    if ((rc = ensure_device(h))) return rc;
    CopyArgs g = copy_args(c);
    g.src = src; g.dst = dst; g.count = n;
    return copy_and_report(h, g, n, nullptr);
  });
}

}  // extern "C"
