// C ABI of drafted tokens over the paged cache (see include/spdraft.h): argument checks, scratch memory, launches.  All device work is in the draft_ headers beside this file.
#include "../../include/spdraft.h"

#include "attn_host.hpp"
#include "draft_attend.hpp"
#include "draft_keep.hpp"
#include "draft_verify.hpp"

using namespace spg;

static_assert(kMostNodes == SPDRAFT_MOST, "the header's trees");

namespace {

constexpr int64_t kMaxNodes = int64_t(1) << 24;

int check_trees(spgemm_context* h, const spdraft_trees* t) {
  if (!t) return fail(h, SPGEMM_INVALID_ARG, "trees is null");
  if (t->rows < 0 || t->tokens < 0) return fail(h, SPGEMM_INVALID_ARG, "trees: negative size");
  if (t->tokens >= kMaxNodes || t->rows >= kMaxNodes) return fail(h, SPGEMM_UNSUPPORTED, "trees: rows and tokens must be below 2^24");
  if (t->most < 1) return fail(h, SPGEMM_INVALID_ARG, "trees: most must be positive");
  if (t->most > SPDRAFT_MOST) return fail(h, SPGEMM_UNSUPPORTED, "trees: more than 256 nodes");
  if (!t->ptr) return fail(h, SPGEMM_INVALID_ARG, "trees: ptr is null");
  return SPGEMM_OK;
}

int check_plan(spgemm_context* h, const spdraft_trees* t, const void* plan_mem) {
  const int rc = check_trees(h, t);
  if (rc) return rc;
  return plan_mem ? SPGEMM_OK : fail(h, SPGEMM_INVALID_ARG, "plan_mem is null");
}

TreeView carve_trees(const spdraft_trees* t, void* mem, size_t* bytes, int** error) {
  Carve c{static_cast<unsigned char*>(mem)};
  TreeView v{};
  v.ptr = t->ptr; v.rows = (int)t->rows; v.most = t->most; v.words = (int)ceil_div(t->most, 64); v.tokens = t->tokens;
  *error = c.take<int>(1);
  v.node = c.take<TreeNode>(t->tokens);
  v.place = c.take<int4>(t->tokens);
  v.up = c.take<unsigned long long>(t->tokens * v.words);
  *bytes = c.used;
  return v;
}
TreeView view(const spdraft_trees* t, const void* plan_mem) {
  size_t bytes;
  int* error;
  return carve_trees(t, const_cast<void*>(plan_mem), &bytes, &error);
}

// The rows of a table and of the trees are the same sequences.
int check_rows(spgemm_context* h, const spgemm_csr* table, const spdraft_trees* t) {
  return table->rows == t->rows ? SPGEMM_OK : fail(h, SPGEMM_DIM_MISMATCH, "table and trees: the numbers of sequences differ");
}

}  // namespace

extern "C" {

size_t spdraft_plan_bytes(const spdraft_trees* t) {
  try {
    if (check_trees(nullptr, t) != SPGEMM_OK) return 0;
  } catch (const std::exception&) {
    return 0;
  }
  size_t bytes;
  int* error;
  carve_trees(t, nullptr, &bytes, &error);
  return bytes;
}

int spdraft_symbolic(spgemm_handle h, const spdraft_trees* t, void* plan_mem, size_t plan_bytes, int32_t* checked) {
  return guarded(h, [&]() -> int {
    int rc = check_plan(h, t, plan_mem);
    if (rc) return rc;
    size_t need;
    int* error;
    const TreeView v = carve_trees(t, plan_mem, &need, &error);
    if (plan_bytes < need) return fail(h, SPGEMM_INVALID_ARG, "plan_mem is smaller than spdraft_plan_bytes");
    if (reinterpret_cast<uintptr_t>(plan_mem) % 256) return fail(h, SPGEMM_INVALID_ARG, "plan_mem must be 256-byte aligned");
    if (t->tokens > 0 && !t->parent) return fail(h, SPGEMM_INVALID_ARG, "trees: parent is null");
    if ((rc = ensure_device(h))) return rc;
    if (t->rows > 0 && t->tokens > 0) k_trees<<<dim3((unsigned)t->rows), dim3(kMostNodes), 0, h->stream>>>(v, t->parent);
    if (checked) k_trees_check<<<dim3(1), dim3(1024), 0, h->stream>>>(v, t->parent, error);
    if ((rc = launched(h))) return rc;
    if (!checked) return SPGEMM_OK;
    int32_t bad = 0;
    if ((rc = fetch(h, error, &bad))) return rc;
    *checked = bad ? 0 : 1;
    return bad ? fail(h, SPGEMM_INVALID_INPUT, "trees: ptr out of range, too many nodes, or a parent that is not an earlier node") : SPGEMM_OK;
  });
}

int spdraft_attend(spgemm_handle h, const spcache* c, int64_t layer, const spgemm_csr* table, const int32_t* lens, const spdraft_trees* t, const void* plan_mem,
                   int32_t heads, int32_t dtype, float scale, float cap, const float* slopes, int64_t window, spattn_tensor q, spattn_tensor o) {
  return guarded(h, [&]() -> int {
    int rc = check_cache(h, c);
    if (rc) return rc;
    if ((rc = check_table(h, c, table, lens)) || (rc = check_layer(h, c, layer)) || (rc = check_plan(h, t, plan_mem)) || (rc = check_rows(h, table, t))) return rc;
    if ((rc = check_shape(h, dtype, heads, c->kv_heads, c->head_dim, scale, cap))) return rc;
    if (window < 0) return fail(h, SPGEMM_INVALID_ARG, "negative window");
    if ((rc = check_tensor(h, q, t->tokens, "q")) || (rc = check_tensor(h, o, t->tokens, "o"))) return rc;
    if (t->tokens * heads > 0xffffff) return fail(h, SPGEMM_UNSUPPORTED, "too many nodes and heads");      // (2^32 threads are a launch's limit)
    const int64_t n = table->rows;
    if (n == 0 || t->tokens == 0) return SPGEMM_OK;
    if ((rc = ensure_device(h))) return rc;
    TreeAttendArgs a{};
    a.c = view(c, layer); a.t = view(table, lens); a.trees = view(t, plan_mem); a.q = view(q); a.o = view(o);
    a.heads = heads; a.group = heads / c->kv_heads;
    const int64_t rows = (int64_t)t->most * a.group;
    a.tiles = (int)ceil_div(rows, kTreeRows);
    a.part_rows = (int)(rows < kTreeRows ? ceil_div(rows, 32) * 32 : kTreeRows);
    a.window = (int)(window < kMaxTokens ? window : 0);
    a.score = {scale, cap, slopes};
    const int room = room_of(c);
    a.places = h->num_cus * tree_resident(room);
    // Up to kMostEven sequences every workgroup finds its piece by itself; beyond, places of chunks are found by the table's row pointers.
    const int64_t units = n * c->kv_heads * a.tiles, work = table->nnz * c->kv_heads * a.tiles;
    int64_t pieces, cells;
    if (n <= kMostEven) {
      a.chunk = 0;
      pieces = most_pieces(work, units, a.places);
      cells = most_cells(work, a.places);
    } else {
      a.chunk = chunk_pages(work, a.places);
      pieces = (table->nnz / a.chunk + n) * c->kv_heads * a.tiles;
      cells = chunk_cell(table->nnz, a.chunk) * c->kv_heads * a.tiles;
    }
    if (pieces > 0xffffff - 128) return fail(h, SPGEMM_UNSUPPORTED, "too many pages");      // (2^32 threads are a launch's limit)
    const size_t part = align_up((size_t)cells * a.part_rows * room * sizeof(float)), ml = align_up((size_t)cells * a.part_rows * sizeof(float2)), cuts = n <= kMostEven ? (size_t)n * sizeof(int4) : 0;
    void* mem = nullptr;
    if ((rc = scratch(h, part + ml + cuts, &mem))) return rc;
    a.cells = cells;
    a.part = static_cast<float*>(mem);
    a.part_ml = reinterpret_cast<float2*>(static_cast<unsigned char*>(mem) + part);
    a.cuts = reinterpret_cast<int4*>(static_cast<unsigned char*>(mem) + part + ml);
    const dim3 grid((unsigned)(ceil_div(pieces, 128) * 128)), join((unsigned)t->tokens, (unsigned)c->kv_heads);
    dispatch(dtype, c->head_dim, cap > 0, slopes != nullptr, [&](auto type, auto dim, auto capped, auto bias) {
      k_tree_attend<decltype(type), dim(), capped(), bias()><<<grid, dim3(256), 0, h->stream>>>(a);
    });
    dispatch(dtype, c->head_dim, false, false, [&](auto type, auto dim, auto, auto) {
      k_tree_join<decltype(type), dim()><<<join, dim3(256), 0, h->stream>>>(a);
    });
    return launched(h);
  });
}

int spdraft_verify(spgemm_handle h, const spdraft_trees* t, const void* plan_mem, int64_t vocab, int32_t dtype, spdraft_rows target, spdraft_rows draft, const int32_t* ids,
                   const float* u, int32_t* path, int32_t* kept, int32_t* next) {
  return guarded(h, [&]() -> int {
    int rc = check_plan(h, t, plan_mem);
    if (rc) return rc;
    if (vocab < 1) return fail(h, SPGEMM_INVALID_ARG, "vocab must be positive");
    if (vocab > (int64_t(1) << 24)) return fail(h, SPGEMM_UNSUPPORTED, "vocab must be at most 2^24");
    if (dtype != SPATTN_F16 && dtype != SPATTN_BF16 && dtype != SPDRAFT_F32) return fail(h, SPGEMM_INVALID_ARG, "unknown dtype");
    if (target.stride < 0 || draft.stride < 0) return fail(h, SPGEMM_INVALID_ARG, "negative stride");
    const uintptr_t size = dtype == SPDRAFT_F32 ? 4 : 2;
    if (reinterpret_cast<uintptr_t>(target.data) % size || reinterpret_cast<uintptr_t>(draft.data) % size) return fail(h, SPGEMM_INVALID_ARG, "rows must be aligned to their elements");
    if (t->rows == 0) return SPGEMM_OK;
    if (!kept || !next || (t->tokens > 0 && (!target.data || !ids || !u || !path))) return fail(h, SPGEMM_INVALID_ARG, "null array");
    if (t->tokens > 0x3fffff) return fail(h, SPGEMM_UNSUPPORTED, "too many nodes");      // (2^32 threads are a launch's limit)
    if ((rc = ensure_device(h))) return rc;
    VerifyArgs a{};
    a.trees = view(t, plan_mem);
    a.target = target.data; a.target_stride = target.stride;
    a.draft = draft.data; a.draft_stride = draft.stride;
    a.vocab = (int)vocab; a.ids = ids; a.u = u;
    a.path = path; a.kept = kept; a.next = next;
    void* mem = nullptr;
    if ((rc = scratch(h, (size_t)t->tokens * sizeof(int2), &mem))) return rc;
    a.onward = static_cast<int2*>(mem);
    if (t->tokens > 0) {
      const dim3 grid((unsigned)t->tokens), block(kVerifyThreads);
      auto nodes = [&](auto type) {
        using T = decltype(type);
        if (draft.data) k_verify_nodes<T, true><<<grid, block, 0, h->stream>>>(a);
        else k_verify_nodes<T, false><<<grid, block, 0, h->stream>>>(a);
      };
      if (dtype == SPDRAFT_F32) nodes(float{});
      else if (dtype == SPATTN_BF16) nodes(bf16_t{});
      else nodes(f16_t{});
    }
    k_verify_walk<<<dim3((unsigned)ceil_div(t->rows, 4)), dim3(256), 0, h->stream>>>(a);
    return launched(h);
  });
}

int spdraft_keep(spgemm_handle h, const spcache* c, const spgemm_csr* table, const int32_t* lens, const spdraft_trees* t, const int32_t* path, const int32_t* kept,
                 int32_t* new_lens) {
  return guarded(h, [&]() -> int {
    int rc = check_cache(h, c);
    if (rc) return rc;
    if ((rc = check_table(h, c, table, lens)) || (rc = check_trees(h, t)) || (rc = check_rows(h, table, t))) return rc;
    if (t->rows == 0) return SPGEMM_OK;
    if (!kept || !new_lens || (t->tokens > 0 && !path)) return fail(h, SPGEMM_INVALID_ARG, "null array");
    if (c->layers * 2 > 65535) return fail(h, SPGEMM_UNSUPPORTED, "too many layers");
    if (t->rows * c->kv_heads * c->layers * 2 > 0xffffff) return fail(h, SPGEMM_UNSUPPORTED, "too many sequences, heads and layers");      // (2^32 threads are a launch's limit)
    auto overlaps = [&](const int32_t* p, int64_t n) { return new_lens < p + n && p < new_lens + t->rows; };
    if (overlaps(lens, t->rows) || overlaps(kept, t->rows) || overlaps(path, t->tokens)) return fail(h, SPGEMM_INVALID_ARG, "new_lens must not overlap lens, path or kept");
    if ((rc = ensure_device(h))) return rc;
    KeepArgs a{};
    a.data[0] = static_cast<unsigned char*>(c->k); a.data[1] = static_cast<unsigned char*>(c->v);
    a.scale[0] = c->k_scale; a.scale[1] = c->v_scale;
    a.pages = c->pages; a.layers = (int)c->layers; a.heads = c->kv_heads; a.bytes8 = c->head_dim;
    a.t = view(table, lens);
    a.trees = view(t, nullptr);
    a.path = path; a.kept = kept; a.new_lens = new_lens;
    const dim3 grid((unsigned)t->rows, (unsigned)c->kv_heads, (unsigned)ceil_div(2 * c->layers, 4));
    if (room_of(c) == 64) k_draft_keep<64><<<grid, dim3(256), 0, h->stream>>>(a);
    else k_draft_keep<128><<<grid, dim3(256), 0, h->stream>>>(a);
    return launched(h);
  });
}

}  // extern "C"
