// C ABI of libspork (declared in include/spork.h): the step whose lengths live
// on the GPU. Argument checks and dispatch of the block tables, the batched
// block copy and the attention of a chunk of new tokens.
#include <cfloat>
#include <climits>
#include <cmath>
#include <cstdint>

#include "capi_common.h"
#include "chunk_kernels.h"
#include "spork.h"
#include "tables_kernels.h"

namespace {

using namespace spork::capi;

// A launch has fewer than 2^32 threads: so many workgroups of 256.
constexpr int64_t kMostGroups = (int64_t{1} << 24) - 1;

// Loops over positions and table columns count in 32 bits and run a step of up to
// 1,024 past the last, or look a few of 256 ahead: so far below 2^31 none wraps.
constexpr int64_t kHeadroom = 4096;

bool aligned256(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 255) == 0; }

// The sizes that every tables call checks.
int check_tables(const spork_tables* t) {
  if (t == nullptr) return fail(SPORK_E_INVAL, "tables is NULL");
  if (t->num_blocks <= 0 || t->block_size <= 0 || t->n_seqs <= 0 || t->max_blocks <= 0)
    return fail(SPORK_E_INVAL, "num_blocks, block_size, n_seqs and max_blocks must be positive");
  if (t->n_seqs * (int64_t{1} + t->max_blocks) >= INT_MAX ||
      static_cast<int64_t>(t->max_blocks) * t->block_size > INT_MAX || t->max_blocks > INT_MAX - kHeadroom)
    return fail(SPORK_E_UNSUPPORTED,
                "n_seqs * (max_blocks + 1) must be below 2^31 - 1, max_blocks * block_size below 2^31 and max_blocks below 2^31 - 4096");
  return SPORK_OK;
}

int check_tables_memory(const spork_tables* t) {
  const int rc = check_tables(t);
  if (rc != SPORK_OK) return rc;
  if (!t->table || !t->held || !t->refcount || !t->free_queue || !t->queue)
    return fail(SPORK_E_INVAL, "a pointer of tables is NULL");
  return SPORK_OK;
}

int check_tables_workspace(const spork_tables* t, const void* workspace, size_t ws_bytes) {
  if (workspace == nullptr || !aligned256(workspace))
    return fail(SPORK_E_INVAL, "workspace must be non-NULL and 256-byte aligned");
  if (ws_bytes < spork::tables_workspace_bytes(t->num_blocks, t->n_seqs))
    return fail(SPORK_E_CAPACITY, "workspace is smaller than spork_tables_workspace_bytes");
  return SPORK_OK;
}

// What a step writes lies apart from all else that it is given: its launches read
// lengths, parents and tables while others of their workgroups write outputs.
int check_step_apart(const spork::TablesArgs& a, const void* workspace) {
  const size_t n = static_cast<size_t>(a.n_seqs), nb = static_cast<size_t>(a.num_blocks), tokens = static_cast<size_t>(a.max_tokens);
  const struct {
    const void* at;
    size_t bytes;
  } runs[] = {{a.table, 4 * n * a.max_blocks}, {a.held, 4 * n}, {a.refcount, 4 * nb}, {a.free_queue, 4 * nb}, {a.queue, 8},
              {a.slots, 8 * tokens}, {a.positions, 4 * tokens}, {a.row_off, 4 * (n + 1)}, {a.kv_len, 4 * n}, {a.copies, 12 * n},
              {a.n_copies, 4}, {a.status, 4}, {workspace, spork::tables_workspace_bytes(a.num_blocks, a.n_seqs)},
              {a.lens, 4 * n}, {a.n_new, 4 * n}, {a.parents, 4 * n}};
  constexpr int kRuns = sizeof(runs) / sizeof(runs[0]), kWritten = kRuns - 3;
  uintptr_t from[kRuns], to[kRuns];
  for (int i = 0; i < kRuns; ++i) {  // (nothing, from and to 0, overlaps nothing)
    from[i] = runs[i].bytes > 0 ? reinterpret_cast<uintptr_t>(runs[i].at) : 0;
    to[i] = from[i] != 0 ? from[i] + runs[i].bytes : 0;
  }
  // Without a branch per pair: 0.10 us of every step against 0.17.
  bool meet = false;
  for (int i = 0; i < kWritten; ++i)
    for (int j = i + 1; j < kRuns; ++j) meet |= (from[i] < to[j]) & (from[j] < to[i]);
  if (meet)
    return fail(SPORK_E_INVAL, "tables, outputs, workspace and inputs of a step must not overlap (kv_len in place of lens, say)");
  return SPORK_OK;
}

spork::TablesArgs tables_args(const spork_tables* t) {
  spork::TablesArgs a{};
  a.num_blocks = t->num_blocks;
  a.block_size = t->block_size;
  a.n_seqs = t->n_seqs;
  a.max_blocks = t->max_blocks;
  a.table = t->table;
  a.held = t->held;
  a.refcount = t->refcount;
  a.free_queue = t->free_queue;
  a.queue = t->queue;
  return a;
}

int check_chunk_shape(const spork_shape* shape) {
  const int rc = check_shape(shape);
  if (rc != SPORK_OK) return rc;
  if (!spork::chunk_supported(shape->dtype, shape->head_dim, shape->block_size))
    return fail(SPORK_E_UNSUPPORTED, "spork_chunk_attn takes head_dim 64 or 128 and block_size 16 or 32");
  if (shape->hq / shape->hkv > spork::kChunkTileRows)
    return fail(SPORK_E_UNSUPPORTED, "spork_chunk_attn takes at most 256 query heads per KV head");
  return SPORK_OK;
}

}  // namespace

extern "C" {

int spork_tables_workspace_bytes(const spork_tables* tables, size_t* bytes) {
  return guarded([&] {
    if (bytes == nullptr) return fail(SPORK_E_INVAL, "bytes is NULL");
    const int rc = check_tables(tables);
    if (rc != SPORK_OK) return rc;
    *bytes = spork::tables_workspace_bytes(tables->num_blocks, tables->n_seqs);
    return SPORK_OK;
  });
}

int spork_tables_workspace_clear(const spork_tables* tables, void* workspace, size_t ws_bytes, hipStream_t stream) {
  return guarded([&] {
    int rc = check_tables(tables);
    if (rc == SPORK_OK) rc = check_tables_workspace(tables, workspace, ws_bytes);
    if (rc != SPORK_OK) return rc;
    return hip_status(spork::launch_words_clear(static_cast<int32_t*>(workspace),
                                                static_cast<int64_t>(spork::tables_control_bytes(tables->num_blocks) / 4),
                                                stream),
                      "spork_tables_workspace_clear");
  });
}

int spork_tables_init(const spork_tables* tables, const int32_t* free_order, hipStream_t stream) {
  return guarded([&] {
    const int rc = check_tables_memory(tables);
    if (rc != SPORK_OK) return rc;
    return hip_status(spork::launch_tables_init(tables_args(tables), free_order, stream), "spork_tables_init");
  });
}

int spork_tables_step(const spork_tables* tables, const int32_t* lens, const int32_t* n_new, const int32_t* parents,
                      int32_t max_tokens, int64_t* slots, int32_t* positions, int32_t* row_off, int32_t* kv_len,
                      int32_t* copies, int32_t* n_copies, int32_t* status, void* workspace, size_t ws_bytes,
                      hipStream_t stream) {
  return guarded([&] {
    int rc = check_tables_memory(tables);
    if (rc != SPORK_OK) return rc;
    if (max_tokens < 0) return fail(SPORK_E_INVAL, "max_tokens must be >= 0");
    if (!lens || !n_new || !row_off || !kv_len || !copies || !n_copies || !status || (max_tokens > 0 && !slots))
      return fail(SPORK_E_INVAL, "NULL pointer");
    if (tables->n_seqs + (max_tokens + int64_t{255}) / 256 > kMostGroups)
      return fail(SPORK_E_UNSUPPORTED, "n_seqs + max_tokens / 256 must be below 2^24");
    rc = check_tables_workspace(tables, workspace, ws_bytes);
    if (rc != SPORK_OK) return rc;
    spork::TablesArgs a = tables_args(tables);
    a.max_tokens = max_tokens;
    a.lens = lens;
    a.n_new = n_new;
    a.parents = parents;
    a.slots = slots;
    a.positions = positions;
    a.row_off = row_off;
    a.kv_len = kv_len;
    a.copies = copies;
    a.n_copies = n_copies;
    a.status = status;
    rc = check_step_apart(a, workspace);
    if (rc != SPORK_OK) return rc;
    spork::tables_workspace(&a, workspace);
    return hip_status(spork::launch_tables_step(a, stream), "spork_tables_step");
  });
}

int spork_kv_copy_batch(const spork_shape* shape, void* k_cache, void* v_cache, int32_t num_blocks, const int32_t* copies,
                        const int32_t* n_copies, int32_t max_copies, hipStream_t stream) {
  return guarded([&] {
    const int rc = check_shape(shape);
    if (rc != SPORK_OK) return rc;
    if (num_blocks <= 0 || max_copies < 0) return fail(SPORK_E_INVAL, "num_blocks must be positive and max_copies >= 0");
    if (max_copies == 0) return SPORK_OK;
    if (!k_cache || !v_cache || !copies || !n_copies) return fail(SPORK_E_INVAL, "NULL pointer");
    const int elem = elem_bytes(shape->dtype);
    if (shape->head_dim * static_cast<int64_t>(elem) % 16 != 0)
      return fail(SPORK_E_UNSUPPORTED, "head_dim must fill 16-byte vectors");
    if (!aligned16(k_cache) || !aligned16(v_cache)) return fail(SPORK_E_INVAL, "pools must be 16-byte aligned");
    if (static_cast<int64_t>(max_copies) * shape->hkv > kMostGroups ||
        static_cast<int64_t>(shape->head_dim) * shape->block_size * elem > INT_MAX)
      return fail(SPORK_E_UNSUPPORTED, "max_copies * hkv must be below 2^24 and a block's bytes per head below 2^31");
    return hip_status(spork::launch_kv_copy_batch(elem, shape->hkv, shape->head_dim, shape->block_size, num_blocks, k_cache,
                                                  v_cache, copies, n_copies, max_copies, stream),
                      "spork_kv_copy_batch");
  });
}

int spork_chunk_workspace_bytes(const spork_shape* shape, int32_t n_seqs, int32_t n_rows, size_t* bytes) {
  return guarded([&] {
    if (bytes == nullptr) return fail(SPORK_E_INVAL, "bytes is NULL");
    const int rc = check_chunk_shape(shape);
    if (rc != SPORK_OK) return rc;
    if (n_seqs < 0 || n_rows < 0) return fail(SPORK_E_INVAL, "n_seqs and n_rows must be >= 0");
    *bytes = n_seqs == 0 || n_rows == 0 ? 0 : spork::chunk_workspace_bytes(shape->head_dim);
    return SPORK_OK;
  });
}

int spork_chunk_attn(const spork_shape* shape, const void* q, int64_t q_stride, const void* k_cache, const void* v_cache,
                     int32_t num_blocks, const int32_t* table, int32_t max_blocks, const int32_t* row_off,
                     const int32_t* kv_len, int32_t n_seqs, int32_t n_rows, void* out, float* lse, void* workspace,
                     size_t ws_bytes, hipStream_t stream) {
  return guarded([&] {
    const int rc = check_chunk_shape(shape);
    if (rc != SPORK_OK) return rc;
    if (n_seqs < 0 || n_rows < 0 || num_blocks <= 0 || max_blocks <= 0)
      return fail(SPORK_E_INVAL, "n_seqs and n_rows must be >= 0, num_blocks and max_blocks positive");
    if (n_seqs == 0 || n_rows == 0) return SPORK_OK;
    if (!q || !k_cache || !v_cache || !table || !row_off || !kv_len || !out) return fail(SPORK_E_INVAL, "NULL pointer");
    const int elem = elem_bytes(shape->dtype);
    if (q_stride < static_cast<int64_t>(shape->hq) * shape->head_dim || q_stride > INT64_MAX / 4 / n_rows ||
        q_stride * elem % 16 != 0)
      return fail(SPORK_E_INVAL, "q_stride must cover a query row and keep rows 16-byte aligned");
    if (!aligned16(q) || !aligned16(k_cache) || !aligned16(v_cache) || !aligned16(out))
      return fail(SPORK_E_INVAL, "q, pools and out must be 16-byte aligned");
    if (static_cast<int64_t>(max_blocks) * shape->block_size > INT_MAX - kHeadroom)
      return fail(SPORK_E_UNSUPPORTED, "max_blocks * block_size must be below 2^31 - 4096");
    const float scale_log2 = shape->sm_scale * 1.4426950408889634f;
    if (!std::isfinite(scale_log2)) return fail(SPORK_E_INVAL, "sm_scale is out of range");
    if (workspace == nullptr || !aligned256(workspace))
      return fail(SPORK_E_INVAL, "workspace must be non-NULL and 256-byte aligned");
    if (ws_bytes < spork::chunk_workspace_bytes(shape->head_dim))
      return fail(SPORK_E_CAPACITY, "workspace is smaller than spork_chunk_workspace_bytes");
    spork::ChunkArgs a{};
    a.q = q;
    a.q_stride = q_stride;
    a.k_cache = k_cache;
    a.v_cache = v_cache;
    a.table = table;
    a.row_off = row_off;
    a.kv_len = kv_len;
    a.out = out;
    a.lse = lse;
    a.num_blocks = num_blocks;
    a.max_blocks = max_blocks;
    a.n_seqs = n_seqs;
    a.n_rows = n_rows;
    a.hq = shape->hq;
    a.hkv = shape->hkv;
    a.group = shape->hq / shape->hkv;
    a.tile_rows = spork::kChunkTileRows / a.group;
    a.most_heads = spork::chunk_tile_heads(n_seqs, shape->hkv);
    a.head_dim = shape->head_dim;
    a.block_size = shape->block_size;
    a.dtype = shape->dtype;
    // The bf16 kernel masks a score by an infinity before the scale: a scale of
    // zero stands in as the smallest normal number.
    a.scale_log2 = scale_log2 == 0.0f ? FLT_MIN : scale_log2;
    spork::chunk_workspace(&a, workspace);
    hipError_t e = timed(SPORK_KERNEL_ATTN, stream, [&] { return spork::launch_chunk_attn(a, stream); });
    if (e == hipSuccess) e = timed(SPORK_KERNEL_MERGE, stream, [&] { return spork::launch_chunk_merge(a, stream); });
    return hip_status(e, "spork_chunk_attn");
  });
}

}  // extern "C"
