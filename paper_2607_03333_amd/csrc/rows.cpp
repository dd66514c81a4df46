// C ABI of libspork (declared in include/spork.h): from a projection's rows to
// the cache. Argument checks and dispatch of the norms and rotations, and of the
// cache of 8-bit codes.
#include <algorithm>
#include <cfloat>
#include <climits>
#include <cmath>
#include <cstdint>

#include "capi_common.h"
#include "chunk_kernels.h"
#include "rows_kernels.h"
#include "spork.h"

namespace {

using namespace spork::capi;

// A launch has fewer than 2^32 threads: so many workgroups of 256.
constexpr int64_t kMostGroups = (int64_t{1} << 24) - 1;
// Rows of heads that a write takes, so that its workgroups (kvq.hip) are fewer than these:
// for keys and values some 1,500, or from windows of 16 rows on (n_rows / 16 + 2) (hkv + 3) / 2
// at most, and n_rows (hq + 15) / 64 + 1 for queries.
constexpr int64_t kMostHeadRows = int64_t{1} << 25;
// Of norms: far past any use, and where factors in 32 bits are exact enough (norm_head, turn.h).
constexpr double kMostEps = 0x1p100;
// Positions run a few stages past a context's end, in 32 bits.
constexpr int64_t kHeadroom = 4096;

// Rows of [heads][D] elements, `stride` elements apart.
struct Rows {
  const void* at;
  int64_t stride, width;  // in elements
};

int check_rows(const Rows& r, int32_t n_rows, int elem, const char* what) {
  if (r.at == nullptr) return fail(SPORK_E_INVAL, std::string(what) + " is NULL");
  if (r.stride < r.width || r.stride > INT64_MAX / 4 / n_rows || r.stride * elem % 16 != 0)
    return fail(SPORK_E_INVAL, std::string(what) + ": the stride must cover a row and keep rows 16-byte aligned");
  if (!aligned16(r.at)) return fail(SPORK_E_INVAL, std::string(what) + " must be 16-byte aligned");
  return SPORK_OK;
}

// Whether any two of the n_rows rows meet. Rows of one stride may lie side by side.
bool rows_meet(const Rows& x, const Rows& y, int32_t n_rows, int elem) {
  if (x.at == nullptr || y.at == nullptr) return false;
  const auto bytes = [&](int64_t e) { return static_cast<uintptr_t>(e) * static_cast<uintptr_t>(elem); };
  const auto from = [](const Rows& r) { return reinterpret_cast<uintptr_t>(r.at); };
  const auto to = [&](const Rows& r) { return from(r) + bytes(r.stride * (n_rows - 1) + r.width); };
  if (from(x) >= to(y) || from(y) >= to(x)) return false;
  if (x.stride != y.stride) return true;
  const uintptr_t s = bytes(x.stride);
  const Rows &low = from(x) <= from(y) ? x : y, &high = from(x) <= from(y) ? y : x;
  const uintptr_t apart = (from(high) - from(low)) % s;
  return apart < bytes(low.width) || s - apart < bytes(high.width);
}

// An output in place of its input, or apart from it.
bool in_place(const Rows& in, const Rows& out) { return in.at == out.at && in.stride == out.stride; }

int check_turn(const spork_shape* shape, const spork_rope* rope, const spork_qk_norm* norm, bool with_q, bool with_k) {
  if (rope != nullptr) {
    if (rope->rotary_dim < 16 || rope->rotary_dim > shape->head_dim || rope->rotary_dim % 16 != 0)
      return fail(SPORK_E_UNSUPPORTED, "rotary_dim must be a multiple of 16 from 16 to head_dim");
    if (rope->layout != SPORK_ROPE_HALF && rope->layout != SPORK_ROPE_INTERLEAVED)
      return fail(SPORK_E_INVAL, "layout must be SPORK_ROPE_HALF or SPORK_ROPE_INTERLEAVED");
    const double m = std::abs(rope->magnitude);  // (cosines and sines times it are kept in 32 bits)
    if (m != 0 && !(m >= FLT_MIN && m <= FLT_MAX)) return fail(SPORK_E_INVAL, "magnitude must be 0 or in float32's normal range");
    if (rope->inv_freq == nullptr || !aligned16(rope->inv_freq))
      return fail(SPORK_E_INVAL, "inv_freq must be non-NULL and 16-byte aligned");
  }
  if (norm != nullptr) {
    if ((with_q && norm->q_weight == nullptr) || (with_k && norm->k_weight == nullptr))
      return fail(SPORK_E_INVAL, "a norm's weight is NULL");
    if ((with_q && !aligned16(norm->q_weight)) || (with_k && !aligned16(norm->k_weight)))
      return fail(SPORK_E_INVAL, "the norms' weights must be 16-byte aligned");
    if (!(norm->eps >= 0 && norm->eps <= kMostEps)) return fail(SPORK_E_INVAL, "eps must be from 0 to 2^100");
  }
  return SPORK_OK;
}

spork::TurnArgs turn_args(const spork_rope* rope, const spork_qk_norm* norm) {
  spork::TurnArgs t{};
  if (rope != nullptr) {
    t.inv_freq = rope->inv_freq;
    t.rotary_dim = rope->rotary_dim;
    t.interleaved = rope->layout == SPORK_ROPE_INTERLEAVED;
    t.magnitude = rope->magnitude;
  }
  if (norm != nullptr) {
    t.q_weight = norm->q_weight;
    t.k_weight = norm->k_weight;
    t.eps = norm->eps;
  }
  return t;
}

int check_row_heads(const spork_shape* shape) {
  const int rc = check_shape(shape);
  if (rc != SPORK_OK) return rc;
  if (!spork::rows_supported(shape->dtype, shape->head_dim)) return fail(SPORK_E_UNSUPPORTED, "head_dim must be 64 or 128");
  if (shape->hq > INT_MAX / 2 / shape->head_dim)
    return fail(SPORK_E_UNSUPPORTED, "hq * head_dim must be below 2^30");
  return SPORK_OK;
}

int check_kvq_shape(const spork_shape* shape) {
  const int rc = check_row_heads(shape);
  if (rc != SPORK_OK) return rc;
  if (!spork::kvq_supported(shape->dtype, shape->head_dim, shape->block_size))
    return fail(SPORK_E_UNSUPPORTED, "the cache of 8-bit codes takes head_dim 64 or 128 and block_size 16 or 32");
  if (static_cast<int64_t>(shape->hkv) * shape->head_dim * shape->block_size > INT_MAX)
    return fail(SPORK_E_UNSUPPORTED, "hkv * head_dim * block_size must be below 2^31");
  return SPORK_OK;
}

int check_cache(const spork_kvq* c) {
  if (c == nullptr) return fail(SPORK_E_INVAL, "cache is NULL");
  if (c->num_blocks <= 0) return fail(SPORK_E_INVAL, "num_blocks must be positive");
  if (!c->k_codes || !c->v_codes || !c->k_scale || !c->v_scale) return fail(SPORK_E_INVAL, "a pointer of cache is NULL");
  if (!aligned16(c->k_codes) || !aligned16(c->v_codes)) return fail(SPORK_E_INVAL, "codes must be 16-byte aligned");
  return SPORK_OK;
}

spork::KvqPools pools_of(const spork_kvq* c) {
  return spork::KvqPools{c->k_codes, c->v_codes, c->k_scale, c->v_scale, c->num_blocks};
}

}  // namespace

extern "C" {

int spork_rope_frequencies(int32_t rotary_dim, double base, const spork_rope_scaling* scaling, double* inv_freq,
                           double* magnitude) {
  return guarded([&] {
    if (inv_freq == nullptr || magnitude == nullptr) return fail(SPORK_E_INVAL, "NULL pointer");
    if (rotary_dim <= 0 || rotary_dim % 2 != 0) return fail(SPORK_E_INVAL, "rotary_dim must be positive and even");
    if (!std::isfinite(base) || base <= 1) return fail(SPORK_E_INVAL, "base must be finite and above 1");
    const int kind = scaling != nullptr ? scaling->kind : 0;
    double factor = 1;
    if (scaling != nullptr) {
      factor = scaling->factor;
      if (kind < SPORK_ROPE_SCALE_LINEAR || kind > SPORK_ROPE_SCALE_BANDS) return fail(SPORK_E_INVAL, "unknown kind of scaling");
      if (!std::isfinite(factor) || factor <= 0) return fail(SPORK_E_INVAL, "factor must be finite and positive");
      if (kind == SPORK_ROPE_SCALE_BASE && rotary_dim <= 2) return fail(SPORK_E_INVAL, "this scaling needs a rotary_dim above 2");
      if (kind >= SPORK_ROPE_SCALE_PARTS &&
          (scaling->trained_len <= 0 || !std::isfinite(scaling->fast) || !(scaling->slow > 0) || !(scaling->fast > scaling->slow)))
        return fail(SPORK_E_INVAL, "this scaling needs trained_len > 0 and fast > slow > 0");
    }
    const double two_pi = 6.283185307179586477, r = rotary_dim;
    const double b = kind == SPORK_ROPE_SCALE_BASE ? base * std::pow(factor, r / (r - 2)) : base;
    // PARTS: between these pairs
    double low = 0, high = 0;
    if (kind == SPORK_ROPE_SCALE_PARTS) {
      const auto pair = [&](double turns) { return r * std::log(scaling->trained_len / (turns * two_pi)) / (2 * std::log(base)); };
      low = std::max(std::floor(pair(scaling->fast)), 0.0);
      high = std::min(std::ceil(pair(scaling->slow)), r - 1);
    }
    const auto frequency = [&](int32_t i) {
      double f = std::pow(b, -2 * static_cast<double>(i) / r);
      double stretched = 0;  // how much of it is
      if (kind == SPORK_ROPE_SCALE_LINEAR) stretched = 1;
      if (kind == SPORK_ROPE_SCALE_PARTS) stretched = std::min(std::max((i - low) / std::max(high - low, 1e-3), 0.0), 1.0);
      if (kind == SPORK_ROPE_SCALE_BANDS) {
        const double turns = scaling->trained_len * f / two_pi;
        stretched = 1 - std::min(std::max((turns - scaling->slow) / (scaling->fast - scaling->slow), 0.0), 1.0);
      }
      if (stretched > 0) f = f * (1 - stretched) + f / factor * stretched;
      return f;
    };
    for (int32_t i = 0; i < rotary_dim / 2; ++i)
      if (!std::isfinite(frequency(i))) return fail(SPORK_E_INVAL, "factor is so small that frequencies are not finite");
    for (int32_t i = 0; i < rotary_dim / 2; ++i) inv_freq[i] = frequency(i);
    *magnitude = kind == SPORK_ROPE_SCALE_PARTS && factor > 1 ? 0.1 * std::log(factor) + 1 : 1.0;
    return SPORK_OK;
  });
}

int spork_qk_rope(const spork_shape* shape, const spork_rope* rope, const spork_qk_norm* norm, const int32_t* positions,
                  int32_t n_rows, const void* q, int64_t q_stride, const void* k, int64_t k_stride, void* q_out,
                  int64_t q_out_stride, void* k_out, int64_t k_out_stride, hipStream_t stream) {
  return guarded([&] {
    int rc = check_row_heads(shape);
    if (rc != SPORK_OK) return rc;
    if (n_rows < 0) return fail(SPORK_E_INVAL, "n_rows must be >= 0");
    if (rope == nullptr && norm == nullptr) return fail(SPORK_E_INVAL, "rope and norm are both NULL");
    if (n_rows == 0) return SPORK_OK;
    const bool with_q = q != nullptr || q_out != nullptr, with_k = k != nullptr || k_out != nullptr;
    if (!with_q && !with_k) return fail(SPORK_E_INVAL, "q and k are both NULL");
    rc = check_turn(shape, rope, norm, with_q, with_k);
    if (rc != SPORK_OK) return rc;
    if (rope != nullptr && positions == nullptr) return fail(SPORK_E_INVAL, "positions is NULL");
    const int elem = elem_bytes(shape->dtype);
    const int64_t qw = static_cast<int64_t>(shape->hq) * shape->head_dim, kw = static_cast<int64_t>(shape->hkv) * shape->head_dim;
    const Rows in[2] = {{q, q_stride, qw}, {k, k_stride, kw}}, out[2] = {{q_out, q_out_stride, qw}, {k_out, k_out_stride, kw}};
    const bool with[2] = {with_q, with_k};
    const char* names[4] = {"q", "k", "q_out", "k_out"};
    for (int i = 0; i < 2 && rc == SPORK_OK; ++i) {
      if (!with[i]) continue;
      rc = check_rows(in[i], n_rows, elem, names[i]);
      if (rc == SPORK_OK) rc = check_rows(out[i], n_rows, elem, names[2 + i]);
    }
    if (rc != SPORK_OK) return rc;
    bool meet = rows_meet(out[0], out[1], n_rows, elem);
    for (int o = 0; o < 2; ++o)
      for (int i = 0; i < 2; ++i) meet |= !(o == i && in_place(in[i], out[o])) && rows_meet(out[o], in[i], n_rows, elem);
    if (meet) return fail(SPORK_E_INVAL, "outputs must not overlap, nor the inputs unless in place of their own");
    if ((static_cast<int64_t>(shape->hq) + shape->hkv + 7) / 8 * n_rows / 4 >= kMostGroups)
      return fail(SPORK_E_UNSUPPORTED, "n_rows * ((hq + hkv + 7) / 8) must be below 2^26 - 4");
    spork::RopeArgs a{};
    a.turn = turn_args(rope, norm);
    a.positions = rope != nullptr ? positions : nullptr;
    a.q = q;
    a.k = k;
    a.q_out = q_out;
    a.k_out = k_out;
    a.q_stride = q_stride;
    a.k_stride = k_stride;
    a.q_out_stride = q_out_stride;
    a.k_out_stride = k_out_stride;
    a.n_rows = n_rows;
    a.hq = with_q ? shape->hq : 0;
    a.hkv = with_k ? shape->hkv : 0;
    a.head_dim = shape->head_dim;
    a.dtype = shape->dtype;
    return hip_status(spork::launch_qk_rope(a, stream), "spork_qk_rope");
  });
}

int spork_kvq_write(const spork_shape* shape, const spork_kvq* cache, const spork_rope* rope, const spork_qk_norm* norm,
                    const int64_t* slots, const int32_t* positions, int32_t n_rows, const void* q, int64_t q_stride,
                    const void* k, int64_t k_stride, const void* v, int64_t v_stride, void* q_out, int64_t q_out_stride,
                    int32_t* bad_slots, hipStream_t stream) {
  return guarded([&] {
    int rc = check_kvq_shape(shape);
    if (rc == SPORK_OK) rc = check_cache(cache);
    if (rc != SPORK_OK) return rc;
    if (n_rows < 0) return fail(SPORK_E_INVAL, "n_rows must be >= 0");
    if (n_rows == 0) return SPORK_OK;
    const bool with_q = q != nullptr || q_out != nullptr;
    if (with_q && rope == nullptr && norm == nullptr) return fail(SPORK_E_INVAL, "q needs rope or norm: without them it is ready");
    rc = check_turn(shape, rope, norm, with_q, true);
    if (rc != SPORK_OK) return rc;
    if (slots == nullptr || (rope != nullptr && positions == nullptr)) return fail(SPORK_E_INVAL, "slots or positions is NULL");
    const int elem = elem_bytes(shape->dtype);
    const int64_t qw = static_cast<int64_t>(shape->hq) * shape->head_dim, kw = static_cast<int64_t>(shape->hkv) * shape->head_dim;
    const Rows qr{q, q_stride, qw}, kr{k, k_stride, kw}, vr{v, v_stride, kw}, qo{q_out, q_out_stride, qw};
    rc = check_rows(kr, n_rows, elem, "k");
    if (rc == SPORK_OK) rc = check_rows(vr, n_rows, elem, "v");
    if (rc == SPORK_OK && with_q) rc = check_rows(qr, n_rows, elem, "q");
    if (rc == SPORK_OK && with_q) rc = check_rows(qo, n_rows, elem, "q_out");
    if (rc != SPORK_OK) return rc;
    if ((!in_place(qr, qo) && rows_meet(qo, qr, n_rows, elem)) || rows_meet(qo, kr, n_rows, elem) || rows_meet(qo, vr, n_rows, elem))
      return fail(SPORK_E_INVAL, "q_out must not overlap what is read, unless in place of q");
    if (static_cast<int64_t>(n_rows) * (static_cast<int64_t>(shape->hq) + shape->hkv) >= kMostHeadRows)
      return fail(SPORK_E_UNSUPPORTED, "n_rows * (hq + hkv) must be below 2^25");
    spork::KvqWriteArgs a{};
    a.turn = turn_args(rope, norm);
    a.pools = pools_of(cache);
    a.slots = slots;
    a.positions = positions;
    a.q = q;
    a.k = k;
    a.v = v;
    a.q_out = q_out;
    a.q_stride = q_stride;
    a.k_stride = k_stride;
    a.v_stride = v_stride;
    a.q_out_stride = q_out_stride;
    a.bad_slots = bad_slots;
    a.n_rows = n_rows;
    a.hq = shape->hq;
    a.hkv = shape->hkv;
    a.head_dim = shape->head_dim;
    a.block_size = shape->block_size;
    a.dtype = shape->dtype;
    return hip_status(spork::launch_kvq_write(a, stream), "spork_kvq_write");
  });
}

int spork_kvq_copy_batch(const spork_shape* shape, const spork_kvq* cache, const int32_t* copies, const int32_t* n_copies,
                         int32_t max_copies, hipStream_t stream) {
  return guarded([&] {
    int rc = check_kvq_shape(shape);
    if (rc == SPORK_OK) rc = check_cache(cache);
    if (rc != SPORK_OK) return rc;
    if (max_copies < 0) return fail(SPORK_E_INVAL, "max_copies must be >= 0");
    if (max_copies == 0) return SPORK_OK;
    if (!copies || !n_copies) return fail(SPORK_E_INVAL, "NULL pointer");
    if (static_cast<int64_t>(max_copies) * shape->hkv > kMostGroups)
      return fail(SPORK_E_UNSUPPORTED, "max_copies * hkv must be below 2^24");
    return hip_status(spork::launch_kvq_copy_batch(pools_of(cache), shape->hkv, shape->head_dim, shape->block_size, copies,
                                                   n_copies, max_copies, stream),
                      "spork_kvq_copy_batch");
  });
}

int spork_kvq_attn(const spork_shape* shape, const void* q, int64_t q_stride, const spork_kvq* cache, const int32_t* table,
                   int32_t max_blocks, const int32_t* row_off, const int32_t* kv_len, int32_t n_seqs, int32_t n_rows,
                   void* out, float* lse, void* workspace, size_t ws_bytes, hipStream_t stream) {
  return guarded([&] {
    int rc = check_kvq_shape(shape);
    if (rc != SPORK_OK) return rc;
    if (shape->hq / shape->hkv > spork::kChunkTileRows)
      return fail(SPORK_E_UNSUPPORTED, "spork_kvq_attn takes at most 256 query heads per KV head");
    rc = check_cache(cache);
    if (rc != SPORK_OK) return rc;
    if (n_seqs < 0 || n_rows < 0 || max_blocks <= 0)
      return fail(SPORK_E_INVAL, "n_seqs and n_rows must be >= 0, max_blocks positive");
    if (n_seqs == 0 || n_rows == 0) return SPORK_OK;
    if (!table || !row_off || !kv_len || !out) return fail(SPORK_E_INVAL, "NULL pointer");
    const int64_t width = static_cast<int64_t>(shape->hq) * shape->head_dim;
    rc = check_rows(Rows{q, q_stride, width}, n_rows, elem_bytes(shape->dtype), "q");
    if (rc != SPORK_OK) return rc;
    if (!aligned16(out)) return fail(SPORK_E_INVAL, "out must be 16-byte aligned");
    if (static_cast<int64_t>(max_blocks) * shape->block_size > INT_MAX - kHeadroom)
      return fail(SPORK_E_UNSUPPORTED, "max_blocks * block_size must be below 2^31 - 4096");
    const float scale_log2 = shape->sm_scale * 1.4426950408889634f;
    if (!std::isfinite(scale_log2)) return fail(SPORK_E_INVAL, "sm_scale is out of range");
    if (workspace == nullptr || (reinterpret_cast<uintptr_t>(workspace) & 255) != 0)
      return fail(SPORK_E_INVAL, "workspace must be non-NULL and 256-byte aligned");
    if (ws_bytes < spork::chunk_workspace_bytes(shape->head_dim))
      return fail(SPORK_E_CAPACITY, "workspace is smaller than spork_chunk_workspace_bytes");
    if (rows_meet(Rows{q, q_stride, width}, Rows{out, width, width}, n_rows, elem_bytes(shape->dtype)))
      return fail(SPORK_E_INVAL, "out must not overlap q");
    spork::ChunkArgs a{};
    a.q = q;
    a.q_stride = q_stride;
    a.k_cache = cache->k_codes;
    a.v_cache = cache->v_codes;
    a.k_scale = cache->k_scale;
    a.v_scale = cache->v_scale;
    a.table = table;
    a.row_off = row_off;
    a.kv_len = kv_len;
    a.out = out;
    a.lse = lse;
    a.num_blocks = cache->num_blocks;
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
    // A score is masked by an infinity before the scale: a scale of zero stands in
    // as the smallest normal number.
    a.scale_log2 = scale_log2 == 0.0f ? FLT_MIN : scale_log2;
    spork::chunk_workspace(&a, workspace);
    hipError_t e = timed(SPORK_KERNEL_ATTN, stream, [&] { return spork::launch_kvq_attn(a, stream); });
    if (e == hipSuccess) e = timed(SPORK_KERNEL_MERGE, stream, [&] { return spork::launch_chunk_merge(a, stream); });
    return hip_status(e, "spork_kvq_attn");
  });
}

}  // extern "C"
