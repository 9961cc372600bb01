// Validation and translation of arguments that the entry points of the cached
// decoding share (abi_cache.cpp, abi_cache_norm.cpp).
#pragma once

#include "abi_common.h"
#include "cache.h"

namespace mosaic {

constexpr int64_t kMaxSlots = (int64_t)1 << 30;     // of one sequence: slots fit int32 with room

// Bytes of an element (of a cache in 4 bits, the unit of its strides).
inline int64_t size_of(int32_t ftype) { return ftype == MOSAIC_F32 ? 4 : ftype == MOSAIC_E2M1 ? 1 : 2; }

inline bool overlap(const void* a, int64_t an, const void* b, int64_t bn) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + (uintptr_t)bn && y < x + (uintptr_t)an;
}

// Bytes from the first to the last element of rows x cols.
inline int64_t extent(int64_t rows, int64_t ld, int64_t cols, int64_t size) { return ((rows - 1) * ld + cols) * size; }

// Whether `rows` rows of an bytes and as many of bn bytes overlap; rows as far apart
// in both may lie side by side.
inline bool rows_overlap(const void* a, int64_t lda, int64_t an, const void* b, int64_t ldb, int64_t bn, int64_t rows) {
  if (!overlap(a, (rows - 1) * lda + an, b, (rows - 1) * ldb + bn)) return false;
  if (lda != ldb) return true;
  const int64_t apart = (int64_t)(reinterpret_cast<uintptr_t>(b) - reinterpret_cast<uintptr_t>(a));
  const int64_t at = (apart % lda + lda) % lda;      // where the one's rows begin, from the other's
  return at < an || at + bn > lda;
}

inline mosaic_status view_of(const mosaic_kv_cache* c, CacheView* v) {
  if (c == nullptr) return fail(MOSAIC_ERR_INVALID_ARG, "cache is NULL");
  if ((c->dtype < MOSAIC_F32 || c->dtype > MOSAIC_F16) && c->dtype != MOSAIC_E2M1)
    return fail(MOSAIC_ERR_INVALID_ARG, "unknown cache dtype %d", c->dtype);
  if (c->batch < 0 || c->pages < 0 || c->max_blocks < 0 || c->kv_heads < 1)
    return fail(MOSAIC_ERR_INVALID_ARG, "negative size, or no key/value heads");
  if (c->head_dim < 8 || c->head_dim > 256 || c->head_dim % 8 != 0)
    return fail(MOSAIC_ERR_UNSUPPORTED, "head_dim %d is not a multiple of 8 in [8, 256]", c->head_dim);
  if (c->page_size < 16 || c->page_size > 4096 || (c->page_size & (c->page_size - 1)) != 0)
    return fail(MOSAIC_ERR_UNSUPPORTED, "page_size %d is not a power of two in [16, 4096]", c->page_size);
  if (c->kv_heads > 1024) return fail(MOSAIC_ERR_UNSUPPORTED, "more than 1024 key/value heads");
  if (c->batch > 65535 || c->pages > 0x7FFFFFFF || c->max_blocks > kMaxSlots / c->page_size)
    return fail(MOSAIC_ERR_UNSUPPORTED, "more than 65535 sequences, 2^31 - 1 pages or 2^30 slots of a sequence");
  const int64_t es = size_of(c->dtype), row = c->dtype == MOSAIC_E2M1 ? MOSAIC_E2M1_ROW_BYTES(c->head_dim) : c->head_dim;
  // the stride of a dimension of one has no meaning
  const int64_t page_stride = c->pages > 1 ? c->page_stride : 0, head_stride = c->kv_heads > 1 ? c->head_stride : 0;
  if (page_stride < 0 || head_stride < 0 || c->token_stride < 0) return fail(MOSAIC_ERR_INVALID_ARG, "negative stride");
  if (head_stride > INT32_MAX / 4096 || c->token_stride > (1 << 27) / c->page_size ||   // a page within 2^30 bytes
      page_stride > INT64_MAX / 8 / (c->pages > 0 ? c->pages : 1))
    return fail(MOSAIC_ERR_UNSUPPORTED, "stride too large");
  if (page_stride * es % 16 != 0 || head_stride * es % 16 != 0 || c->token_stride * es % 16 != 0)
    return fail(MOSAIC_ERR_INVALID_ARG, "strides must be multiples of 16 bytes");
  // rows of a page lie apart: by places within heads, or by heads within places
  const int64_t places = (int64_t)(c->page_size - 1) * c->token_stride, heads = (int64_t)(c->kv_heads - 1) * head_stride;
  const bool by_head = c->token_stride >= row && (c->kv_heads == 1 || head_stride >= places + row);
  const bool by_place = (c->kv_heads == 1 || head_stride >= row) && c->token_stride >= heads + row;
  if (!by_head && !by_place) return fail(MOSAIC_ERR_INVALID_ARG, "rows of a page overlap");
  if (c->pages > 1 && page_stride < places + heads + row)
    return fail(MOSAIC_ERR_INVALID_ARG, "pages overlap");
  if (c->batch > 0 && c->max_blocks > 0) {
    if (c->block_table == nullptr) return fail(MOSAIC_ERR_INVALID_ARG, "block_table is NULL");
    if (c->ldt != 0 && c->ldt < c->max_blocks) return fail(MOSAIC_ERR_INVALID_ARG, "ldt < max_blocks");
  }
  if (c->pages > 0 && (c->k == nullptr || c->v == nullptr)) return fail(MOSAIC_ERR_INVALID_ARG, "k or v is NULL");
  if (!aligned16(c->k) || !aligned16(c->v)) return fail(MOSAIC_ERR_INVALID_ARG, "k and v must be 16-byte aligned");
  v->k = (char*)c->k;
  v->v = (char*)c->v;
  v->weights = c->weights;
  v->order = c->order;
  v->table = c->block_table;
  v->ldt = c->ldt;
  v->page_stride = page_stride * es;
  v->head_stride = head_stride * es;
  v->token_stride = c->token_stride * es;
  v->pages = (int32_t)c->pages;
  v->batch = c->batch;
  v->max_blocks = c->max_blocks;
  v->kv_heads = c->kv_heads;
  v->head_dim = c->head_dim;
  v->log2_page = __builtin_ctz((unsigned)c->page_size);
  v->dtype = c->dtype;
  return MOSAIC_OK;
}

// Calls that write to pages: not to those of a table that all sequences share.
inline mosaic_status check_own_pages(const CacheView& v) {
  if (v.batch > 1 && v.max_blocks > 0 && v.ldt == 0)
    return fail(MOSAIC_ERR_INVALID_ARG, "sequences that share their block table cannot be written to");
  return MOSAIC_OK;
}

inline int64_t slots_of(const CacheView& v) { return (int64_t)v.max_blocks << v.log2_page; }

inline mosaic_status check_heads(const CacheView& v, int32_t heads, int32_t x_dtype) {
  if (heads < 1 || heads % v.kv_heads != 0)
    return fail(MOSAIC_ERR_INVALID_ARG, "%d query heads are no multiple of %d key/value heads", heads, v.kv_heads);
  if (heads > 4096) return fail(MOSAIC_ERR_UNSUPPORTED, "more than 4096 query heads");
  if (x_dtype < MOSAIC_F32 || x_dtype > MOSAIC_F16) return fail(MOSAIC_ERR_INVALID_ARG, "unknown dtype %d", x_dtype);
  if (x_dtype != MOSAIC_F32 && x_dtype != v.dtype && v.dtype != MOSAIC_E2M1)
    return fail(MOSAIC_ERR_UNSUPPORTED, "activations must be float32 or of the cache's type");
  return MOSAIC_OK;
}

// A rows x cols matrix that kernels access 16 bytes at a time.
inline mosaic_status check_rows(const void* p, int64_t rows, int64_t ld, int64_t cols, int64_t size, const char* name) {
  if (p == nullptr) return fail(MOSAIC_ERR_INVALID_ARG, "%s is NULL", name);
  if (ld < cols) return fail(MOSAIC_ERR_INVALID_ARG, "leading dimension of %s < %lld", name, (long long)cols);
  if (ld > INT64_MAX / 16 / rows) return fail(MOSAIC_ERR_INVALID_ARG, "leading dimension of %s too large", name);
  if (!aligned16(p) || ld * size % 16 != 0) return fail(MOSAIC_ERR_INVALID_ARG, "rows of %s must be 16-byte aligned", name);
  return MOSAIC_OK;
}

inline mosaic_status check_state(const CacheView& v, const int32_t* state, const int32_t* new_state) {
  if (state == nullptr || new_state == nullptr) return fail(MOSAIC_ERR_INVALID_ARG, "state or new_state is NULL");
  if (state != new_state && overlap(state, 8 * (int64_t)v.batch, new_state, 8 * (int64_t)v.batch))
    return fail(MOSAIC_ERR_INVALID_ARG, "new_state overlaps state");
  return MOSAIC_OK;
}

inline mosaic_status check_workspace(const void* p, int64_t bytes, int64_t needed) {
  if (bytes < needed)
    return fail(MOSAIC_ERR_INVALID_ARG, "workspace of %lld bytes, needs %lld", (long long)bytes, (long long)needed);
  if (needed > 0 && (p == nullptr || !aligned16(p)))
    return fail(MOSAIC_ERR_INVALID_ARG, "workspace is NULL or not 16-byte aligned");
  return MOSAIC_OK;
}

// New tokens (mosaic_cache_append, mosaic_cache_append_norm); norm NULL: none.
inline mosaic_status append_tokens(const mosaic_kv_cache* cache, const void* qkv, int64_t ldx, int32_t x_dtype,
                                   int64_t rows, const int32_t* starts, int32_t heads, const mosaic_qk_norm* norm,
                                   const mosaic_rotary* rotary, void* q_out, int64_t ldq, const int32_t* state,
                                   int32_t* new_state, void* stream) {
  AppendLaunch a{};
  mosaic_status st = view_of(cache, &a.c);
  if (st != MOSAIC_OK || (st = check_own_pages(a.c)) != MOSAIC_OK) return st;
  if ((st = check_heads(a.c, heads, x_dtype)) != MOSAIC_OK) return st;
  if (rows < 0) return fail(MOSAIC_ERR_INVALID_ARG, "negative size");
  if (rows > (1 << 22)) return fail(MOSAIC_ERR_UNSUPPORTED, "more than 2^22 tokens");
  if (starts == nullptr && rows != a.c.batch)
    return fail(MOSAIC_ERR_INVALID_ARG, "%lld rows for %d sequences need starts", (long long)rows, a.c.batch);
  if (a.c.batch == 0 && rows > 0) return fail(MOSAIC_ERR_INVALID_ARG, "tokens of no sequence");
  const int64_t size = size_of(x_dtype), D = a.c.head_dim, width = (heads + 2 * (int64_t)a.c.kv_heads) * D;
  if (rotary != nullptr) {
    if (rotary->naxes < 1 || rotary->naxes > kMaxAxes)
      return fail(MOSAIC_ERR_INVALID_ARG, "%d axes outside [1, %d]", rotary->naxes, kMaxAxes);
    int64_t pairs = 0;
    for (int i = 0; i < kMaxAxes; ++i) {
      if (i < rotary->naxes) {
        if (rotary->sections[i] < 0 || rotary->sections[i] > D)
          return fail(MOSAIC_ERR_INVALID_ARG, "section outside [0, head_dim]");
        pairs += rotary->sections[i];
      }
      a.rot.ends[i] = (int32_t)pairs;
    }
    for (int i = rotary->naxes - 1; i < kMaxAxes; ++i) a.rot.ends[i] = INT32_MAX;   // the last axis has the rest
    if (pairs < 1 || 2 * pairs > D)
      return fail(MOSAIC_ERR_INVALID_ARG, "%lld pairs in heads of %lld", (long long)pairs, (long long)D);
    if (rotary->table == nullptr || rotary->rows < 1) return fail(MOSAIC_ERR_INVALID_ARG, "rotary table is NULL or empty");
    if (rotary->rows > INT32_MAX) return fail(MOSAIC_ERR_UNSUPPORTED, "more than 2^31 - 1 rows of the rotary table");
    if (rotary->positions != nullptr && rotary->ldp != 0 && rotary->ldp < rows)
      return fail(MOSAIC_ERR_INVALID_ARG, "ldp < rows");
    a.rot.table = rotary->table;
    a.rot.rows = rotary->rows;
    a.rot.positions = rotary->positions;
    a.rot.ldp = rotary->ldp;
    a.rot.pairs = (int32_t)pairs;
    a.rot.interleaved = rotary->interleaved != 0;
  }
  if (norm != nullptr) {
    if (norm->q_weight == nullptr || norm->k_weight == nullptr) return fail(MOSAIC_ERR_INVALID_ARG, "norm weights are NULL");
    if (!(norm->eps >= 0.0f) || !std::isfinite(norm->eps)) return fail(MOSAIC_ERR_INVALID_ARG, "eps must be finite and >= 0");
    a.norm = {norm->q_weight, norm->k_weight, (double)norm->eps};
  }
  if (a.c.batch == 0) return MOSAIC_OK;
  if ((st = check_state(a.c, state, new_state)) != MOSAIC_OK) return st;
  if (rows > 0) {
    if ((st = check_rows(qkv, rows, ldx, width, size, "qkv")) != MOSAIC_OK) return st;
    if ((st = check_rows(q_out, rows, ldq, heads * D, size, "q_out")) != MOSAIC_OK) return st;
    if (overlap(qkv, extent(rows, ldx, width, size), q_out, extent(rows, ldq, heads * D, size)))
      return fail(MOSAIC_ERR_INVALID_ARG, "q_out overlaps qkv");
  }
  a.x = qkv;
  a.q = q_out;
  a.ldx = ldx * size;
  a.ldq = ldq * size;
  a.x_dtype = x_dtype;
  a.rows = rows;
  a.starts = starts;
  a.heads = heads;
  a.state = state;
  a.new_state = new_state;
  return hip_status(launch_cache_append(a, (hipStream_t)stream), "cache append launch");
}

}  // namespace mosaic
