// C ABI of the cached decoding (include/mosaic_cache.h): validation and
// dispatch.
#include "abi_common.h"
#include "cache.h"

using namespace mosaic;

namespace {

constexpr int64_t kMaxSlots = (int64_t)1 << 30;     // of one sequence: slots fit int32 with room

int64_t size_of(int32_t ftype) { return ftype == MOSAIC_F32 ? 4 : 2; }

bool overlap(const void* a, int64_t an, const void* b, int64_t bn) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + (uintptr_t)bn && y < x + (uintptr_t)an;
}

// Bytes from the first to the last element of rows x cols.
int64_t extent(int64_t rows, int64_t ld, int64_t cols, int64_t size) { return ((rows - 1) * ld + cols) * size; }

mosaic_status view_of(const mosaic_kv_cache* c, CacheView* v) {
  if (c == nullptr) return fail(MOSAIC_ERR_INVALID_ARG, "cache is NULL");
  if (c->dtype < MOSAIC_F32 || c->dtype > MOSAIC_F16) return fail(MOSAIC_ERR_INVALID_ARG, "unknown cache dtype %d", c->dtype);
  if (c->batch < 0 || c->pages < 0 || c->max_blocks < 0 || c->kv_heads < 1)
    return fail(MOSAIC_ERR_INVALID_ARG, "negative size, or no key/value heads");
  if (c->head_dim < 8 || c->head_dim > 256 || c->head_dim % 8 != 0)
    return fail(MOSAIC_ERR_UNSUPPORTED, "head_dim %d is not a multiple of 8 in [8, 256]", c->head_dim);
  if (c->page_size < 16 || c->page_size > 4096 || (c->page_size & (c->page_size - 1)) != 0)
    return fail(MOSAIC_ERR_UNSUPPORTED, "page_size %d is not a power of two in [16, 4096]", c->page_size);
  if (c->kv_heads > 1024) return fail(MOSAIC_ERR_UNSUPPORTED, "more than 1024 key/value heads");
  if (c->batch > 65535 || c->pages > 0x7FFFFFFF || c->max_blocks > kMaxSlots / c->page_size)
    return fail(MOSAIC_ERR_UNSUPPORTED, "more than 65535 sequences, 2^31 - 1 pages or 2^30 slots of a sequence");
  const int64_t es = size_of(c->dtype);
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
  const bool by_head = c->token_stride >= c->head_dim && (c->kv_heads == 1 || head_stride >= places + c->head_dim);
  const bool by_place = (c->kv_heads == 1 || head_stride >= c->head_dim) && c->token_stride >= heads + c->head_dim;
  if (!by_head && !by_place) return fail(MOSAIC_ERR_INVALID_ARG, "rows of a page overlap");
  if (c->pages > 1 && page_stride < places + heads + c->head_dim)
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
mosaic_status check_own_pages(const CacheView& v) {
  if (v.batch > 1 && v.max_blocks > 0 && v.ldt == 0)
    return fail(MOSAIC_ERR_INVALID_ARG, "sequences that share their block table cannot be written to");
  return MOSAIC_OK;
}

int64_t slots_of(const CacheView& v) { return (int64_t)v.max_blocks << v.log2_page; }

mosaic_status check_heads(const CacheView& v, int32_t heads, int32_t x_dtype) {
  if (heads < 1 || heads % v.kv_heads != 0)
    return fail(MOSAIC_ERR_INVALID_ARG, "%d query heads are no multiple of %d key/value heads", heads, v.kv_heads);
  if (heads > 4096) return fail(MOSAIC_ERR_UNSUPPORTED, "more than 4096 query heads");
  if (x_dtype < MOSAIC_F32 || x_dtype > MOSAIC_F16) return fail(MOSAIC_ERR_INVALID_ARG, "unknown dtype %d", x_dtype);
  if (x_dtype != MOSAIC_F32 && x_dtype != v.dtype)
    return fail(MOSAIC_ERR_UNSUPPORTED, "activations must be float32 or of the cache's type");
  return MOSAIC_OK;
}

// A rows x cols matrix that kernels access 16 bytes at a time.
mosaic_status check_rows(const void* p, int64_t rows, int64_t ld, int64_t cols, int64_t size, const char* name) {
  if (p == nullptr) return fail(MOSAIC_ERR_INVALID_ARG, "%s is NULL", name);
  if (ld < cols) return fail(MOSAIC_ERR_INVALID_ARG, "leading dimension of %s < %lld", name, (long long)cols);
  if (ld > INT64_MAX / 16 / rows) return fail(MOSAIC_ERR_INVALID_ARG, "leading dimension of %s too large", name);
  if (!aligned16(p) || ld * size % 16 != 0) return fail(MOSAIC_ERR_INVALID_ARG, "rows of %s must be 16-byte aligned", name);
  return MOSAIC_OK;
}

mosaic_status check_state(const CacheView& v, const int32_t* state, const int32_t* new_state) {
  if (state == nullptr || new_state == nullptr) return fail(MOSAIC_ERR_INVALID_ARG, "state or new_state is NULL");
  if (state != new_state && overlap(state, 8 * (int64_t)v.batch, new_state, 8 * (int64_t)v.batch))
    return fail(MOSAIC_ERR_INVALID_ARG, "new_state overlaps state");
  return MOSAIC_OK;
}

mosaic_status check_workspace(const void* p, int64_t bytes, int64_t needed) {
  if (bytes < needed)
    return fail(MOSAIC_ERR_INVALID_ARG, "workspace of %lld bytes, needs %lld", (long long)bytes, (long long)needed);
  if (needed > 0 && (p == nullptr || !aligned16(p)))
    return fail(MOSAIC_ERR_INVALID_ARG, "workspace is NULL or not 16-byte aligned");
  return MOSAIC_OK;
}

mosaic_status check_attend(const mosaic_kv_cache* cache, int32_t heads, int64_t max_len, int32_t accumulate,
                           AttendLaunch* a) {
  const mosaic_status st = view_of(cache, &a->c);
  if (st != MOSAIC_OK) return st;
  if (max_len < 0) return fail(MOSAIC_ERR_INVALID_ARG, "negative max_len");
  if (heads < 1 || heads % a->c.kv_heads != 0)
    return fail(MOSAIC_ERR_INVALID_ARG, "%d query heads are no multiple of %d key/value heads", heads, a->c.kv_heads);
  if (heads > 4096) return fail(MOSAIC_ERR_UNSUPPORTED, "more than 4096 query heads");
  const mosaic_status own = accumulate != 0 ? check_own_pages(a->c) : MOSAIC_OK;
  if (own != MOSAIC_OK) return own;
  a->heads = heads;
  a->max_len = max_len < slots_of(a->c) ? max_len : slots_of(a->c);
  a->accumulate = accumulate != 0;
  if (a->c.batch > 0 && a->max_len > ((int64_t)1 << 36) / a->c.batch)     // steps of all sequences are counted in 32 bits
    return fail(MOSAIC_ERR_UNSUPPORTED, "more than 2^36 slots");
  return MOSAIC_OK;
}

mosaic_status check_evict(const mosaic_kv_cache* cache, int64_t max_len, int64_t budget, EvictLaunch* a) {
  mosaic_status st = view_of(cache, &a->c);
  if (st != MOSAIC_OK || (st = check_own_pages(a->c)) != MOSAIC_OK) return st;
  if (max_len < 0 || budget < 1) return fail(MOSAIC_ERR_INVALID_ARG, "negative max_len, or a budget below 1");
  a->max_len = max_len < slots_of(a->c) ? max_len : slots_of(a->c);
  a->budget = budget;
  return MOSAIC_OK;
}

}  // namespace

extern "C" {

mosaic_status mosaic_cache_append(const mosaic_kv_cache* cache, const void* qkv, int64_t ldx, int32_t x_dtype,
                                  int64_t rows, const int32_t* starts, int32_t heads, const mosaic_rotary* rotary,
                                  void* q_out, int64_t ldq, const int32_t* state, int32_t* new_state, void* stream) {
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

mosaic_status mosaic_cache_attend_workspace(const mosaic_kv_cache* cache, int32_t heads, int64_t max_len,
                                            int32_t accumulate, int64_t* bytes) {
  AttendLaunch a{};
  if (bytes == nullptr) return fail(MOSAIC_ERR_INVALID_ARG, "bytes is NULL");
  const mosaic_status st = check_attend(cache, heads, max_len, accumulate, &a);
  if (st == MOSAIC_OK) *bytes = a.c.batch == 0 ? 0 : cache_attend_workspace(a.c, heads, a.max_len, a.accumulate);
  return st;
}

mosaic_status mosaic_cache_attend(const mosaic_kv_cache* cache, const void* q, int64_t ldq, int32_t x_dtype,
                                  int32_t heads, const int32_t* lengths, int64_t max_len, float scale,
                                  int32_t accumulate, void* out, int64_t ldo, void* workspace,
                                  int64_t workspace_bytes, void* stream) {
  AttendLaunch a{};
  mosaic_status st = check_attend(cache, heads, max_len, accumulate, &a);
  if (st != MOSAIC_OK) return st;
  if ((st = check_heads(a.c, heads, x_dtype)) != MOSAIC_OK) return st;
  a.scale_log2 = scale * 1.44269504088896340736f;
  if (!std::isfinite(a.scale_log2)) return fail(MOSAIC_ERR_INVALID_ARG, "scale is not finite, or too large");
  if (a.c.batch == 0) return MOSAIC_OK;
  const int64_t size = size_of(x_dtype), width = (int64_t)heads * a.c.head_dim;
  if ((st = check_rows(q, a.c.batch, ldq, width, size, "q")) != MOSAIC_OK) return st;
  if ((st = check_rows(out, a.c.batch, ldo, width, size, "out")) != MOSAIC_OK) return st;
  if (overlap(q, extent(a.c.batch, ldq, width, size), out, extent(a.c.batch, ldo, width, size)))
    return fail(MOSAIC_ERR_INVALID_ARG, "out overlaps q");
  if (lengths == nullptr) return fail(MOSAIC_ERR_INVALID_ARG, "lengths is NULL");
  if (a.accumulate && a.c.weights == nullptr) return fail(MOSAIC_ERR_INVALID_ARG, "the cache has no weights to add to");
  st = check_workspace(workspace, workspace_bytes, cache_attend_workspace(a.c, heads, a.max_len, a.accumulate));
  if (st != MOSAIC_OK) return st;
  a.q = q;
  a.out = out;
  a.ldq = ldq * size;
  a.ldo = ldo * size;
  a.x_dtype = x_dtype;
  a.lengths = lengths;
  a.workspace = workspace;
  return hip_status(launch_cache_attend(a, (hipStream_t)stream), "cache attend launch");
}

mosaic_status mosaic_cache_evict_workspace(const mosaic_kv_cache* cache, int64_t max_len, int64_t budget,
                                           int64_t* bytes) {
  EvictLaunch a{};
  if (bytes == nullptr) return fail(MOSAIC_ERR_INVALID_ARG, "bytes is NULL");
  const mosaic_status st = check_evict(cache, max_len, budget, &a);
  if (st == MOSAIC_OK) *bytes = a.c.batch == 0 ? 0 : cache_evict_workspace(a.c, a.max_len, budget);
  return st;
}

mosaic_status mosaic_cache_evict(const mosaic_kv_cache* cache, const int32_t* state, int32_t* new_state,
                                 int64_t max_len, int64_t budget, int64_t recent, float* new_weights,
                                 int32_t* new_order, int32_t* kept, void* workspace, int64_t workspace_bytes,
                                 void* stream) {
  EvictLaunch a{};
  mosaic_status st = check_evict(cache, max_len, budget, &a);
  if (st != MOSAIC_OK) return st;
  if (recent < 0 || recent > budget)
    return fail(MOSAIC_ERR_INVALID_ARG, "recent %lld outside [0, budget = %lld]", (long long)recent, (long long)budget);
  if (a.c.batch == 0) return MOSAIC_OK;
  if ((st = check_state(a.c, state, new_state)) != MOSAIC_OK) return st;
  const int64_t numbers = a.c.pages * (int64_t)a.c.kv_heads * 4 << a.c.log2_page;
  if (numbers > 0) {
    if (a.c.weights == nullptr || a.c.order == nullptr || new_weights == nullptr || new_order == nullptr)
      return fail(MOSAIC_ERR_INVALID_ARG, "eviction needs weights, order, new_weights and new_order");
    if ((new_weights != a.c.weights && overlap(new_weights, numbers, a.c.weights, numbers)) ||
        (new_order != a.c.order && overlap(new_order, numbers, a.c.order, numbers)))
      return fail(MOSAIC_ERR_INVALID_ARG, "new_weights or new_order overlaps the cache's");
  }
  st = check_workspace(workspace, workspace_bytes, cache_evict_workspace(a.c, a.max_len, budget));
  if (st != MOSAIC_OK) return st;
  a.state = state;
  a.new_state = new_state;
  a.recent = recent;
  a.new_weights = new_weights;
  a.new_order = new_order;
  a.kept = kept;
  a.workspace = workspace;
  return hip_status(launch_cache_evict(a, (hipStream_t)stream), "cache evict launch");
}

}  // extern "C"
