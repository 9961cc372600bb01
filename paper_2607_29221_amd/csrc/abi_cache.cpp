// C ABI of the cached decoding (include/mosaic_cache.h): validation and
// dispatch.
#include "abi_cache_common.h"

using namespace mosaic;

namespace {

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
  return append_tokens(cache, qkv, ldx, x_dtype, rows, starts, heads, nullptr, rotary, q_out, ldq, state, new_state, stream);
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
