// C ABI of the cached decoding (include/mosaic_cache.h): new tokens with norms
// of queries and keys, and cached tokens as rows.
#include "abi_cache_common.h"

using namespace mosaic;

extern "C" {

mosaic_status mosaic_cache_append_norm(const mosaic_kv_cache* cache, const void* qkv, int64_t ldx, int32_t x_dtype,
                                       int64_t rows, const int32_t* starts, int32_t heads, const mosaic_qk_norm* norm,
                                       const mosaic_rotary* rotary, void* q_out, int64_t ldq, const int32_t* state,
                                       int32_t* new_state, void* stream) {
  if (norm == nullptr) return fail(MOSAIC_ERR_INVALID_ARG, "norm is NULL");
  return append_tokens(cache, qkv, ldx, x_dtype, rows, starts, heads, norm, rotary, q_out, ldq, state, new_state, stream);
}

mosaic_status mosaic_cache_read(const mosaic_kv_cache* cache, const int32_t* lengths, int64_t rows,
                                const int32_t* starts, const int32_t* first, int32_t out_dtype, void* k_out,
                                int64_t ldk, void* v_out, int64_t ldv, void* stream) {
  ReadLaunch a{};
  mosaic_status st = view_of(cache, &a.c);
  if (st != MOSAIC_OK) return st;
  if (rows < 0) return fail(MOSAIC_ERR_INVALID_ARG, "negative size");
  if (rows > (1 << 24)) return fail(MOSAIC_ERR_UNSUPPORTED, "more than 2^24 rows");
  if (starts == nullptr && rows != a.c.batch)
    return fail(MOSAIC_ERR_INVALID_ARG, "%lld rows for %d sequences need starts", (long long)rows, a.c.batch);
  if (a.c.batch == 0 && rows > 0) return fail(MOSAIC_ERR_INVALID_ARG, "tokens of no sequence");
  if (out_dtype < MOSAIC_F32 || out_dtype > MOSAIC_F16) return fail(MOSAIC_ERR_INVALID_ARG, "unknown dtype %d", out_dtype);
  if (out_dtype != MOSAIC_F32 && out_dtype != a.c.dtype && a.c.dtype != MOSAIC_E2M1)
    return fail(MOSAIC_ERR_UNSUPPORTED, "rows must be float32 or of the cache's type");
  if (rows == 0) return MOSAIC_OK;
  if (lengths == nullptr) return fail(MOSAIC_ERR_INVALID_ARG, "lengths is NULL");
  const int64_t size = size_of(out_dtype), width = (int64_t)a.c.kv_heads * a.c.head_dim;
  if ((st = check_rows(k_out, rows, ldk, width, size, "k_out")) != MOSAIC_OK) return st;
  if ((st = check_rows(v_out, rows, ldv, width, size, "v_out")) != MOSAIC_OK) return st;
  const int64_t kn = extent(rows, ldk, width, size), vn = extent(rows, ldv, width, size);
  if (rows_overlap(k_out, ldk * size, width * size, v_out, ldv * size, width * size, rows))
    return fail(MOSAIC_ERR_INVALID_ARG, "k_out overlaps v_out");
  if (a.c.pages > 0) {
    const int64_t row = a.c.dtype == MOSAIC_E2M1 ? MOSAIC_E2M1_ROW_BYTES(a.c.head_dim) : a.c.head_dim * size_of(a.c.dtype);
    const int64_t held = (a.c.pages - 1) * a.c.page_stride + (a.c.kv_heads - 1) * a.c.head_stride +
                         ((1 << a.c.log2_page) - 1) * a.c.token_stride + row;
    for (const char* p : {a.c.k, a.c.v})
      if (overlap(p, held, k_out, kn) || overlap(p, held, v_out, vn))
        return fail(MOSAIC_ERR_INVALID_ARG, "k_out or v_out overlaps the cache");
  }
  a.lengths = lengths;
  a.rows = rows;
  a.starts = starts;
  a.first = first;
  a.out_dtype = out_dtype;
  a.k = k_out;
  a.v = v_out;
  a.ldk = ldk * size;
  a.ldv = ldv * size;
  return hip_status(launch_cache_read(a, (hipStream_t)stream), "cache read launch");
}

}  // extern "C"
