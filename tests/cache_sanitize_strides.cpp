// Row strides of the cached decoding's block table and positions under the
// sanitizers: 0 (a row that is shared) is taken where nothing is written
// through it, any other stride below the row's length is refused.
#include <cstdio>

#include "../include/mosaic_cache.h"

extern int g_launches;
static int failures = 0;

#define EXPECT(status, launches, call)                                                       \
  do {                                                                                       \
    g_launches = 0;                                                                          \
    const int st = (call);                                                                   \
    if (st != (status) || g_launches != (launches)) {                                        \
      ++failures;                                                                            \
      std::printf("line %d: status %d, %d launches: %s\n", __LINE__, st, g_launches,         \
                  mosaic_last_error_message());                                              \
    }                                                                                        \
  } while (0)

static char* const P = (char*)(uintptr_t)(1 << 20);   // aligned, never read

static mosaic_kv_cache cache(int64_t ldt, int32_t batch) {
  mosaic_kv_cache c{};
  c.k = P;
  c.v = P + (1 << 24);
  c.weights = (float*)(P + (2 << 24));
  c.order = (int32_t*)(P + (3 << 24));
  c.block_table = (const int32_t*)P;
  c.ldt = ldt;
  c.pages = 16;
  c.page_stride = 2 * 16 * 64;
  c.head_stride = 16 * 64;
  c.token_stride = 64;
  c.dtype = MOSAIC_BF16;
  c.batch = batch;
  c.max_blocks = 8;
  c.kv_heads = 2;
  c.head_dim = 64;
  c.page_size = 16;
  return c;
}

static int append(int64_t ldt, int32_t batch, int64_t ldp, int32_t axes) {
  const mosaic_kv_cache c = cache(ldt, batch);
  const mosaic_rotary r{(const float*)P, 100, (const int32_t*)P, ldp, axes, {8, 12, 12, 0}, 0};
  return mosaic_cache_append(&c, P, 512, MOSAIC_F32, batch, nullptr, 4, &r, P + (1 << 22), 256, (const int32_t*)P,
                             (int32_t*)P, nullptr);
}
static int attend(int64_t ldt, int32_t batch, int32_t accumulate) {
  const mosaic_kv_cache c = cache(ldt, batch);
  return mosaic_cache_attend(&c, P, 256, MOSAIC_F32, 4, (const int32_t*)P, 100, 0.125f, accumulate, P + (1 << 22), 256,
                             P + (1 << 23), 1 << 20, nullptr);
}
static int evict(int64_t ldt, int32_t batch) {
  const mosaic_kv_cache c = cache(ldt, batch);
  return mosaic_cache_evict(&c, (const int32_t*)P, (int32_t*)P, 100, 50, 10, c.weights, c.order, nullptr, P + (1 << 23),
                            1 << 20, nullptr);
}

int main() {
  const int invalid = MOSAIC_ERR_INVALID_ARG;
  EXPECT(0, 1, append(8, 3, 3, 3));
  EXPECT(0, 1, append(8, 3, 0, 3));
  EXPECT(0, 1, append(8, 1, 0, 1));
  for (int64_t ldp : {1, 2, -1}) EXPECT(invalid, 0, append(8, 3, ldp, 3));

  EXPECT(0, 1, attend(0, 3, 0));
  for (int64_t ldt : {1, 7, -8}) EXPECT(invalid, 0, attend(ldt, 3, 0));
  EXPECT(invalid, 0, attend(0, 3, 1));
  EXPECT(invalid, 0, append(0, 3, 3, 3));
  EXPECT(invalid, 0, evict(0, 3));
  // one sequence shares its table with nobody
  EXPECT(0, 1, attend(0, 1, 1));
  EXPECT(0, 1, append(0, 1, 1, 3));
  EXPECT(0, 1, evict(0, 1));
  std::printf(failures == 0 ? "PASS\n" : "%d FAILED\n", failures);
  return failures != 0;
}
