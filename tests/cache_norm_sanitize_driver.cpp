// Calls of the cached decoding's C ABI with norms and caches in 4 bits under the
// sanitizers: refusals, empty calls, and extreme sizes and strides.
#include <climits>
#include <cmath>
#include <cstdio>
#include <functional>

#include "../include/mosaic_cache.h"

extern int g_launches;
static int failures = 0;
static char* const P = (char*)(uintptr_t)(1 << 20);   // aligned, never read

// heads of 80 elements in 4 bits: rows of 64 bytes
static mosaic_kv_cache cache() {
  mosaic_kv_cache c{};
  c.k = P;
  c.v = P + (1 << 24);
  c.weights = (float*)(P + (2 << 24));
  c.order = (int32_t*)(P + (3 << 24));
  c.block_table = (const int32_t*)P;
  c.ldt = 8;
  c.pages = 16;
  c.page_stride = 2 * 16 * 64;
  c.head_stride = 16 * 64;
  c.token_stride = 64;
  c.dtype = MOSAIC_E2M1;
  c.batch = 2;
  c.max_blocks = 8;
  c.kv_heads = 2;
  c.head_dim = 80;
  c.page_size = 16;
  return c;
}

struct Append {
  mosaic_kv_cache c = cache();
  mosaic_rotary r{(const float*)P, 100, nullptr, 0, 1, {40, 0, 0, 0}, 0};
  mosaic_qk_norm n{(const float*)P, (const float*)P, 1e-6f};
  int64_t ldx = 8 * 80, rows = 2, ldq = 320;
  int32_t dtype = MOSAIC_F32, heads = 4;
  const int32_t* starts = nullptr;
  bool rotary = true, norm = true;
  void* q = P + (1 << 22);
  const int32_t* state = (const int32_t*)P;
  int32_t* new_state = (int32_t*)P;
  int call() {
    return mosaic_cache_append_norm(&c, P, ldx, dtype, rows, starts, heads, norm ? &n : nullptr, rotary ? &r : nullptr, q,
                                    ldq, state, new_state, nullptr);
  }
};
struct Plain : Append {
  int call() { return mosaic_cache_append(&c, P, ldx, dtype, rows, starts, heads, rotary ? &r : nullptr, q, ldq, state, new_state, nullptr); }
};
struct Read {
  mosaic_kv_cache c = cache();
  const int32_t *lengths = (const int32_t*)P, *starts = nullptr, *first = nullptr;
  int64_t rows = 2, ldk = 160, ldv = 160;
  int32_t dtype = MOSAIC_F32;
  void *k = P + (40 << 20), *v = P + (41 << 20);
  int call() { return mosaic_cache_read(&c, lengths, rows, starts, first, dtype, k, ldk, v, ldv, nullptr); }
};
struct Attend {
  mosaic_kv_cache c = cache();
  int64_t max_len = 100, bytes = 1 << 20;
  int32_t dtype = MOSAIC_F32, heads = 4;
  int call() {
    return mosaic_cache_attend(&c, P, 320, dtype, heads, (const int32_t*)P, max_len, 0.125f, 1, P + (1 << 22), 320, P + (1 << 23),
                               bytes, nullptr);
  }
};
struct Evict {
  mosaic_kv_cache c = cache();
  int call() {
    return mosaic_cache_evict(&c, (const int32_t*)P, (int32_t*)P, 100, 50, 10, c.weights, c.order, nullptr, P + (1 << 23), 1 << 20, nullptr);
  }
};

template <class T> static void expect(int line, int status, int launches, std::function<void(T&)> change) {
  T t;
  change(t);
  g_launches = 0;
  const int st = t.call();
  if (st != status || g_launches != launches) {
    ++failures;
    std::printf("line %d: status %d, %d launches: %s\n", line, st, g_launches, mosaic_last_error_message());
  }
}
#define EXPECT(T, launches, change) expect<T>(__LINE__, 0, launches, [](T& t) { change; })
#define REFUSE(T, status, change) expect<T>(__LINE__, status, 0, [](T& t) { change; })
#define INVALID MOSAIC_ERR_INVALID_ARG
#define UNSUPPORTED MOSAIC_ERR_UNSUPPORTED
#define REFUSE_CACHE(status, change) \
  REFUSE(Append, status, change);    \
  REFUSE(Plain, status, change);     \
  REFUSE(Read, status, change);      \
  REFUSE(Attend, status, change);    \
  REFUSE(Evict, status, change)

int main() {
  EXPECT(Append, 1, (void)t);
  EXPECT(Plain, 1, (void)t);
  EXPECT(Read, 1, (void)t);
  EXPECT(Attend, 1, (void)t);
  EXPECT(Evict, 1, (void)t);
  // any activations over 4 bits; of 16 and 32 bits float32 or the cache's
  for (int d = 0; d < 3; ++d) {
    static int dtype;
    dtype = d;
    EXPECT(Append, 1, t.dtype = dtype);
    EXPECT(Plain, 1, t.dtype = dtype);
    EXPECT(Read, 1, t.dtype = dtype);
    EXPECT(Attend, 1, t.dtype = dtype);
  }
  REFUSE(Append, INVALID, t.dtype = MOSAIC_E2M1);
  REFUSE(Read, INVALID, t.dtype = MOSAIC_E2M1);
  REFUSE(Attend, INVALID, t.dtype = MOSAIC_E2M1);
  REFUSE(Read, INVALID, t.dtype = -1);
  EXPECT(Append, 1, t.c.dtype = MOSAIC_BF16; t.c.head_dim = 64; t.r.sections[0] = 32; t.dtype = MOSAIC_BF16);
  REFUSE(Append, UNSUPPORTED, t.c.dtype = MOSAIC_BF16; t.c.head_dim = 64; t.r.sections[0] = 32; t.dtype = MOSAIC_F16);
  EXPECT(Read, 1, t.c.dtype = MOSAIC_BF16; t.c.head_dim = 64);
  REFUSE(Read, UNSUPPORTED, t.c.dtype = MOSAIC_BF16; t.c.head_dim = 64; t.dtype = MOSAIC_F16);

  // rows of 64 bytes: by heads, by places, with gaps, and what overlaps
  EXPECT(Read, 1, t.c.token_stride = 2 * 64; t.c.head_stride = 64);
  EXPECT(Read, 1, t.c.token_stride = 80; t.c.head_stride = 16 * 80; t.c.page_stride = 2 * 16 * 80);
  EXPECT(Read, 1, t.c.head_dim = 72; t.c.token_stride = 48; t.c.head_stride = 16 * 48);
  EXPECT(Read, 1, t.c.head_dim = 256; t.c.token_stride = 160; t.c.head_stride = 16 * 160; t.c.page_stride = 2 * 16 * 160; t.ldk = t.ldv = 512);
  REFUSE_CACHE(INVALID, t.c.token_stride = 48);
  REFUSE_CACHE(INVALID, t.c.head_dim = 104);
  REFUSE_CACHE(INVALID, t.c.head_stride = 15 * 64);
  REFUSE_CACHE(INVALID, t.c.page_stride = 2 * 16 * 64 - 16);
  REFUSE_CACHE(INVALID, t.c.token_stride = 72);
  REFUSE_CACHE(INVALID, t.c.token_stride = -64);
  REFUSE_CACHE(UNSUPPORTED, t.c.head_stride = INT64_MAX);
  REFUSE_CACHE(UNSUPPORTED, t.c.token_stride = INT64_MAX);
  REFUSE_CACHE(UNSUPPORTED, t.c.page_stride = INT64_MAX);
  REFUSE_CACHE(UNSUPPORTED, t.c.head_dim = 84);
  REFUSE_CACHE(UNSUPPORTED, t.c.head_dim = 0);
  REFUSE_CACHE(UNSUPPORTED, t.c.head_dim = 264);
  REFUSE_CACHE(UNSUPPORTED, t.c.head_dim = INT_MIN);
  REFUSE_CACHE(INVALID, t.c.dtype = 3);
  REFUSE_CACHE(INVALID, t.c.dtype = 5);
  REFUSE_CACHE(INVALID, t.c.dtype = INT_MIN);
  REFUSE_CACHE(INVALID, t.c.k = nullptr);
  REFUSE_CACHE(INVALID, t.c.v = P + 8);
  REFUSE_CACHE(INVALID, t.c.block_table = nullptr);
  REFUSE_CACHE(INVALID, t.c.ldt = 7);
  EXPECT(Read, 1, t.c.ldt = 0);                         // a shared table is read, not written to
  REFUSE(Append, INVALID, t.c.ldt = 0);
  REFUSE(Evict, INVALID, t.c.ldt = 0);

  REFUSE(Append, INVALID, t.norm = false);
  REFUSE(Append, INVALID, t.n.q_weight = nullptr);
  REFUSE(Append, INVALID, t.n.k_weight = nullptr);
  REFUSE(Append, INVALID, t.n.eps = -1e-9f);
  REFUSE(Append, INVALID, t.n.eps = NAN);
  REFUSE(Append, INVALID, t.n.eps = INFINITY);
  EXPECT(Append, 1, t.n.eps = 0.0f);
  EXPECT(Append, 1, t.rotary = false);
  REFUSE(Append, INVALID, t.heads = 3);
  REFUSE(Append, INVALID, t.rows = 3);
  REFUSE(Append, INVALID, t.rows = -1);
  REFUSE(Append, UNSUPPORTED, t.rows = ((int64_t)1 << 22) + 1; t.starts = (const int32_t*)P);
  REFUSE(Append, INVALID, t.q = P);
  REFUSE(Append, INVALID, t.ldx = 8 * 80 - 8);
  REFUSE(Append, INVALID, t.ldx = INT64_MAX);
  REFUSE(Append, INVALID, t.r.sections[0] = 41);
  REFUSE(Append, INVALID, t.new_state = nullptr);
  EXPECT(Append, 0, t.c.batch = 0; t.rows = 0);

  REFUSE(Read, INVALID, t.rows = -1);
  REFUSE(Read, INVALID, t.rows = 3);
  REFUSE(Read, UNSUPPORTED, t.rows = ((int64_t)1 << 24) + 1; t.starts = (const int32_t*)P);
  REFUSE(Read, UNSUPPORTED, t.rows = INT64_MAX; t.starts = (const int32_t*)P);
  EXPECT(Read, 0, t.rows = 0; t.starts = (const int32_t*)P);
  EXPECT(Read, 0, t.c.batch = 0; t.rows = 0);
  REFUSE(Read, INVALID, t.c.batch = 0; t.rows = 2; t.starts = (const int32_t*)P);
  REFUSE(Read, INVALID, t.lengths = nullptr);
  REFUSE(Read, INVALID, t.k = nullptr);
  REFUSE(Read, INVALID, t.v = (char*)t.v + 4);
  REFUSE(Read, INVALID, t.ldk = 152);
  REFUSE(Read, INVALID, t.ldv = 162);
  REFUSE(Read, INVALID, t.ldv = INT64_MAX);
  REFUSE(Read, INVALID, t.v = (char*)t.k + 640);
  EXPECT(Read, 1, t.v = (char*)t.k + 1280);
  // the last byte of the cache's keys is at 16 pages of 2 x 16 rows of 64
  EXPECT(Read, 1, t.k = P + 16 * 2 * 16 * 64);
  REFUSE(Read, INVALID, t.k = P + 16 * 2 * 16 * 64 - 16);
  REFUSE(Read, INVALID, t.v = P + (1 << 24));
  EXPECT(Read, 1, t.c.pages = 0; t.c.k = t.c.v = nullptr);
  std::printf(failures == 0 ? "PASS\n" : "%d failures\n", failures);
  return failures != 0;
}
