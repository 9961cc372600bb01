// Calls of the cached decoding's C ABI under the sanitizers: every refusal,
// empty calls, and extreme sizes and strides, whose checks must not overflow.
#include <climits>
#include <cmath>
#include <cstdio>
#include <functional>

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
  c.dtype = MOSAIC_BF16;
  c.batch = 2;
  c.max_blocks = 8;
  c.kv_heads = 2;
  c.head_dim = 64;
  c.page_size = 16;
  return c;
}

struct Append {
  mosaic_kv_cache c = cache();
  mosaic_rotary r{(const float*)P, 100, nullptr, 0, 1, {32, 0, 0, 0}, 0};
  const void* x = P;
  int64_t ldx = 8 * 64, rows = 2, ldq = 256;
  int32_t dtype = MOSAIC_F32, heads = 4;
  const int32_t* starts = nullptr;
  bool rotary = true;
  void* q = P + (1 << 22);
  const int32_t* state = (const int32_t*)P;
  int32_t* new_state = (int32_t*)P;
  int call() { return mosaic_cache_append(&c, x, ldx, dtype, rows, starts, heads, rotary ? &r : nullptr, q, ldq, state, new_state, nullptr); }
};
struct Attend {
  mosaic_kv_cache c = cache();
  const void* q = P;
  int64_t ldq = 256, ldo = 256, max_len = 100, bytes = 1 << 20;
  int32_t dtype = MOSAIC_F32, heads = 4, accumulate = 1;
  const int32_t* lengths = (const int32_t*)P;
  float scale = 0.125f;
  void *out = P + (1 << 22), *work = P + (1 << 23);
  int call() { return mosaic_cache_attend(&c, q, ldq, dtype, heads, lengths, max_len, scale, accumulate, out, ldo, work, bytes, nullptr); }
};
struct Evict {
  mosaic_kv_cache c = cache();
  const int32_t* state = (const int32_t*)P;
  int32_t* new_state = (int32_t*)P;
  int64_t max_len = 100, budget = 50, recent = 10, bytes = 1 << 20;
  float* weights = cache().weights;
  int32_t *order = cache().order, *kept = nullptr;
  void* work = P + (1 << 23);
  int call() { return mosaic_cache_evict(&c, state, new_state, max_len, budget, recent, weights, order, kept, work, bytes, nullptr); }
};

template <class T> static void refuse(int line, int status, std::function<void(T&)> change) {
  T t;
  change(t);
  g_launches = 0;
  const int st = t.call();
  if (st != status || g_launches != 0) {
    ++failures;
    std::printf("line %d: status %d, %d launches: %s\n", line, st, g_launches, mosaic_last_error_message());
  }
}
#define REFUSE(T, status, change) refuse<T>(__LINE__, status, [](T& t) { change; })
#define INVALID MOSAIC_ERR_INVALID_ARG
#define UNSUPPORTED MOSAIC_ERR_UNSUPPORTED
#define REFUSE_CACHE(status, change) \
  REFUSE(Append, status, change);    \
  REFUSE(Attend, status, change);    \
  REFUSE(Evict, status, change)

int main() {
  EXPECT(0, 1, Append().call());
  EXPECT(0, 1, Attend().call());
  EXPECT(0, 1, Evict().call());

  REFUSE_CACHE(INVALID, t.c.dtype = 3);
  REFUSE_CACHE(INVALID, t.c.batch = -1);
  REFUSE_CACHE(INVALID, t.c.pages = -1);
  REFUSE_CACHE(INVALID, t.c.kv_heads = 0);
  REFUSE_CACHE(INVALID, t.c.max_blocks = -1);
  REFUSE_CACHE(UNSUPPORTED, t.c.head_dim = 60);
  REFUSE_CACHE(UNSUPPORTED, t.c.head_dim = 0);
  REFUSE_CACHE(UNSUPPORTED, t.c.head_dim = 264);
  REFUSE_CACHE(UNSUPPORTED, t.c.page_size = 24);
  REFUSE_CACHE(UNSUPPORTED, t.c.page_size = 8);
  REFUSE_CACHE(UNSUPPORTED, t.c.page_size = 8192);
  REFUSE_CACHE(UNSUPPORTED, t.c.page_size = INT_MIN);
  REFUSE_CACHE(UNSUPPORTED, t.c.kv_heads = 1025);
  REFUSE_CACHE(UNSUPPORTED, t.c.batch = 65536);
  REFUSE_CACHE(UNSUPPORTED, t.c.pages = (int64_t)1 << 31);
  REFUSE_CACHE(UNSUPPORTED, t.c.max_blocks = INT_MAX);
  REFUSE_CACHE(INVALID, t.c.page_stride = -16);
  REFUSE_CACHE(INVALID, t.c.token_stride = INT64_MIN);
  REFUSE_CACHE(UNSUPPORTED, t.c.page_stride = INT64_MAX);
  REFUSE_CACHE(UNSUPPORTED, t.c.head_stride = INT64_MAX);
  REFUSE_CACHE(UNSUPPORTED, t.c.token_stride = INT64_MAX);
  REFUSE_CACHE(INVALID, t.c.token_stride = 68);
  REFUSE_CACHE(INVALID, t.c.token_stride = 56);
  REFUSE_CACHE(INVALID, t.c.head_stride = 8);
  REFUSE_CACHE(INVALID, t.c.page_stride = 2040);
  REFUSE_CACHE(INVALID, t.c.block_table = nullptr);
  REFUSE_CACHE(INVALID, t.c.ldt = 7);
  REFUSE_CACHE(INVALID, t.c.k = nullptr);
  REFUSE_CACHE(INVALID, t.c.v = P + 8);

  REFUSE(Append, INVALID, t.rows = -1);
  REFUSE(Append, INVALID, t.rows = 3);
  REFUSE(Append, INVALID, t.c.batch = 0);
  REFUSE(Append, UNSUPPORTED, t.starts = (const int32_t*)P; t.rows = INT64_MAX);
  REFUSE(Append, INVALID, t.heads = 3);
  REFUSE(Append, INVALID, t.heads = 0);
  REFUSE(Append, INVALID, t.heads = INT_MIN);
  REFUSE(Append, UNSUPPORTED, t.heads = 8192);
  REFUSE(Append, INVALID, t.dtype = -1);
  REFUSE(Append, UNSUPPORTED, t.dtype = MOSAIC_F16);
  REFUSE(Append, INVALID, t.x = nullptr);
  REFUSE(Append, INVALID, t.x = P + 4);
  REFUSE(Append, INVALID, t.ldx = 508);
  REFUSE(Append, INVALID, t.ldx = 513);
  REFUSE(Append, INVALID, t.ldx = INT64_MAX);
  REFUSE(Append, INVALID, t.q = nullptr);
  REFUSE(Append, INVALID, t.q = P + 64);
  REFUSE(Append, INVALID, t.ldq = 255);
  REFUSE(Append, INVALID, t.state = nullptr);
  REFUSE(Append, INVALID, t.new_state = nullptr);
  REFUSE(Append, INVALID, t.new_state = (int32_t*)P + 3);
  REFUSE(Append, INVALID, t.r.naxes = 0);
  REFUSE(Append, INVALID, t.r.naxes = 5);
  REFUSE(Append, INVALID, t.r.sections[0] = 33);
  REFUSE(Append, INVALID, t.r.sections[0] = 0);
  REFUSE(Append, INVALID, t.r.sections[0] = INT_MAX);
  REFUSE(Append, INVALID, t.r.naxes = 2; t.r.sections[1] = -8);
  REFUSE(Append, INVALID, t.r.table = nullptr);
  REFUSE(Append, INVALID, t.r.rows = 0);
  REFUSE(Append, UNSUPPORTED, t.r.rows = INT64_MAX);
  REFUSE(Append, INVALID, t.r.positions = (const int32_t*)P; t.r.ldp = 1);

  REFUSE(Attend, INVALID, t.heads = 5);
  REFUSE(Attend, INVALID, t.heads = -4);
  REFUSE(Attend, UNSUPPORTED, t.heads = 8192);
  REFUSE(Attend, UNSUPPORTED, t.dtype = MOSAIC_F16);
  REFUSE(Attend, INVALID, t.dtype = 9);
  REFUSE(Attend, INVALID, t.max_len = -1);
  REFUSE(Attend, UNSUPPORTED, t.c.batch = 65535; t.c.max_blocks = t.c.ldt = 1 << 26; t.max_len = INT64_MAX);
  REFUSE(Attend, INVALID, t.scale = NAN);
  REFUSE(Attend, INVALID, t.scale = 3e38f);
  REFUSE(Attend, INVALID, t.q = nullptr);
  REFUSE(Attend, INVALID, t.out = (void*)(P + 128));
  REFUSE(Attend, INVALID, t.ldq = 252);
  REFUSE(Attend, INVALID, t.ldo = 257);
  REFUSE(Attend, INVALID, t.ldo = INT64_MAX);
  REFUSE(Attend, INVALID, t.lengths = nullptr);
  REFUSE(Attend, INVALID, t.c.weights = nullptr);
  REFUSE(Attend, INVALID, t.bytes = 0);
  REFUSE(Attend, INVALID, t.work = nullptr);
  REFUSE(Attend, INVALID, t.work = P + 8);

  REFUSE(Evict, INVALID, t.max_len = -1);
  REFUSE(Evict, INVALID, t.budget = 0);
  REFUSE(Evict, INVALID, t.recent = -1);
  REFUSE(Evict, INVALID, t.recent = 51);
  REFUSE(Evict, INVALID, t.weights = nullptr);
  REFUSE(Evict, INVALID, t.order = nullptr);
  REFUSE(Evict, INVALID, t.c.order = nullptr);
  REFUSE(Evict, INVALID, t.weights = t.c.weights + 1);
  REFUSE(Evict, INVALID, t.order = t.c.order - 1);
  REFUSE(Evict, INVALID, t.state = nullptr);
  REFUSE(Evict, INVALID, t.new_state = (int32_t*)P + 1);
  REFUSE(Evict, INVALID, t.bytes = 8);
  REFUSE(Evict, INVALID, t.work = P + 4);

  EXPECT(INVALID, 0, mosaic_cache_append(nullptr, P, 512, 0, 2, nullptr, 4, nullptr, P, 256, nullptr, nullptr, nullptr));
  EXPECT(INVALID, 0, mosaic_cache_evict(nullptr, nullptr, nullptr, 0, 1, 0, nullptr, nullptr, nullptr, nullptr, 0, nullptr));
  int64_t bytes = -1;
  mosaic_kv_cache c = cache();
  EXPECT(INVALID, 0, mosaic_cache_attend_workspace(&c, 4, 100, 0, nullptr));
  EXPECT(INVALID, 0, mosaic_cache_attend_workspace(nullptr, 4, 100, 0, &bytes));
  EXPECT(INVALID, 0, mosaic_cache_evict_workspace(&c, 100, 0, &bytes));
  EXPECT(INVALID, 0, mosaic_cache_evict_workspace(&c, 100, 5, nullptr));
  EXPECT(0, 0, mosaic_cache_attend_workspace(&c, 4, INT64_MAX, 1, &bytes));
  if (bytes != 2 * 4 * 128 * 4) ++failures, std::printf("workspace of %lld bytes\n", (long long)bytes);

  // nothing to do, nothing needed
  {
    Attend t;
    t.c.batch = 0;
    t.q = t.out = t.work = nullptr;
    t.lengths = nullptr;
    t.bytes = 0;
    EXPECT(0, 0, t.call());
    Evict e;
    e.c.batch = 0;
    e.state = e.new_state = nullptr;
    EXPECT(0, 0, e.call());
    Append a;
    a.c.batch = 0;
    a.rows = 0;
    a.x = a.q = nullptr;
    a.state = a.new_state = nullptr;
    EXPECT(0, 0, a.call());
  }
  // a head or page alone has no stride; heads within places; no rotation
  {
    Append t;
    t.c.kv_heads = 1;
    t.c.head_stride = -5;
    t.ldx = 384;
    EXPECT(0, 1, t.call());
    t = Append();
    t.c.pages = 1;
    t.c.page_stride = INT64_MIN;
    EXPECT(0, 1, t.call());
    t = Append();
    t.c.head_stride = 64;
    t.c.token_stride = 128;
    t.rotary = false;
    EXPECT(0, 1, t.call());
  }
  std::printf(failures == 0 ? "PASS\n" : "%d FAILED\n", failures);
  return failures != 0;
}
