// Outputs of mosaic_cache_read side by side in one matrix, and every way in which
// they overlap, under the sanitizers.
#include <cstdio>
#include <set>

#include "../include/mosaic_cache.h"

extern int g_launches;
static char* const P = (char*)(uintptr_t)(1 << 20);   // aligned, never read

static int read(char* k, int64_t ldk, char* v, int64_t ldv, int64_t rows) {
  mosaic_kv_cache c{};
  c.k = P;
  c.v = P + (1 << 20);
  c.block_table = (const int32_t*)P;
  c.ldt = 4;
  c.pages = 4;
  c.page_stride = 16 * 16;
  c.token_stride = 16;
  c.dtype = MOSAIC_E2M1;
  c.batch = 1;
  c.max_blocks = 4;
  c.kv_heads = 1;
  c.head_dim = 8;                                     // rows of 32 bytes as float32
  c.page_size = 16;
  g_launches = 0;
  const int st = mosaic_cache_read(&c, (const int32_t*)P, rows, (const int32_t*)P, nullptr, MOSAIC_F32, k, ldk, v, ldv, nullptr);
  return st == MOSAIC_OK && g_launches == 1 ? 1 : st == MOSAIC_ERR_INVALID_ARG && g_launches == 0 ? 0 : -1;
}

int main() {
  int failures = 0;
  char* const base = P + (16 << 20);
  // all distances and row strides (float32 elements) of a few rows, against the bytes themselves
  for (int64_t rows : {1, 2, 3, 7})
    for (int64_t ldk : {8, 12, 16, 20, 24, 40})
      for (int64_t ldv : {8, 12, 16, 20, 24, 40})
        for (int64_t at = -280; at <= 280; at += 4) {
          std::set<int64_t> bytes;
          for (int64_t i = 0; i < rows; ++i)
            for (int64_t j = 0; j < 8; ++j) bytes.insert(i * ldk + j);
          bool meet = false;
          for (int64_t i = 0; i < rows; ++i)
            for (int64_t j = 0; j < 8; ++j) meet = meet || bytes.count(at + i * ldv + j);
          const int got = read(base, ldk, base + 4 * at, ldv, rows);
          // what overlaps is refused; of the others, all with one stride and all that lie apart as wholes are taken
          const bool apart = at >= (rows - 1) * ldk + 8 || at + (rows - 1) * ldv + 8 <= 0;
          if (got < 0 || (meet && got != 0) || (!meet && (apart || (ldk == ldv && at % ldk != 0)) && got != 1)) {
            ++failures;
            std::printf("rows %d ldk %d ldv %d at %d: %d, overlap %d\n", (int)rows, (int)ldk, (int)ldv, (int)at, got, meet);
          }
        }
  std::printf(failures == 0 ? "PASS\n" : "%d failures\n", failures);
  return failures != 0;
}
