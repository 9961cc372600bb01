// What the two kernels that append to the cache share (cache_append.hip,
// cache_append_norm.hip).
#pragma once

#include "cache.h"
#include "device_common.h"

namespace mosaic {
namespace {

constexpr int kFewRows = 256;     // no more than one workgroup per compute unit
// Rows that the 32 MiB of second-level cache cannot hold pass by it (168 MB of
// q|k|v: 61 us, 69 us through it); fewer are left there for the attention that
// comes next.
constexpr int64_t kStreamBytes = (int64_t)32 << 20;

// (held, seen) of sequence b after n new tokens.
__device__ __forceinline__ void advance(const AppendLaunch& a, int b, int32_t n, int64_t slots) {
  const int64_t held = (int64_t)held_tokens(a.state, b, slots) + n;
  const int32_t seen = a.state[a.c.batch + b];
  a.new_state[b] = (int32_t)(held < slots ? held : slots);
  a.new_state[a.c.batch + b] = (int32_t)((uint32_t)seen + (uint32_t)n);
}

__device__ __forceinline__ int32_t fresh_tokens(const AppendLaunch& a, int b) {
  if (a.starts == nullptr) return 1;
  const int64_t n = (int64_t)a.starts[b + 1] - a.starts[b];
  return n < 0 ? 0 : n > a.rows ? (int32_t)a.rows : (int32_t)n;
}

template <class T, int V> struct alignas(sizeof(T) * V) Chunk { T e[V]; };

// STREAM: past the caches.
template <bool STREAM, class T> __device__ __forceinline__ T load_piece(const char* p) {
  if constexpr (STREAM) return __builtin_bit_cast(T, __builtin_nontemporal_load((const u32x4*)p));
  else return *(const T*)p;
}
template <bool STREAM, class T> __device__ __forceinline__ void store_piece(char* p, T v) {
  if constexpr (STREAM && sizeof(T) == 16) __builtin_nontemporal_store(__builtin_bit_cast(u32x4, v), (u32x4*)p);
  else *(T*)p = v;
}

}  // namespace
}  // namespace mosaic
