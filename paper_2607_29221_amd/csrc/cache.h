// Launch interfaces between the C ABI layer of the cached decoding
// (abi_cache.cpp) and its kernels, and what the kernels share. Every launcher
// assumes its arguments were validated by the ABI layer.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/mosaic_cache.h"

namespace mosaic {

// The cache as the kernels see it: strides in bytes, the page size by its
// logarithm.
struct CacheView {
  char* k;
  char* v;
  float* weights;
  int32_t* order;
  const int32_t* table;
  int64_t ldt;
  int64_t page_stride, head_stride, token_stride;
  int32_t pages, batch, max_blocks, kv_heads, head_dim, log2_page;
  int32_t dtype;
};

constexpr int kMaxAxes = 4;
struct RotaryView {
  const float* table;       // null: no rotation
  int64_t rows;
  const int32_t* positions; // null: the token's number
  int64_t ldp;
  int32_t ends[kMaxAxes];   // pairs up to ends[a] belong to axis a or an earlier one
  int32_t pairs;
  int32_t interleaved;
};

struct AppendLaunch {
  CacheView c;
  RotaryView rot;
  const void* x;
  void* q;
  int64_t ldx, ldq;         // bytes
  int32_t x_dtype;
  int64_t rows;
  const int32_t* starts;
  int32_t heads;
  const int32_t* state;
  int32_t* new_state;
};
hipError_t launch_cache_append(const AppendLaunch& a, hipStream_t s);

struct AttendLaunch {
  CacheView c;
  const void* q;
  void* out;
  int64_t ldq, ldo;         // bytes
  int32_t x_dtype;
  int32_t heads;
  const int32_t* lengths;
  int64_t max_len;          // at most the slots of the block table
  float scale_log2;         // scale * log2(e): scores are kept in powers of two
  int32_t accumulate;
  void* workspace;
};
int64_t cache_attend_workspace(const CacheView& c, int32_t heads, int64_t max_len, int32_t accumulate);
hipError_t launch_cache_attend(const AttendLaunch& a, hipStream_t s);

struct EvictLaunch {
  CacheView c;
  const int32_t* state;
  int32_t* new_state;
  int64_t max_len;          // at most the slots of the block table
  int64_t budget, recent;
  float* new_weights;
  int32_t* new_order;
  int32_t* kept;
  void* workspace;
};
int64_t cache_evict_workspace(const CacheView& c, int64_t max_len, int64_t budget);
hipError_t launch_cache_evict(const EvictLaunch& a, hipStream_t s);

#ifdef __HIPCC__

// Element types of activations and cache rows by mosaic_ftype.
template <int FT> struct FloatType;
template <> struct FloatType<MOSAIC_F32> { typedef float type; };
template <> struct FloatType<MOSAIC_BF16> { typedef __bf16 type; };
template <> struct FloatType<MOSAIC_F16> { typedef _Float16 type; };

// Memory that no kernel on the stream writes while this one reads it, at
// addresses that a wave has in common: through the scalar cache, so the answer
// does not wait for the vector loads that are under way.
typedef const __attribute__((address_space(4))) int32_t* uniform_i32;

// Tokens that sequence b holds, as far as slots reach.
__device__ __forceinline__ int32_t held_of(int32_t n, int64_t most) { return n < 0 ? 0 : n > most ? (int32_t)most : n; }
__device__ __forceinline__ int32_t held_tokens(const int32_t* lengths, int b, int64_t most) {
  return held_of(lengths[b], most);
}
__device__ __forceinline__ int32_t held_tokens_uniform(const int32_t* lengths, int b, int64_t most) {
  return held_of(((uniform_i32)(uintptr_t)lengths)[b], most);
}

// The page of a slot of sequence b, -1 if it is not there.
__device__ __forceinline__ int32_t page_of(const CacheView& c, int64_t b, int64_t slot) {
  const int32_t p = c.table[b * c.ldt + (slot >> c.log2_page)];
  return p >= 0 && p < c.pages ? p : -1;
}

// The same for a slot that the whole wave asks for.
__device__ __forceinline__ int32_t page_of_uniform(const CacheView& c, int64_t b, int32_t slot) {
  const int32_t p = ((uniform_i32)(uintptr_t)c.table)[b * c.ldt + (slot >> c.log2_page)];
  return p >= 0 && p < c.pages ? p : -1;
}

// Bytes from the start of k or v to the row of a head at a place of a page.
__device__ __forceinline__ int64_t row_offset(const CacheView& c, int32_t page, int32_t head, int64_t slot) {
  return page * c.page_stride + head * c.head_stride + (slot & ((1 << c.log2_page) - 1)) * c.token_stride;
}

// The same in the arrays of one number per row.
__device__ __forceinline__ int64_t row_index(const CacheView& c, int32_t page, int32_t head, int64_t slot) {
  return (((int64_t)page * c.kv_heads + head) << c.log2_page) + (slot & ((1 << c.log2_page) - 1));
}

// Sums of v over the lanes up to this one: within rows of 16 by shifts, then
// across rows.
template <int CTRL, int ROWS> __device__ __forceinline__ int lanes_before(int v) {
  return __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xF, true);
}
__device__ __forceinline__ int wave_scan(int v) {
  v += lanes_before<0x111, 0xF>(v);
  v += lanes_before<0x112, 0xF>(v);
  v += lanes_before<0x114, 0xF>(v);
  v += lanes_before<0x118, 0xF>(v);
  v += lanes_before<0x142, 0xA>(v);       // a row's last lane to the next row (rows 1 and 3)
  v += lanes_before<0x143, 0xC>(v);       // lane 31 to rows 2 and 3
  return v;
}

#endif

}  // namespace mosaic
