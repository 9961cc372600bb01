// Cached tokens as rows (mosaic_cache_read).
//
// A thread takes 8 elements of a key and the same 8 of the value: 4 bits are a
// dword of codes and a scale byte of each. A workgroup takes one token. Bound by the
// traffic of rows read and written.
#include "cache.h"
#include "device_common.h"
#include "e2m1.h"

namespace mosaic {
namespace {

template <class T> struct alignas(16) Piece { T e[16 / sizeof(T)]; };

// 8 elements of a cached row as float32.
template <int CT> struct Held {
  typedef typename FloatType<CT>::type C;
  static constexpr int kLoads = sizeof(C) / 2;
  Piece<C> c[kLoads];
  __device__ __forceinline__ void load(const char* row, int, int chunk) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) c[i] = *(const Piece<C>*)(row + 8 * chunk * (int)sizeof(C) + 16 * i);
  }
  __device__ __forceinline__ void get(float* x) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (float)c[i / (8 / kLoads)].e[i % (8 / kLoads)];
  }
};
template <> struct Held<MOSAIC_E2M1> {
  uint32_t codes, scale;
  __device__ __forceinline__ void load(const char* row, int D, int chunk) {
    codes = *(const uint32_t*)(row + 4 * chunk);
    scale = *(const uint8_t*)(row + D / 2 + chunk);
  }
  __device__ __forceinline__ void get(float* x) const {
    uint32_t pair[4];
    e2m1_decode(codes, e2m1_scale(scale), pair);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(pair[i] << 16);
      x[2 * i + 1] = __uint_as_float(pair[i] & 0xFFFF0000u);
    }
  }
};

template <int CT, int OT>
__global__ __launch_bounds__(256) void cache_read_kernel(ReadLaunch a) {
  typedef typename FloatType<OT>::type O;
  constexpr int kStores = sizeof(O) / 2, PER = 16 / (int)sizeof(O);
  const int D = a.c.head_dim, chunks = D / 8, units = a.c.kv_heads * chunks;
  const int64_t slots = (int64_t)a.c.max_blocks << a.c.log2_page;
  for (int64_t t = blockIdx.x; t < a.rows; t += gridDim.x) {
    const int b = a.starts == nullptr ? (int)t : sequence_of(a.starts, a.c.batch, t);
    const int64_t slot = (a.first != nullptr ? (int64_t)a.first[b] : 0) + (a.starts != nullptr ? t - a.starts[b] : 0);
    const int64_t held = held_tokens(a.lengths, b, slots);
    const int32_t page = slot >= 0 && slot < held ? page_of(a.c, b, slot) : -1;
    const int64_t off = page >= 0 ? row_offset(a.c, page, 0, slot) : 0;
    for (int u = threadIdx.x; u < units; u += 256) {
      const int h = u / chunks, chunk = u - h * chunks;
      float k[8] = {}, v[8] = {};
      if (page >= 0) {
        Held<CT> key, value;
        key.load(a.c.k + off + h * a.c.head_stride, D, chunk);
        value.load(a.c.v + off + h * a.c.head_stride, D, chunk);
        key.get(k);
        value.get(v);
      }
      Piece<O> ko[kStores], vo[kStores];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        ko[i / PER].e[i % PER] = (O)k[i];
        vo[i / PER].e[i % PER] = (O)v[i];
      }
#pragma unroll
      for (int i = 0; i < kStores; ++i) {
        *(Piece<O>*)((char*)a.k + t * a.ldk + 8 * u * (int64_t)sizeof(O) + 16 * i) = ko[i];
        *(Piece<O>*)((char*)a.v + t * a.ldv + 8 * u * (int64_t)sizeof(O) + 16 * i) = vo[i];
      }
    }
  }
}

template <int CT, int OT>
void launch_types(const ReadLaunch& a, hipStream_t s) {
  constexpr int64_t kMost = 1 << 22;               // workgroups; a launch takes less than 2^32 threads
  cache_read_kernel<CT, OT><<<(unsigned)(a.rows < kMost ? a.rows : kMost), 256, 0, s>>>(a);
}

}  // namespace

hipError_t launch_cache_read(const ReadLaunch& a, hipStream_t s) {
  if (a.c.dtype == MOSAIC_E2M1) {
    if (a.out_dtype == MOSAIC_F32) launch_types<MOSAIC_E2M1, MOSAIC_F32>(a, s);
    else if (a.out_dtype == MOSAIC_BF16) launch_types<MOSAIC_E2M1, MOSAIC_BF16>(a, s);
    else launch_types<MOSAIC_E2M1, MOSAIC_F16>(a, s);
  } else if (a.c.dtype == MOSAIC_F32) {
    launch_types<MOSAIC_F32, MOSAIC_F32>(a, s);
  } else if (a.c.dtype == MOSAIC_BF16) {
    if (a.out_dtype == MOSAIC_F32) launch_types<MOSAIC_BF16, MOSAIC_F32>(a, s);
    else launch_types<MOSAIC_BF16, MOSAIC_BF16>(a, s);
  } else {
    if (a.out_dtype == MOSAIC_F32) launch_types<MOSAIC_F16, MOSAIC_F32>(a, s);
    else launch_types<MOSAIC_F16, MOSAIC_F16>(a, s);
  }
  return hipGetLastError();
}

}  // namespace mosaic
