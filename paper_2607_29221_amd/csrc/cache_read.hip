// Cached tokens as rows (mosaic_cache_read).
//
// A thread writes 16 bytes of a row of k_out and the same of v_out: 4 or 8
// elements, of 4 bits a half or a whole dword of codes and a scale byte; groups of
// threads, a power of two each, take a row at a time. A workgroup takes several
// neighbouring rows and looks all their places up at once, a lane each: the chain
// of starts, lengths, table and rows (4 us) is then paid once for them. Bound by the
// traffic of rows read and written (16384 tokens of 8 x 128 to float32: 155 MB in
// 26 us; 184000 of 1 x 64 to bf16: 62 MB in 13 us, 43 us with a workgroup per row).
#include "cache.h"
#include "device_common.h"
#include "e2m1.h"

namespace mosaic {
namespace {

constexpr int kThreads = 256;
// Rows of a group of threads at most (4096 x 4 tokens of 8 x 128 to float32: 26.4
// us, 27.6 with 16), and groups of a workgroup.
constexpr int kMostRows = 4, kMostGroups = 64;
// Rows that the 32 MiB of second-level cache cannot hold pass by it.
constexpr int64_t kStreamBytes = (int64_t)32 << 20;

// N elements of a cached row, from element e on.
template <int CT, int N> struct Held {
  typedef typename FloatType<CT>::type C;
  struct alignas(N * sizeof(C) < 16 ? N * sizeof(C) : 16) Piece { C e[N]; } c;
  __device__ __forceinline__ void load(const char* row, int, int e) { c = *(const Piece*)(row + e * (int)sizeof(C)); }
  __device__ __forceinline__ void get(float* x) const {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = (float)c.e[i];
  }
};
template <int N> struct Held<MOSAIC_E2M1, N> {
  uint32_t codes, scale;
  __device__ __forceinline__ void load(const char* row, int D, int e) {
    codes = N == 8 ? *(const uint32_t*)(row + e / 2) : *(const uint16_t*)(row + e / 2);
    scale = *(const uint8_t*)(row + D / 2 + e / 8);
  }
  __device__ __forceinline__ void get(float* x) const {
    uint32_t pair[4];
    e2m1_decode(codes, e2m1_scale(scale), pair);
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
      x[2 * i] = __uint_as_float(pair[i] << 16);
      x[2 * i + 1] = __uint_as_float(pair[i] & 0xFFFF0000u);
    }
  }
};

template <int CT, int OT, bool STREAM>
__global__ __launch_bounds__(kThreads) void cache_read_kernel(ReadLaunch a, int rows_of, int log2_group) {
  typedef typename FloatType<OT>::type O;
  constexpr int N = 16 / (int)sizeof(O);
  struct alignas(16) Out { O e[N]; };
  __shared__ int64_t place[kMostRows * kMostGroups];   // from the start of k or v, -1 without a token
  const int D = a.c.head_dim, of_head = D / N, units = a.c.kv_heads * of_head;
  const int tid = threadIdx.x, group = 1 << log2_group, groups = kThreads >> log2_group;
  const int64_t t0 = (int64_t)blockIdx.x * rows_of;
  const int count = (int)(a.rows - t0 < rows_of ? a.rows - t0 : rows_of);
  if (tid < count) {
    const int64_t t = t0 + tid;
    const int b = a.starts == nullptr ? (int)t : sequence_of(a.starts, a.c.batch, t);
    const int64_t slot = (a.first != nullptr ? (int64_t)a.first[b] : 0) + (a.starts != nullptr ? t - a.starts[b] : 0);
    const int64_t held = held_tokens(a.lengths, b, (int64_t)a.c.max_blocks << a.c.log2_page);
    const int32_t page = slot >= 0 && slot < held ? page_of(a.c, b, slot) : -1;
    place[tid] = page >= 0 ? row_offset(a.c, page, 0, slot) : -1;
  }
  __syncthreads();
  for (int u = tid & (group - 1); u < units; u += group) {
    const int h = u / of_head, e = (u - h * of_head) * N;
    const int64_t head = h * a.c.head_stride;
    char *ko = (char*)a.k + t0 * a.ldk + 16 * (int64_t)u, *vo = (char*)a.v + t0 * a.ldv + 16 * (int64_t)u;
#pragma unroll 4
    for (int r = tid >> log2_group; r < count; r += groups) {
      const int64_t at = place[r];
      float k[N] = {}, v[N] = {};
      if (at >= 0) {
        Held<CT, N> key, value;
        key.load(a.c.k + at + head, D, e);
        value.load(a.c.v + at + head, D, e);
        key.get(k);
        value.get(v);
      }
      Out x, y;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        x.e[i] = (O)k[i];
        y.e[i] = (O)v[i];
      }
      if constexpr (STREAM) {
        __builtin_nontemporal_store(__builtin_bit_cast(u32x4, x), (u32x4*)(ko + r * a.ldk));
        __builtin_nontemporal_store(__builtin_bit_cast(u32x4, y), (u32x4*)(vo + r * a.ldv));
      } else {
        *(Out*)(ko + r * a.ldk) = x;
        *(Out*)(vo + r * a.ldv) = y;
      }
    }
  }
}

template <int CT, int OT>
void launch_types(const ReadLaunch& a, hipStream_t s) {
  const int64_t row = (int64_t)a.c.kv_heads * a.c.head_dim * (OT == MOSAIC_F32 ? 4 : 2);   // of one of the outputs
  int log2_group = 2;                              // 4 to 256 threads
  while (log2_group < 8 && 16 << log2_group < row) ++log2_group;
  // as many rows for a group as leave 1024 workgroups
  const int groups = kThreads >> log2_group;
  const int64_t share = a.rows / (1024 * groups);
  const int rows_of = groups * (share < 1 ? 1 : share > kMostRows ? kMostRows : (int)share);
  const unsigned grid = (unsigned)((a.rows + rows_of - 1) / rows_of);
  if (2 * a.rows * row >= kStreamBytes) cache_read_kernel<CT, OT, true><<<grid, kThreads, 0, s>>>(a, rows_of, log2_group);
  else cache_read_kernel<CT, OT, false><<<grid, kThreads, 0, s>>>(a, rows_of, log2_group);
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
