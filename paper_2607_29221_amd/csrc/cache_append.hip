// New tokens into the cache (mosaic_cache_append): rotary positions on several
// axes and the write of keys and values into their pages, in one pass over the
// fused q|k|v rows.
//
// A pair (x, y) at place p turns into (x c - y s, y c + x s), c and s from the
// caller's table. One workgroup takes one token: it gathers the token's 2P
// cosines and sines into LDS once and every head reads them from there, so a
// row of q|k|v is read once and every output written once, and the call is
// bound by that traffic: 4096 tokens of 64 + 2 * 8 heads of 128 floats in 61 us
// (5.5 TB/s). A single token takes 3.3 us and 48 take 3.7 us, the latency of
// launch, state, page and table; its row is asked for before these.
#include "cache.h"
#include "device_common.h"
#include "dispatch.h"

namespace mosaic {
namespace {

constexpr int kFewRows = 256;     // no more than one workgroup per compute unit
// Rows that the 32 MiB of second-level cache cannot hold pass by it (168 MB of
// q|k|v: 61 us, 69 us through it); fewer are left there for the attention that
// comes next.
constexpr int64_t kStreamBytes = (int64_t)32 << 20;

// How the elements of a pair lie. A thread works on V consecutive elements
// (16 bytes of the row).
enum RotaryMode {
  ROT_HALVES,         // j and P + j, P a multiple of V: a thread takes both chunks of a pair
  ROT_HALVES_RAGGED,  // j and P + j, any P: a thread takes one chunk and reads its partners one by one
  ROT_NEIGHBOURS      // 2j and 2j + 1 (and P = 0, nothing rotated): a chunk holds whole pairs
};

// The sequence that row t belongs to: the last b < batch with starts[b] <= t.
__device__ __forceinline__ int sequence_of(const int32_t* starts, int batch, int64_t t) {
  int lo = 0, hi = batch - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (starts[mid] <= t) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

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

__global__ __launch_bounds__(256) void cache_advance_kernel(AppendLaunch a) {
  const int b = blockIdx.x * 256 + threadIdx.x;
  if (b < a.c.batch) advance(a, b, fresh_tokens(a, b), (int64_t)a.c.max_blocks << a.c.log2_page);
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

// Where a chunk of a head goes: q_out, or the head's row of k or v.
template <int XT, int CT, bool STREAM, int V>
__device__ __forceinline__ void store_chunk(const AppendLaunch& a, char* q, int64_t kv_off, bool kept, int head,
                                            int e0, const float* y) {
  typedef typename FloatType<XT>::type X;
  typedef typename FloatType<CT>::type C;
  const int D = a.c.head_dim;
  if (head < a.heads) {
    Chunk<X, V> o;
#pragma unroll
    for (int i = 0; i < V; ++i) o.e[i] = (X)y[i];
    store_piece<STREAM>(q + ((int64_t)head * D + e0) * sizeof(X), o);
  } else if (kept) {
    const int h = head - a.heads;
    const bool value = h >= a.c.kv_heads;
    Chunk<C, V> o;
#pragma unroll
    for (int i = 0; i < V; ++i) o.e[i] = (C)y[i];
    char* base = (value ? a.c.v : a.c.k) + kv_off + (value ? h - a.c.kv_heads : h) * a.c.head_stride;
    store_piece<STREAM>(base + e0 * sizeof(C), o);
  }
}

// A thread's piece of the row: V elements of a head, and the V that they are
// paired with P further on (ROT_HALVES).
template <int XT, int MODE, bool STREAM> struct Unit {
  typedef typename FloatType<XT>::type X;
  static constexpr int V = 16 / sizeof(X);
  int head, e0;                                  // of the row; first element in the head
  bool turned, pair;                             // rotated head; with a partner chunk
  Chunk<X, V> a, b;

  __device__ __forceinline__ void load(const AppendLaunch& l, const char* x, int u) {
    const int D = l.c.head_dim, P = l.rot.pairs, chunks = D / V, pc = MODE == ROT_HALVES ? P / V : 0;
    const int turned_heads = l.heads + l.c.kv_heads, per_turned = chunks - pc, first = turned_heads * per_turned;
    turned = u < first;
    const int w = turned ? u : u - first, per = turned ? per_turned : chunks;
    const int q = w / per, r = w - q * per;
    head = q + (turned ? 0 : turned_heads);
    pair = turned && MODE == ROT_HALVES && r < pc;
    e0 = V * (MODE == ROT_HALVES && turned && r >= pc ? r + pc : r);
    const char* at = x + ((int64_t)head * D + e0) * sizeof(X);
    a = load_piece<STREAM, Chunk<X, V>>(at);
    if (pair) b = load_piece<STREAM, Chunk<X, V>>(at + P * sizeof(X));
  }
};

template <int XT, int CT, int MODE, bool STREAM>
__global__ __launch_bounds__(1024) void cache_append_kernel(AppendLaunch a) {
  typedef typename FloatType<XT>::type X;
  constexpr int V = 16 / sizeof(X);
  __shared__ float turn[256];                    // cosines of the P pairs, then sines
  const int64_t t = blockIdx.x;
  const int threads = blockDim.x, tid = threadIdx.x;
  const char* x = (const char*)a.x + t * a.ldx;
  char* q = (char*)a.q + t * a.ldq;
  const int P = a.rot.pairs, D = a.c.head_dim;
  const int units = (a.heads + a.c.kv_heads) * (D / V - (MODE == ROT_HALVES ? P / V : 0)) + a.c.kv_heads * (D / V);
  Unit<XT, MODE, STREAM> unit;
  if (tid < units) unit.load(a, x, tid);         // under way while the token's place is found

  const int b = a.starts == nullptr ? (int)t : sequence_of(a.starts, a.c.batch, t);
  const int32_t i = a.starts == nullptr ? 0 : (int32_t)(t - a.starts[b]);
  const int64_t slots = (int64_t)a.c.max_blocks << a.c.log2_page;
  const int64_t slot = (int64_t)__builtin_amdgcn_readfirstlane(held_tokens(a.state, b, slots)) + i;
  const int32_t number = (int32_t)((uint32_t)a.state[a.c.batch + b] + (uint32_t)i);
  const int32_t page = slot >= 0 && slot < slots ? page_of_uniform(a.c, b, (int32_t)slot) : -1;
  const bool kept = page >= 0;
  const int64_t kv_off = kept ? row_offset(a.c, page, 0, slot) : 0;

  for (int j = tid; j < P; j += threads) {
    const int axis = (j >= a.rot.ends[0]) + (j >= a.rot.ends[1]) + (j >= a.rot.ends[2]);
    int64_t p = a.rot.positions != nullptr ? a.rot.positions[axis * a.rot.ldp + t] : number;
    p = p < 0 ? 0 : p >= a.rot.rows ? a.rot.rows - 1 : p;
    const float* r = a.rot.table + p * 2 * P;
    turn[j] = r[j];
    turn[P + j] = r[P + j];
  }
  __syncthreads();                               // also: every thread has read the state
  if (a.starts == nullptr) {
    if (tid == 0) advance(a, b, 1, slots);       // nobody else reads this sequence's
  } else if (t == 0 && a.new_state != a.state) {
    for (int s = tid; s < a.c.batch; s += threads) advance(a, s, fresh_tokens(a, s), slots);
  }
  for (int h = tid; kept && h < a.c.kv_heads; h += threads) {
    const int64_t r = row_index(a.c, page, h, slot);
    if (a.c.weights != nullptr) a.c.weights[r] = 0.0f;
    if (a.c.order != nullptr) a.c.order[r] = number;
  }

  for (int u = tid; u < units; u += threads) {
    if (u != tid) unit.load(a, x, u);
    const int head = unit.head, e0 = unit.e0;
    const bool turned = unit.turned;
    float v[V], y[V];
#pragma unroll
    for (int k = 0; k < V; ++k) v[k] = y[k] = (float)unit.a.e[k];
    if (MODE == ROT_HALVES && unit.pair) {
      float z[V];
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const float o = (float)unit.b.e[k], cs = turn[e0 + k], sn = turn[P + e0 + k];
        y[k] = v[k] * cs - o * sn;
        z[k] = o * cs + v[k] * sn;
      }
      store_chunk<XT, CT, STREAM, V>(a, q, kv_off, kept, head, e0 + P, z);
    } else if (turned && MODE == ROT_HALVES_RAGGED) {
      const X* xh = (const X*)x + (int64_t)head * D;
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const int e = e0 + k;
        if (e < 2 * P) {
          const int j = e < P ? e : e - P;
          const float o = (float)xh[e < P ? e + P : e - P];
          y[k] = e < P ? v[k] * turn[j] - o * turn[P + j] : v[k] * turn[j] + o * turn[P + j];
        }
      }
    } else if (turned && MODE == ROT_NEIGHBOURS) {
#pragma unroll
      for (int k = 0; k < V; k += 2) {
        const int j = (e0 + k) / 2;
        if (j < P) {
          y[k] = v[k] * turn[j] - v[k + 1] * turn[P + j];
          y[k + 1] = v[k + 1] * turn[j] + v[k] * turn[P + j];
        }
      }
    }
    store_chunk<XT, CT, STREAM, V>(a, q, kv_off, kept, head, e0, y);
  }
}

template <int XT, int CT, bool STREAM>
void launch_mode(const AppendLaunch& a, hipStream_t s) {
  constexpr int V = XT == MOSAIC_F32 ? 4 : 8;
  // few tokens: a thread per piece of a row, so that all of it is asked for at once
  const dim3 grid((unsigned)a.rows), block(a.rows <= kFewRows ? 1024 : 256);
  if (a.rot.pairs == 0 || a.rot.interleaved) cache_append_kernel<XT, CT, ROT_NEIGHBOURS, STREAM><<<grid, block, 0, s>>>(a);
  else if (a.rot.pairs % V == 0) cache_append_kernel<XT, CT, ROT_HALVES, STREAM><<<grid, block, 0, s>>>(a);
  else cache_append_kernel<XT, CT, ROT_HALVES_RAGGED, STREAM><<<grid, block, 0, s>>>(a);
}

template <int XT, int CT>
void launch_types(const AppendLaunch& a, hipStream_t s) {
  const int64_t row = (a.heads + 2 * (int64_t)a.c.kv_heads) * a.c.head_dim * (XT == MOSAIC_F32 ? 4 : 2);
  if (a.rows * row >= kStreamBytes) launch_mode<XT, CT, true>(a, s);
  else launch_mode<XT, CT, false>(a, s);
}

}  // namespace

hipError_t launch_cache_append(const AppendLaunch& a, hipStream_t s) {
  if (a.rows > 0) {
    if (a.x_dtype == MOSAIC_F32 && a.c.dtype == MOSAIC_F32) launch_types<MOSAIC_F32, MOSAIC_F32>(a, s);
    else if (a.x_dtype == MOSAIC_F32 && a.c.dtype == MOSAIC_BF16) launch_types<MOSAIC_F32, MOSAIC_BF16>(a, s);
    else if (a.x_dtype == MOSAIC_F32) launch_types<MOSAIC_F32, MOSAIC_F16>(a, s);
    else if (a.c.dtype == MOSAIC_BF16) launch_types<MOSAIC_BF16, MOSAIC_BF16>(a, s);
    else launch_types<MOSAIC_F16, MOSAIC_F16>(a, s);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  // the workgroups above read the state of a sequence in any order, so one
  // that is written in place waits for the last of them
  if (a.starts != nullptr && (a.rows == 0 || a.new_state == a.state)) {
    cache_advance_kernel<<<(a.c.batch + 255) / 256, 256, 0, s>>>(a);
    return hipGetLastError();
  }
  return hipSuccess;
}

}  // namespace mosaic
