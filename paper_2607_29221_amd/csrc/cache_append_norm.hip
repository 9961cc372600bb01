// New tokens into the cache with norms of queries and keys
// (mosaic_cache_append_norm), and into a cache in 4 bits with or without them.
//
// Of a head x, with f = 1 / sqrt(mean x^2 + eps): y = (x f) w, then the pairs of
// y are turned as in cache_append.hip. A lane takes 8 consecutive elements, a
// head 1 to 32 neighbouring lanes (a power of two): the mean is a sum over these, the
// 8 elements are what shares a scale in 4 bits (a dword of codes and a byte,
// found by the lane alone), and the partner of an element P further on comes
// from the other lane through LDS, normalised.
//
// The sum of squares is float64 and what follows is rounded step by step, not
// fused: a key near the border of two codes then takes the one that the
// formulas give, however they are computed.
//
// Bound by the traffic of the q|k|v rows.
#include "cache_append.h"
#include "e2m1.h"

namespace mosaic {
namespace {

// Who a pair's elements are, of a lane's 8: both its own; or j and P + j, with
// whole chunks of 8 paired (P a multiple of 8) or not.
enum PairMode { PAIRS_OWN, PAIRS_CHUNKS, PAIRS_ANY };

// 8 elements of a row.
template <int XT, bool STREAM> struct Eight {
  typedef typename FloatType<XT>::type X;
  static constexpr int kLoads = sizeof(X) / 2;    // of 16 bytes
  Chunk<X, 16 / sizeof(X)> c[kLoads];
  __device__ __forceinline__ void load(const char* p) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) c[i] = load_piece<STREAM, Chunk<X, 16 / sizeof(X)>>(p + 16 * i);
  }
  __device__ __forceinline__ void store(char* p) const {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) store_piece<STREAM>(p + 16 * i, c[i]);
  }
  __device__ __forceinline__ void get(float* x) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (float)c[i / (8 / kLoads)].e[i % (8 / kLoads)];
  }
  __device__ __forceinline__ void set(const float* x) {
#pragma unroll
    for (int i = 0; i < 8; ++i) c[i / (8 / kLoads)].e[i % (8 / kLoads)] = (X)x[i];
  }
};

__device__ __forceinline__ double lanes_sum(double v, int lanes) {
  for (int off = lanes >> 1; off > 0; off >>= 1) v += __shfl_xor(v, off);
  return v;
}

// A workgroup takes one token; lanes: 2^log2_lanes of a head.
template <int XT, int CT, int MODE, bool STREAM, int THREADS>
__global__ __launch_bounds__(THREADS) void cache_append_norm_kernel(AppendLaunch a, int log2_lanes) {
#pragma clang fp contract(off)
  typedef typename FloatType<XT>::type X;
  __shared__ float turn[256];                    // cosines of the P pairs, then sines
  __shared__ f32x4 shared[MODE == PAIRS_OWN ? 1 : THREADS / 64][2][64];
  const int64_t t = blockIdx.x;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int P = a.rot.pairs, D = a.c.head_dim, chunks = D / 8;
  const int lanes = 1 << log2_lanes, chunk = lane & (lanes - 1), slot0 = lane - chunk;
  const int turned_heads = a.heads + a.c.kv_heads, all_heads = turned_heads + a.c.kv_heads;
  const bool own = chunk < chunks;
  const char* x = (const char*)a.x + t * a.ldx;
  char* q = (char*)a.q + t * a.ldq;
  const int head_step = THREADS >> log2_lanes;
  int head = tid >> log2_lanes;
  Eight<XT, STREAM> next;
  auto load = [&](int h) {
    if (own && h < all_heads) next.load(x + ((int64_t)h * D + 8 * chunk) * sizeof(X));
  };
  load(head);                                    // under way while the token's place is found

  const int b = a.starts == nullptr ? (int)t : sequence_of(a.starts, a.c.batch, t);
  const int32_t i = a.starts == nullptr ? 0 : (int32_t)(t - a.starts[b]);
  const int64_t slots = (int64_t)a.c.max_blocks << a.c.log2_page;
  const int64_t slot = (int64_t)__builtin_amdgcn_readfirstlane(held_tokens(a.state, b, slots)) + i;
  const int32_t number = (int32_t)((uint32_t)a.state[a.c.batch + b] + (uint32_t)i);
  const int32_t page = slot >= 0 && slot < slots ? page_of_uniform(a.c, b, (int32_t)slot) : -1;
  const bool kept = page >= 0;
  const int64_t kv_off = kept ? row_offset(a.c, page, 0, slot) : 0;

  for (int j = tid; j < P; j += THREADS) {
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
    for (int s = tid; s < a.c.batch; s += THREADS) advance(a, s, fresh_tokens(a, s), slots);
  }
  for (int h = tid; kept && h < a.c.kv_heads; h += THREADS) {
    const int64_t r = row_index(a.c, page, h, slot);
    if (a.c.weights != nullptr) a.c.weights[r] = 0.0f;
    if (a.c.order != nullptr) a.c.order[r] = number;
  }

  // every lane of a wave goes round as often (lanes of a head work together)
  for (int first = (wave << 6) >> log2_lanes; first < all_heads; first += head_step, head += head_step) {
    float v[8] = {};
    if (own && head < all_heads) next.get(v);
    load(head + head_step);
    if (a.norm.q_weight != nullptr) {
      double square = 0.0;
#pragma unroll
      for (int k = 0; k < 8; ++k) square += (double)v[k] * (double)v[k];
      const float f = (float)(1.0 / sqrt(lanes_sum(square, lanes) / D + a.norm.eps));
      if (own && head < turned_heads) {
        const float* w = (head < a.heads ? a.norm.q_weight : a.norm.k_weight) + 8 * chunk;
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = v[k] * f * w[k];
      }
    }
    if (MODE == PAIRS_OWN) {
      if (head < turned_heads) {
#pragma unroll
        for (int k = 0; k < 8; k += 2) {
          const int j = 4 * chunk + k / 2;
          if (j < P) {
            const float x0 = v[k], x1 = v[k + 1];
            v[k] = x0 * turn[j] - x1 * turn[P + j];
            v[k + 1] = x1 * turn[j] + x0 * turn[P + j];
          }
        }
      }
    } else {
      f32x4(*mine)[64] = shared[wave];
      mine[0][lane] = f32x4{v[0], v[1], v[2], v[3]};
      mine[1][lane] = f32x4{v[4], v[5], v[6], v[7]};
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
      __builtin_amdgcn_wave_barrier();
      if (own && head < turned_heads && 8 * chunk < 2 * P) {
        if (MODE == PAIRS_CHUNKS) {
          const bool low = 8 * chunk < P;
          const int other = lane + (low ? P / 8 : -(P / 8)), j = 8 * chunk - (low ? 0 : P);
          const f32x4 o[2] = {mine[0][other], mine[1][other]};
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const float z = o[k / 4][k % 4], cs = turn[j + k], sn = turn[P + j + k];
            v[k] = low ? v[k] * cs - z * sn : v[k] * cs + z * sn;
          }
        } else {
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const int e = 8 * chunk + k;
            if (e < 2 * P) {
              const bool low = e < P;
              const int j = low ? e : e - P, at = low ? e + P : e - P;
              const float z = mine[at % 8 / 4][slot0 + at / 8][at % 4], cs = turn[j], sn = turn[P + j];
              v[k] = low ? v[k] * cs - z * sn : v[k] * cs + z * sn;
            }
          }
        }
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
      __builtin_amdgcn_wave_barrier();           // read before the next heads are written
    }
    if (!own || head >= all_heads) continue;
    if (head < a.heads) {
      Eight<XT, STREAM> out;
      out.set(v);
      out.store(q + ((int64_t)head * D + 8 * chunk) * sizeof(X));
    } else if (kept) {
      const bool value = head >= turned_heads;
      char* row = (value ? a.c.v : a.c.k) + kv_off + (value ? head - turned_heads : head - a.heads) * a.c.head_stride;
      if constexpr (CT == MOSAIC_E2M1) {
        uint32_t code;
        const uint32_t scale = e2m1_encode(v, &code);
        *(uint32_t*)(row + 4 * chunk) = code;
        *(uint8_t*)(row + D / 2 + chunk) = (uint8_t)scale;
      } else {
        Eight<CT, STREAM> out;
        out.set(v);
        out.store(row + 8 * chunk * (int)sizeof(typename FloatType<CT>::type));
      }
    }
  }
}

template <int XT, int CT, bool STREAM, int THREADS>
void launch_pairs(const AppendLaunch& a, int log2_lanes, hipStream_t s) {
  const dim3 grid((unsigned)a.rows);
  if (a.rot.pairs == 0 || a.rot.interleaved)
    cache_append_norm_kernel<XT, CT, PAIRS_OWN, STREAM, THREADS><<<grid, THREADS, 0, s>>>(a, log2_lanes);
  else if (a.rot.pairs % 8 == 0)
    cache_append_norm_kernel<XT, CT, PAIRS_CHUNKS, STREAM, THREADS><<<grid, THREADS, 0, s>>>(a, log2_lanes);
  else
    cache_append_norm_kernel<XT, CT, PAIRS_ANY, STREAM, THREADS><<<grid, THREADS, 0, s>>>(a, log2_lanes);
}

template <int XT, int CT>
void launch_types(const AppendLaunch& a, hipStream_t s) {
  int log2_lanes = 0;
  while (8 << log2_lanes < a.c.head_dim) ++log2_lanes;
  const int64_t row = (a.heads + 2 * (int64_t)a.c.kv_heads) * a.c.head_dim * (XT == MOSAIC_F32 ? 4 : 2);
  if (a.rows * row >= kStreamBytes) launch_pairs<XT, CT, true, 256>(a, log2_lanes, s);
  else if (a.rows > kFewRows) launch_pairs<XT, CT, false, 256>(a, log2_lanes, s);
  else launch_pairs<XT, CT, false, 1024>(a, log2_lanes, s);
}

}  // namespace

void launch_cache_append_norm(const AppendLaunch& a, hipStream_t s) {
  if (a.c.dtype == MOSAIC_E2M1) {
    if (a.x_dtype == MOSAIC_F32) launch_types<MOSAIC_F32, MOSAIC_E2M1>(a, s);
    else if (a.x_dtype == MOSAIC_BF16) launch_types<MOSAIC_BF16, MOSAIC_E2M1>(a, s);
    else launch_types<MOSAIC_F16, MOSAIC_E2M1>(a, s);
  } else if (a.x_dtype == MOSAIC_F32 && a.c.dtype == MOSAIC_F32) {
    launch_types<MOSAIC_F32, MOSAIC_F32>(a, s);
  } else if (a.x_dtype == MOSAIC_F32 && a.c.dtype == MOSAIC_BF16) {
    launch_types<MOSAIC_F32, MOSAIC_BF16>(a, s);
  } else if (a.x_dtype == MOSAIC_F32) {
    launch_types<MOSAIC_F32, MOSAIC_F16>(a, s);
  } else if (a.c.dtype == MOSAIC_BF16) {
    launch_types<MOSAIC_BF16, MOSAIC_BF16>(a, s);
  } else {
    launch_types<MOSAIC_F16, MOSAIC_F16>(a, s);
  }
}

}  // namespace mosaic
