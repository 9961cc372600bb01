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
// formulas give, however they are computed (one head in 2^26 has its factor so near
// the border of two float32 numbers that the float64 sum's own rounding decides).
//
// Bound by the traffic of the q|k|v rows: 4096 tokens of 64 + 2 * 8 heads of 128 in
// 35 to 38 us as bf16 (168 MB, 4.5 to 4.8 TB/s), in 63 to 70 us from float32 to 4
// bits (309 MB, 4.4 to 4.9 TB/s). A single token takes 4.1 us, the latency of state,
// page and table, one after the other, and of the root. Cosines, sines and weights
// are read from LDS for every head: held in registers instead, their way there cost
// more than a token's five rounds of heads got back (norms in bf16 55 us).
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

// The sum over the neighbouring lanes of a head, the same bits in all of them:
// within 16 lanes by data-parallel moves to the other one of a pair, the other
// pair, the other four and the other eight.
template <int CTRL> __device__ __forceinline__ double other_lane(double v) {
  const uint64_t w = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)w, CTRL, 0xF, 0xF, true);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(w >> 32), CTRL, 0xF, 0xF, true);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ double lanes_sum(double v, int log2_lanes) {
  if (log2_lanes > 0) v += other_lane<0xB1>(v);
  if (log2_lanes > 1) v += other_lane<0x4E>(v);
  if (log2_lanes > 2) v += other_lane<0x141>(v);
  if (log2_lanes > 3) v += other_lane<0x140>(v);
  if (log2_lanes > 4) v += __shfl_xor(v, 16);
  return v;
}

// 1 / sqrt(v), good to 2^-50 at least, rounded to float32: the machine's own
// estimate and two steps of Newton's method, which each square its error.
__device__ __forceinline__ float inverse_root(double v) {
  double y = __builtin_amdgcn_rsq(v);
  if (y == 0.0 || y == INFINITY) return (float)y;   // of infinity and of 0
#pragma unroll
  for (int i = 0; i < 2; ++i) y = y + 0.5 * y * __builtin_fma(-v * y, y, 1.0);
  return (float)y;
}

// A workgroup takes rows_of tokens, one after the other (one where there are few;
// several share the latency of finding their places); lanes: 2^log2_lanes of a head.
constexpr int kMostRows = 4;
template <int XT, int CT, int MODE, bool STREAM, int THREADS>
__global__ __launch_bounds__(THREADS) void cache_append_norm_kernel(AppendLaunch a, int log2_lanes, int rows_of) {
#pragma clang fp contract(off)
  typedef typename FloatType<XT>::type X;
  constexpr int kRows = THREADS == 1024 ? 1 : kMostRows;
  struct Place {
    int64_t kv_off;                              // of the token's rows, -1: it is not kept
    int32_t number;
  };
  __shared__ f32x4 turn[kRows][2][32];           // cosines of a token's pairs, sines
  __shared__ f32x4 weight[2][64];                // of queries and keys
  __shared__ f32x4 shared[MODE == PAIRS_OWN ? 1 : THREADS / 64][2][64];
  __shared__ Place place[kRows];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t t0 = (int64_t)blockIdx.x * rows_of;
  const int count = kRows == 1 ? 1 : (int)(a.rows - t0 < rows_of ? a.rows - t0 : rows_of);
  const int P = a.rot.pairs, D = a.c.head_dim, chunks = D / 8;
  const int lanes = 1 << log2_lanes, chunk = lane & (lanes - 1), slot0 = lane - chunk;
  const int turned_heads = a.heads + a.c.kv_heads, all_heads = turned_heads + a.c.kv_heads;
  const bool own = chunk < chunks, norm = a.norm.q_weight != nullptr;
  const int head_step = THREADS >> log2_lanes, rounds = (all_heads + head_step - 1) / head_step;
  Eight<XT, STREAM> next;
  auto load = [&](int r, int h) {
    if (own && h < all_heads) next.load((const char*)a.x + (t0 + r) * a.ldx + ((int64_t)h * D + 8 * chunk) * sizeof(X));
  };
  load(0, tid >> log2_lanes);                    // under way while the tokens' places are found
  if (norm && tid < 2 * D) {
    const int j = tid < D ? tid : tid - D;
    ((float*)weight[tid < D ? 0 : 1])[j] = (tid < D ? a.norm.q_weight : a.norm.k_weight)[j];
  }
  if (THREADS < 512 && norm && 2 * D > THREADS && tid + THREADS < 2 * D) {
    const int j = tid + THREADS, i = j < D ? j : j - D;
    ((float*)weight[j < D ? 0 : 1])[i] = (j < D ? a.norm.q_weight : a.norm.k_weight)[i];
  }

  const int64_t slots = (int64_t)a.c.max_blocks << a.c.log2_page;
  auto place_of = [&](int64_t t, int32_t* page, int64_t* slot) {
    const int b = a.starts == nullptr ? (int)t : sequence_of(a.starts, a.c.batch, t);
    const int32_t i = a.starts == nullptr ? 0 : (int32_t)(t - a.starts[b]);
    *slot = (int64_t)held_tokens(a.state, b, slots) + i;
    *page = *slot >= 0 && *slot < slots ? page_of(a.c, b, *slot) : -1;
    return Place{*page >= 0 ? row_offset(a.c, *page, 0, *slot) : -1, (int32_t)((uint32_t)a.state[a.c.batch + b] + (uint32_t)i)};
  };
  auto number_rows = [&](const Place& at, int32_t page, int64_t slot, int h0, int step) {
    if (at.kv_off < 0) return;
    for (int h = h0; h < a.c.kv_heads; h += step) {
      const int64_t r = row_index(a.c, page, h, slot);
      if (a.c.weights != nullptr) a.c.weights[r] = 0.0f;
      if (a.c.order != nullptr) a.c.order[r] = at.number;
    }
  };
  Place at;
  if (kRows == 1) {
    int32_t page;
    int64_t slot;
    at = place_of(t0, &page, &slot);             // by every thread: the same
    number_rows(at, page, slot, tid, THREADS);
  } else {
    // 32 lanes write the numbers of a token's rows
    const int r = tid >> 5;
    if (r < count) {
      int32_t page;
      int64_t slot;
      at = place_of(t0 + r, &page, &slot);
      number_rows(at, page, slot, tid & 31, 32);
      if ((tid & 31) == 0) place[r] = at;
    }
    __syncthreads();
  }
  for (int w = tid; w < count * P; w += THREADS) {
    const int r = kRows == 1 ? 0 : w / P, j = w - r * P;
    const int axis = (j >= a.rot.ends[0]) + (j >= a.rot.ends[1]) + (j >= a.rot.ends[2]);
    int64_t p = a.rot.positions != nullptr ? a.rot.positions[axis * a.rot.ldp + t0 + r] : kRows == 1 ? at.number : place[r].number;
    p = p < 0 ? 0 : p >= a.rot.rows ? a.rot.rows - 1 : p;
    const float* row = a.rot.table + p * 2 * P;
    ((float*)turn[r][0])[j] = row[j];
    ((float*)turn[r][1])[j] = row[P + j];
  }
  __syncthreads();                               // also: every thread has read the state
  if (a.starts == nullptr) {
    if (tid < count) advance(a, (int)(t0 + tid), 1, slots);   // nobody else reads this sequence's
  } else if (t0 == 0 && a.new_state != a.state) {
    for (int s = tid; s < a.c.batch; s += THREADS) advance(a, s, fresh_tokens(a, s), slots);
  }

  const double per_element = 1.0 / D;
  // every lane of a wave goes round as often (lanes of a head work together)
  for (int k0 = 0, r = 0, round = 0; k0 < count * rounds; ++k0) {
    const int head = (tid >> log2_lanes) + round * head_step;
    float v[8] = {};
    if (own && head < all_heads) next.get(v);
    const int now = r;
    if (++round == rounds) {
      round = 0;
      ++r;
    }
    if (r < count) load(r, (tid >> log2_lanes) + round * head_step);
    if (((wave << 6) >> log2_lanes) + (head - (tid >> log2_lanes)) >= all_heads) continue;   // the whole wave
    if (norm) {
      double square = 0.0;
#pragma unroll
      for (int k = 0; k < 8; ++k) square += (double)v[k] * (double)v[k];
      const float f = inverse_root(lanes_sum(square, log2_lanes) * per_element + a.norm.eps);
      if (own && head < turned_heads) {
        const f32x4* w = &weight[head < a.heads ? 0 : 1][2 * chunk];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = v[k] * f * w[k / 4][k % 4];
      }
    }
    const f32x4 *cosine = turn[now][0], *sine = turn[now][1];
    if (MODE == PAIRS_OWN) {
      if (own && head < turned_heads) {
        const f32x4 cs = cosine[chunk], sn = sine[chunk];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          if (4 * chunk + k < P) {
            const float x0 = v[2 * k], x1 = v[2 * k + 1];
            v[2 * k] = x0 * cs[k] - x1 * sn[k];
            v[2 * k + 1] = x1 * cs[k] + x0 * sn[k];
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
          const int other = lane + (low ? P / 8 : -(P / 8)), j = (low ? 8 * chunk : 8 * chunk - P) / 4;
          const f32x4 o[2] = {mine[0][other], mine[1][other]}, cs[2] = {cosine[j], cosine[j + 1]}, sn[2] = {sine[j], sine[j + 1]};
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const float z = o[k / 4][k % 4] * sn[k / 4][k % 4];
            v[k] = v[k] * cs[k / 4][k % 4] + (low ? -z : z);
          }
        } else {
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const int e = 8 * chunk + k;
            if (e < 2 * P) {
              const bool low = e < P;
              const int j = low ? e : e - P, from = low ? e + P : e - P;
              const float z = mine[from % 8 / 4][slot0 + from / 8][from % 4] * ((const float*)sine)[j];
              v[k] = v[k] * ((const float*)cosine)[j] + (low ? -z : z);
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
      out.store((char*)a.q + (t0 + now) * a.ldq + ((int64_t)head * D + 8 * chunk) * sizeof(X));
    } else {
      const int64_t kv_off = kRows == 1 ? at.kv_off : place[now].kv_off;
      if (kv_off < 0) continue;
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
  // Several tokens where a row is not long enough to cover the latency of finding
  // its token's place (4096 tokens of 80 heads of 128: bf16, 20 KiB each, 40.4 us
  // with one, 40.5 with two or three, 37.8 with four, 45 with eight; float32 into 4
  // bits, 40 KiB each, 70 us with one, 72 with two, 73 with four), but four
  // workgroups per compute unit at least (2048 tokens of 48 heads of 128: 14.2 us so,
  // 17.4 with two, 15.8 with eight; 2224 of 10 heads of 256: 12.2, 15.1 and 12.9).
  const int64_t row = (a.heads + 2 * (int64_t)a.c.kv_heads) * a.c.head_dim * (XT == MOSAIC_F32 ? 4 : 2);
  const int64_t share = THREADS == 1024 || row > 32768 ? 1 : a.rows / 1024;
  const int rows_of = share < 1 ? 1 : share > kMostRows ? kMostRows : (int)share;
  const dim3 grid((unsigned)((a.rows + rows_of - 1) / rows_of));
  if (a.rot.pairs == 0 || a.rot.interleaved)
    cache_append_norm_kernel<XT, CT, PAIRS_OWN, STREAM, THREADS><<<grid, THREADS, 0, s>>>(a, log2_lanes, rows_of);
  else if (a.rot.pairs % 8 == 0)
    cache_append_norm_kernel<XT, CT, PAIRS_CHUNKS, STREAM, THREADS><<<grid, THREADS, 0, s>>>(a, log2_lanes, rows_of);
  else
    cache_append_norm_kernel<XT, CT, PAIRS_ANY, STREAM, THREADS><<<grid, THREADS, 0, s>>>(a, log2_lanes, rows_of);
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
