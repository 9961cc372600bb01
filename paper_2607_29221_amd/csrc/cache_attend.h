// What the kernels of the attention over pages share (cache_attend.hip over 16
// and 32 bits, cache_attend_e2m1.hip over 4): how tokens are dealt out to
// workgroups, the workspace, and the second kernel, which joins the parts.
#pragma once

#include "cache.h"
#include "device_common.h"

namespace mosaic {
namespace {

constexpr int kWaves = 4;                 // per workgroup
constexpr int kHeadTile = 16;

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// max or sum over the four lanes of a head (lane mod 16)
__device__ __forceinline__ float head_max(float v) {
  auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float head_sum(float v) {
  auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

template <class T> struct Chunk { T e[16 / sizeof(T)]; };

// Every wave's writes to LDS before every wave's reads after; memory accesses
// go on (a __syncthreads waits for those too).
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// Tokens are dealt out in steps of kStepTokens (a sequence's last one may be
// short). With `total` steps of all sequences, workgroup u of a key/value head
// takes the steps u * share .. of the sequences laid end to end, share =
// ceil(total / workgroups). Its part of sequence b has slot u + b: going on, a
// workgroup or a sequence ends, so no two parts have the same.
constexpr int kStepTokens = 128;
// Workgroups go to the chip's dies in turn. The blocks of query heads of a
// share lie this far apart, so that they read its keys and values through one
// die's L2 (64 query heads on one key/value head, 64 sequences of up to 16000
// tokens, this kernel alone: 91 us side by side, 75 us so).
constexpr int kXcds = 8;

// The workspace: per slot and query head the base and the sum of the weights
// and the unnormalised output; then scores.
struct Work {
  float* stat;      // [slots][heads][2]
  float* part;      // [slots][heads][head_dim]
  float* scores;    // [batch][kv_heads][row / 16][group][16]: what a wave stores at a time lies together
  int64_t row;
};

struct Plan {
  int32_t workgroups;                     // per key/value head and tile group
  int32_t wave_tiles, tile_groups;        // blocks of 16 query heads of a group: per wave, and so many times
};

// two_fit: whether a unit's LDS holds two workgroups; there are never more of them
// without than with it (which the workspace is sized for).
Plan plan_of(const CacheView& c, int32_t heads, int64_t max_len, bool two_fit = true) {
  Plan p;
  const int32_t tiles = (heads / c.kv_heads + kHeadTile - 1) / kHeadTile;
  // two blocks share a wave's keys and values where the registers hold both outputs
  p.wave_tiles = tiles > 1 && c.head_dim <= 128 ? 2 : 1;
  p.tile_groups = (tiles + p.wave_tiles - 1) / p.wave_tiles;
  // A workgroup per compute unit, or as many as there are steps: its four
  // waves keep 64 KiB of a bf16 cache's rows of 128 in flight, which is
  // enough, and every further workgroup is another part to join (64 sequences
  // with the join: 164 us with 256 workgroups in all, 166 us with 512, 168 us
  // with 768; 8 heads of 256 elements on one 52, 59 and 66 us). Where several
  // blocks of query heads read the same keys, two per unit hide each other's
  // waits (128 heads on one key/value head, kernel alone: float32 over bf16 178
  // us with one, 142 us with two; bf16 122 and 117 us; 48 heads of 256 elements,
  // where the registers hold one, 178 and 180 us). Never more than fit at
  // once, since a unit with two takes twice as long (12 key/value heads: 249 us
  // with 264, 173 us with 252), but more per unit where more than one unit in 16
  // would idle (71 heads: 217 us with 213, 186 us with 497). Over 4 bits, where the
  // arithmetic takes as long as the rows, two per unit as long as its LDS holds them
  // (131072 tokens of 32 and 8 heads: 39 us with 256 in all, 35 with 512, 37.5 with 768),
  // which with float32 activations, weights and blocks of 32 heads it does not (32 heads
  // on one: one sequence of 131072 66 us with 512, 47 with 256, 32 of up to 7168 59 and 51).
  const bool two = two_fit && c.head_dim <= 128 && (p.tile_groups > 1 || c.dtype == MOSAIC_E2M1);
  int32_t slots = two ? 512 : 256;
  int64_t wanted;
  while (true) {
    const int64_t shares = p.tile_groups > 1 ? slots / kXcds / p.tile_groups * kXcds : slots;
    wanted = shares / c.kv_heads;
    if (slots == 1024 || 16 * wanted * c.kv_heads * p.tile_groups >= 15 * slots) break;
    slots += 256;
  }
  if (wanted == 0) wanted = 1;
  const int64_t steps = c.batch * ((max_len + kStepTokens - 1) / kStepTokens);
  p.workgroups = (int32_t)(wanted < steps ? wanted : steps > 0 ? steps : 1);
  return p;
}

int64_t padded_len(int64_t max_len) { return (max_len + 63) / 64 * 64; }

// floats of the workspace before the scores: statistics (padded to 16 bytes) and outputs
int64_t stat_floats(const CacheView& c, int32_t heads, const Plan& p) {
  return (((int64_t)c.batch + p.workgroups) * heads * 2 + 3) / 4 * 4;
}
int64_t part_floats(const CacheView& c, int32_t heads, const Plan& p) {
  return ((int64_t)c.batch + p.workgroups) * heads * c.head_dim;
}

// Over 4 bits a sequence counts kStartSteps more steps behind its own: to begin
// another one costs a workgroup about as long (64 sequences of 512 to 7168 tokens:
// without, a workgroup's end lay between 45 and 70 us). Where shares are shorter
// than kLongShare steps it would leave workgroups without any.
constexpr int kStartSteps = 2, kLongShare = 16;

// Steps of sequence i, 0 beyond the batch.
__device__ __forceinline__ int steps_of(const AttendLaunch& a, int i, int extra) {
  const int steps = i < a.c.batch ? (held_tokens(a.lengths, i, a.max_len) + kStepTokens - 1) / kStepTokens : 0;
  return steps > 0 ? steps + extra : 0;
}
// Steps of the first 64 sequences, a lane each: its own, and all up to it; and
// what all sequences count more.
struct FirstSteps {
  int own, upto, extra;
};
// Steps of all sequences, by one wave.
__device__ __forceinline__ int all_steps(const AttendLaunch& a, int lane, FirstSteps* first) {
  first->own = steps_of(a, lane, first->extra);
  first->upto = wave_scan(first->own);
  int total = __builtin_amdgcn_readlane(first->upto, 63);
  for (int i0 = 64; i0 < a.c.batch; i0 += 64)
    total += __builtin_amdgcn_readlane(wave_scan(steps_of(a, i0 + lane, first->extra)), 63);
  return total;
}
// Steps of a share, at least 1, and in *total those of all sequences. starts:
// whether sequences may count more than their own.
__device__ __forceinline__ int share_of_steps(const AttendLaunch& a, int lane, int workgroups, bool starts, FirstSteps* first,
                                              int* total) {
  first->extra = 0;
  *total = all_steps(a, lane, first);
  if (starts && a.c.batch > 1 && *total / workgroups >= kLongShare) {
    first->extra = kStartSteps;
    *total = all_steps(a, lane, first);
  }
  return max((*total + workgroups - 1) / workgroups, 1);
}
// Steps of the sequences before b.
__device__ __forceinline__ int steps_before(const AttendLaunch& a, int lane, int b, const FirstSteps& first) {
  if (b < 64) return __builtin_amdgcn_readlane(first.upto - first.own, b);
  int carry = __builtin_amdgcn_readlane(first.upto, 63);
  for (int i0 = 64; ; i0 += 64) {
    const int own = steps_of(a, i0 + lane, first.extra), upto = wave_scan(own);
    if (b < i0 + 64) return carry + __builtin_amdgcn_readlane(upto - own, b - i0);
    carry += __builtin_amdgcn_readlane(upto, 63);
  }
}
// The sequence that holds step s, and the steps before it; -1 if the lengths
// do not add up to that.
__device__ __forceinline__ int sequence_at(const AttendLaunch& a, int lane, int s, const FirstSteps& first, int* before) {
  int carry = 0, own = first.own, upto = first.upto;
  for (int i0 = 0; ; ) {
    const uint64_t past = __ballot(carry + upto > s);
    if (past != 0) {
      const int l = __builtin_ctzll(past);
      *before = carry + __builtin_amdgcn_readlane(upto - own, l);
      return i0 + l;
    }
    i0 += 64;
    if (i0 >= a.c.batch) return -1;
    carry += __builtin_amdgcn_readlane(upto, 63);
    own = steps_of(a, i0 + lane, first.extra);
    upto = wave_scan(own);
  }
}

// Base and sum of a head over its parts, `stride` floats apart, by one wave.
__device__ __forceinline__ void head_norm(const float* st, int64_t stride, int parts, int lane, float* common,
                                          float* sum) {
  float m = -INFINITY, l = 0.0f;
  for (int s = lane; s < parts; s += 64) m = fmaxf(m, st[s * stride]);
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) m = fmaxf(m, __shfl_xor(m, off));
  for (int s = lane; s < parts; s += 64)
    l += st[s * stride + 1] * (st[s * stride] == -INFINITY ? 0.0f : exp2_fast(st[s * stride] - m));
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) l += __shfl_xor(l, off);
  *common = m == -INFINITY ? 0.0f : m;
  *sum = l;
}

// Joins the parts (4 to 5 us: the latency of the lengths, the parts and the
// store). The first `out_groups` workgroups of a key/value head write
// the outputs of `out_heads` query heads each: rows of 16-byte columns, a
// head's parts dealt out to its share of the rows of threads. The others add
// weights up over the heads of the group, kJoinTokens tokens at a time (64
// sequences: 21 us in all, 4 TB/s of scores, weights and parts).
constexpr int kJoinHeads = 16, kJoinTokens = 4 * 256;
template <int XT>
__global__ __launch_bounds__(256) void cache_join_kernel(AttendLaunch a, Work wk, int32_t workgroups, int32_t out_heads) {
  typedef typename FloatType<XT>::type X;
  __shared__ f32x4 rows[256];
  __shared__ float row_stat[129][2];              // at most 128 rows of threads, and the threads over
  __shared__ float norm[kJoinHeads][2];           // common base, 1 / sum
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int h = blockIdx.x, b = blockIdx.y, group = a.heads / a.c.kv_heads, D = a.c.head_dim;
  const int out_groups = (group + out_heads - 1) / out_heads;
  const int n = held_tokens_uniform(a.lengths, b, a.max_len);
  FirstSteps first64;
  int total;
  const int share = share_of_steps(a, lane, workgroups, a.c.dtype == MOSAIC_E2M1, &first64, &total);
  const int before = steps_before(a, lane, b, first64);
  const int steps = (n + kStepTokens - 1) / kStepTokens, u0 = before / share;
  const int parts = steps == 0 ? 0 : (before + steps - 1) / share - u0 + 1;
  const int64_t head0 = (int64_t)(u0 + b) * a.heads + h * group;      // of the first part
  const int64_t stride = 2 * (int64_t)a.heads;
  if ((int)blockIdx.z < out_groups) {
    const int g0 = blockIdx.z * out_heads, count = min(group - g0, out_heads);
    const int cols = D / 4, each = 256 / cols / out_heads;            // rows of a head
    const int c = tid % cols, r = tid / cols, hd = r / each, s0 = r - hd * each;
    f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
    float base = -INFINITY, sum = 0.0f;
    // adds what has base m and sum l
    auto add = [&](f32x4 x, float m, float l) {
      const float now = fmaxf(base, m);
      const float f = base == -INFINITY ? 0.0f : exp2_fast(base - now), e = m == -INFINITY ? 0.0f : exp2_fast(m - now);
      o = o * f + x * e;
      sum = sum * f + l * e;
      base = now;
    };
    if (hd < count) {
      const float* st = wk.stat + 2 * (head0 + g0 + hd);
      const float* part = wk.part + (head0 + g0 + hd) * D + 4 * c;
#pragma unroll 4
      for (int s = s0; s < parts; s += each)
        add(*(const f32x4*)(part + (int64_t)s * a.heads * D), st[s * stride], st[s * stride + 1]);
    }
    rows[tid] = o;
    if (c == 0) {
      row_stat[r][0] = base;
      row_stat[r][1] = sum;
    }
    __syncthreads();
    if (hd >= count || s0 > 0) return;
    for (int s = 1; s < each; ++s) add(rows[tid + s * cols], row_stat[r + s][0], row_stat[r + s][1]);
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    X* dst = (X*)((char*)a.out + (int64_t)b * a.ldo) + (int64_t)(h * group + g0 + hd) * D + 4 * c;
#pragma unroll
    for (int i = 0; i < 4; ++i) dst[i] = (X)(o[i] * inv);
    return;
  }
  // base and 1 / sum of heads g0 .. g0 + count - 1 of the group
  auto norms = [&](int g0, int count) {
    for (int g = wave; g < count; g += 4) {
      float common, sum;
      head_norm(wk.stat + 2 * (head0 + g0 + g), stride, parts, lane, &common, &sum);
      if (lane == 0) {
        norm[g][0] = common;
        norm[g][1] = sum == 0.0f ? 0.0f : 1.0f / sum;
      }
    }
    __syncthreads();
  };
  for (int t0 = ((int)blockIdx.z - out_groups) * kJoinTokens; t0 < n; t0 += ((int)gridDim.z - out_groups) * kJoinTokens) {
    const int t = t0 + 4 * tid;                     // four tokens of one page
    const float* scores = wk.scores + ((int64_t)b * a.heads + h * group) * wk.row + (int64_t)(t & ~15) * group + (t & 15);
    f32x4 w = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int g0 = 0; g0 < group; g0 += kJoinHeads) {
      const int count = min(group - g0, kJoinHeads);
      __syncthreads();
      norms(g0, count);
      if (t < n) {
#pragma unroll 8
        for (int g = 0; g < count; ++g) {
          const f32x4 score = *(const f32x4*)(scores + 16 * (g0 + g));
#pragma unroll
          for (int i = 0; i < 4; ++i) w[i] += exp2_fast(score[i] - norm[g][0]) * norm[g][1];
        }
      }
    }
    const int page = t < n ? page_of(a.c, b, t) : -1;
    if (page < 0) continue;
    float* dst = a.c.weights + row_index(a.c, page, h, t);
    if (t + 4 <= n) {
      *(f32x4_any*)dst += w;
    } else {
#pragma unroll
      for (int i = 0; i < 3; ++i)
        if (t + i < n) dst[i] += w[i];
    }
  }
}
Work work_of(const AttendLaunch& a, const Plan& p) {
  Work w;
  w.stat = (float*)a.workspace;
  w.part = w.stat + stat_floats(a.c, a.heads, p);
  w.scores = w.part + part_floats(a.c, a.heads, p);
  w.row = padded_len(a.max_len);
  return w;
}

template <int XT>
void launch_join(const AttendLaunch& a, const Work& w, const Plan& p, hipStream_t s) {
  // weights: a workgroup per range of tokens, fewer where the heads are many
  int64_t ranges = 0;
  if (a.accumulate) {
    const int64_t all = (a.max_len + kJoinTokens - 1) / kJoinTokens;
    const int64_t most = 4096 / ((int64_t)a.c.kv_heads * a.c.batch) + 1;
    ranges = all < most ? all : most;
  }
  // several heads per workgroup where there are many and a sequence has few parts
  const int32_t group = a.heads / a.c.kv_heads, rows = 256 / (a.c.head_dim / 4);
  int32_t out_heads = (int64_t)a.c.kv_heads * a.c.batch < 64 ? 1 : rows < 4 ? rows : 4;
  if (out_heads > group) out_heads = group;
  const unsigned z = (unsigned)((group + out_heads - 1) / out_heads + ranges);
  cache_join_kernel<XT><<<dim3(a.c.kv_heads, a.c.batch, z), 256, 0, s>>>(a, w, p.workgroups, out_heads);
}

}  // namespace
}  // namespace mosaic
