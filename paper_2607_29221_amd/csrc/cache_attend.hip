// Attention of one new token per sequence over its paged cache
// (mosaic_cache_attend), simplest form: all scores to memory, a softmax over
// them and the weighted sum of the values, then the sums of weights.
#include "cache.h"
#include "dispatch.h"

namespace mosaic {
namespace {

// s[b][g][i] = scale_log2 q_g . k_i, -inf where there is no token.
template <int XT, int CT>
__global__ __launch_bounds__(256) void cache_scores_kernel(AttendLaunch a, float* scores, int64_t lp) {
  typedef typename FloatType<XT>::type X;
  typedef typename FloatType<CT>::type C;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int g = blockIdx.y, b = blockIdx.z;
  if (i >= lp) return;
  const int32_t page = i < held_tokens(a.lengths, b, a.max_len) ? page_of(a.c, b, i) : -1;
  float acc = 0.0f;
  if (page >= 0) {
    const X* q = (const X*)((const char*)a.q + b * a.ldq) + (int64_t)g * a.c.head_dim;
    const C* k = (const C*)(a.c.k + row_offset(a.c, page, g / (a.heads / a.c.kv_heads), i));
    for (int d = 0; d < a.c.head_dim; ++d) acc += (float)q[d] * (float)k[d];
  }
  scores[((int64_t)b * a.heads + g) * lp + i] = page >= 0 ? acc * a.scale_log2 : -INFINITY;
}

__device__ __forceinline__ float block_reduce(float v, bool max, float* red) {
  for (int off = 32; off > 0; off >>= 1) {
    const float o = __shfl_xor(v, off);
    v = max ? fmaxf(v, o) : v + o;
  }
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  return max ? fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3])) : red[0] + red[1] + red[2] + red[3];
}

template <int XT, int CT>
__global__ __launch_bounds__(256) void cache_values_kernel(AttendLaunch a, const float* scores, float* norm, int64_t lp) {
  typedef typename FloatType<XT>::type X;
  typedef typename FloatType<CT>::type C;
  __shared__ float red[4];
  const int g = blockIdx.x, b = blockIdx.y;
  const float* s = scores + ((int64_t)b * a.heads + g) * lp;
  const int32_t n = held_tokens(a.lengths, b, a.max_len);
  float m = -INFINITY;
  for (int i = threadIdx.x; i < n; i += 256) m = fmaxf(m, s[i]);
  m = block_reduce(m, true, red);
  const float base = m == -INFINITY ? 0.0f : m;
  float l = 0.0f;
  for (int i = threadIdx.x; i < n; i += 256) l += exp2f(s[i] - base);
  l = block_reduce(l, false, red);
  if (threadIdx.x == 0) {
    norm[2 * ((int64_t)b * a.heads + g)] = base;
    norm[2 * ((int64_t)b * a.heads + g) + 1] = l > 0.0f ? 1.0f / l : 0.0f;
  }
  const int d = threadIdx.x;
  if (d >= a.c.head_dim) return;
  float acc = 0.0f;
  for (int i = 0; i < n; ++i) {
    const int32_t page = page_of(a.c, b, i);
    if (page < 0) continue;
    acc += exp2f(s[i] - base) * (float)((const C*)(a.c.v + row_offset(a.c, page, g / (a.heads / a.c.kv_heads), i)))[d];
  }
  ((X*)((char*)a.out + b * a.ldo))[(int64_t)g * a.c.head_dim + d] = (X)(l > 0.0f ? acc / l : 0.0f);
}

__global__ __launch_bounds__(256) void cache_weights_kernel(AttendLaunch a, const float* scores, const float* norm,
                                                            int64_t lp) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int h = blockIdx.y, b = blockIdx.z;
  if (i >= held_tokens(a.lengths, b, a.max_len)) return;
  const int32_t page = page_of(a.c, b, i);
  if (page < 0) return;
  const int group = a.heads / a.c.kv_heads;
  float w = 0.0f;
  for (int g = 0; g < group; ++g) {
    const int64_t row = (int64_t)b * a.heads + h * group + g;
    w += exp2f(scores[row * lp + i] - norm[2 * row]) * norm[2 * row + 1];
  }
  a.c.weights[row_index(a.c, page, h, i)] += w;
}

int64_t padded_len(int64_t max_len) { return (max_len + 63) / 64 * 64; }

template <int XT, int CT>
void launch_types(const AttendLaunch& a, hipStream_t s) {
  const int64_t lp = padded_len(a.max_len);
  float* scores = (float*)a.workspace;
  float* norm = scores + (int64_t)a.c.batch * a.heads * lp;
  const unsigned blocks = (unsigned)((lp + 255) / 256);
  if (lp > 0) cache_scores_kernel<XT, CT><<<dim3(blocks, a.heads, a.c.batch), 256, 0, s>>>(a, scores, lp);
  cache_values_kernel<XT, CT><<<dim3(a.heads, a.c.batch), 256, 0, s>>>(a, scores, norm, lp);
  if (a.accumulate && lp > 0)
    cache_weights_kernel<<<dim3(blocks, a.c.kv_heads, a.c.batch), 256, 0, s>>>(a, scores, norm, lp);
}

}  // namespace

int64_t cache_attend_workspace(const CacheView& c, int32_t heads, int64_t max_len, int32_t) {
  return (int64_t)c.batch * heads * (padded_len(max_len) + 2) * 4;
}

hipError_t launch_cache_attend(const AttendLaunch& a, hipStream_t s) {
  if (a.x_dtype == MOSAIC_F32 && a.c.dtype == MOSAIC_F32) launch_types<MOSAIC_F32, MOSAIC_F32>(a, s);
  else if (a.x_dtype == MOSAIC_F32 && a.c.dtype == MOSAIC_BF16) launch_types<MOSAIC_F32, MOSAIC_BF16>(a, s);
  else if (a.x_dtype == MOSAIC_F32) launch_types<MOSAIC_F32, MOSAIC_F16>(a, s);
  else if (a.c.dtype == MOSAIC_BF16) launch_types<MOSAIC_BF16, MOSAIC_BF16>(a, s);
  else launch_types<MOSAIC_F16, MOSAIC_F16>(a, s);
  return hipGetLastError();
}

}  // namespace mosaic
