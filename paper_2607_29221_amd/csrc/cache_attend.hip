// Attention of one new token per sequence over its paged cache
// (mosaic_cache_attend).
//
// For the query heads g of one key/value head, with scores in powers of two
// (s = scale log2(e) q k):
//     out = sum_i 2^(s_i - M) v_i / sum_i 2^(s_i - M),
// in one pass over the keys and values with a running M. Every key and value
// is read once from memory and used by all heads of its group, so the call is
// bound by that traffic; the arithmetic is laid out to stay in its shadow:
//
// * A wave works on 32 tokens at a time (16 of a float32 cache), in the
//   matrix cores: S^T = K Q^T, then O^T += V^T P^T. In both products the 16
//   columns are query heads, and a lane holds head (lane mod 16) and a quarter
//   of the tokens: what the first product leaves in a lane is what the second
//   needs there, so P never moves between lanes, and M, the sum and the
//   rescaling of O are a lane's own.
// * Keys are loaded as the first product's operand as they lie. The second
//   takes a value's tokens along its inner dimension: a lane loads 16 bytes
//   of 8 tokens' rows and turns them with byte permutes (32 for 32 tokens of
//   128), so nothing passes through LDS.
// * Activations in float32 over a 16-bit cache keep their precision: q and p
//   are split into 16-bit parts (three of bf16, two of f16 with the range
//   centred) that are multiplied one after the other into the same sums. The
//   matrix cores have room for it (a sixth of their rate at full bandwidth).
// * M is raised, and O rescaled, only when a score passes it by more than
//   kSlack: sums of up to 2^kSlack are as exact as sums of up to 1.
// * Sequences are cut into pieces so that there are workgroups for all
//   compute units; a second kernel joins the pieces, and adds up attention
//   weights from the scores that the first one left in the workspace.
#include "cache.h"
#include "device_common.h"
#include "dispatch.h"

namespace mosaic {
namespace {

constexpr int kWaves = 4;                 // per workgroup
constexpr int kHeadTile = 16;

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// The buffer a page's rows of one head are read through: a load past `bytes`
// gives zeros.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_rsrc(const char* base, int bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(base), (short)0, bytes, 0x00020000);
}
constexpr int kNowhere = 0x40000000;      // an offset past every page
constexpr int kStream = 2;                // cache policy: read once, not to be kept

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

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// What the types of cache and activations make of a wave's step. DP: head_dim
// padded to 64, 128 or 256 (columns beyond head_dim are zeros).
template <int CT, int XT, int DP> struct Form {
  typedef typename FloatType<CT>::type C;
  typedef typename FloatType<XT>::type X;
  static constexpr bool kWide = CT == MOSAIC_F32;
  static constexpr int kParts = kWide || XT != MOSAIC_F32 ? 1 : CT == MOSAIC_BF16 ? 3 : 2;
  static constexpr int kSub = kWide ? 1 : 2;                // blocks of 16 tokens
  static constexpr int kTokens = 16 * kSub;
  static constexpr int kKeyLoads = DP * (int)sizeof(C) / 64;  // 16 bytes per lane and block of 16 tokens
  static constexpr int kEach = kWide ? 4 : DP == 64 ? 4 : 8;  // elements per lane of a value load
  static constexpr int kValueLoads = DP / 16 / kEach;       // per token row
  static constexpr int kRows = 4 * kSub;                    // token rows per lane
  // p <= 2^kSlack / 2^kShift: f16 parts of p keep 22 bits down to 2^-25
  static constexpr float kSlack = CT == MOSAIC_F16 ? 4.0f : 8.0f;
  static constexpr float kShift = CT == MOSAIC_F16 ? 11.0f : 0.0f;
};

template <int CT> struct Matrix;
template <> struct Matrix<MOSAIC_BF16> {
  typedef bf16x8 Frag;
  static __device__ __forceinline__ f32x4 mul(Frag a, Frag b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  }
};
template <> struct Matrix<MOSAIC_F16> {
  typedef f16x8 Frag;
  static __device__ __forceinline__ f32x4 mul(Frag a, Frag b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
  }
};
template <> struct Matrix<MOSAIC_F32> {
  typedef f32x4 Frag;                     // four steps of one product
  static __device__ __forceinline__ f32x4 mul(Frag a, Frag b, f32x4 c) {
#pragma unroll
    for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
    return c;
  }
};

// x as the sum of PARTS 16-bit numbers, each rounded from what the ones before leave.
template <class T, int PARTS>
__device__ __forceinline__ void split(float x, T* part) {
#pragma unroll
  for (int s = 0; s < PARTS; ++s) {
    part[s] = (T)x;
    x -= (float)part[s];
  }
}

// The pieces of the workspace: per (sequence, query head, piece) the base and
// the sum of its weights and its unnormalised output; then scores.
struct Work {
  float* stat;      // [batch][heads][pieces][2]
  float* part;      // [batch][heads][pieces][head_dim]
  float* scores;    // [batch][kv_heads][row / 16][group][16]: what a wave stores at a time lies together
  int64_t row;
  int32_t pieces;
  int32_t piece;    // tokens of a piece
};

struct Plan {
  int32_t pieces, piece;
  int32_t head_tiles, tiles_per_wg;       // blocks of 16 query heads of a group
  bool join;
};

Plan plan_of(const CacheView& c, int32_t heads, int64_t max_len, int32_t accumulate) {
  Plan p;
  p.head_tiles = (heads / c.kv_heads + kHeadTile - 1) / kHeadTile;
  p.tiles_per_wg = p.head_tiles == 1 ? 1 : p.head_tiles == 2 ? 2 : 4;
  const int64_t groups = (int64_t)c.batch * c.kv_heads * ((p.head_tiles + p.tiles_per_wg - 1) / p.tiles_per_wg);
  const int64_t step = 32 * kWaves / p.tiles_per_wg;
  // One sequence: as many workgroups as run at once. Several, of lengths that
  // only the device knows: four times as many, so that short ones even out.
  const int64_t wanted = ((c.batch == 1 ? 512 : 2048) + groups - 1) / groups;
  int64_t piece = (max_len + wanted - 1) / wanted;
  piece = (piece + step - 1) / step * step;
  if (piece < step) piece = step;
  p.piece = (int32_t)piece;
  p.pieces = max_len > 0 ? (int32_t)((max_len + piece - 1) / piece) : 1;
  p.join = p.pieces > 1 || accumulate;
  return p;
}

int64_t padded_len(int64_t max_len) { return (max_len + 63) / 64 * 64; }

// floats of the workspace before the scores: statistics (padded to 16 bytes) and outputs
int64_t stat_floats(const CacheView& c, int32_t heads, const Plan& p) {
  return ((int64_t)c.batch * heads * p.pieces * 2 + 3) / 4 * 4;
}
int64_t part_floats(const CacheView& c, int32_t heads, const Plan& p) {
  return (int64_t)c.batch * heads * p.pieces * c.head_dim;
}

template <int CT, int XT, int DP>
__global__ __launch_bounds__(64 * kWaves, DP == 256 ? 1 : 2) void cache_attend_kernel(AttendLaunch a, Work wk,
                                                                                      int32_t tiles_per_wg, bool join) {
  typedef Form<CT, XT, DP> F;
  typedef typename F::C C;
  typedef typename F::X X;
  typedef Matrix<CT> M;
  constexpr int E = F::kWide ? 4 : 8;           // elements of a 16-byte key chunk
  constexpr int NV = F::kValueLoads, EV = F::kEach;
  constexpr int kHold = 8192 / 16;              // of a wave's scores, 16 bytes each
  union Shared {
    float slab[kWaves][kHeadTile][DP + 4];      // outputs of the waves, at the end
    f32x4 held[kWaves][kHold];                  // scores on their way to memory
  };
  __shared__ Shared shared;
  auto& slab = shared.slab;
  __shared__ float stat[kWaves][kHeadTile][2];

  const int tid = threadIdx.x, lane = tid & 63, col = lane & 15, quad = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // Workgroups go to the XCDs in turn: pieces come last, so that the early
  // ones, which every sequence has, start first, and turn the sequences round,
  // so that no XCD has the long ones to itself.
  const int piece = blockIdx.z, b = (blockIdx.y + blockIdx.z) % a.c.batch;
  const int tile_groups = gridDim.x / a.c.kv_heads;
  const int h = blockIdx.x / tile_groups, tile = (blockIdx.x % tile_groups) * tiles_per_wg + wave % tiles_per_wg;
  const int group = a.heads / a.c.kv_heads, D = a.c.head_dim;
  const int n = held_tokens(a.lengths, b, a.max_len);
  const int t0 = piece * wk.piece, t1 = min(n, t0 + wk.piece);
  const int lanes_of_tokens = kWaves / tiles_per_wg;
  if (t0 > 0 && t0 >= n) return;                // pieces past the end are not read back

  // queries of head `head` of the group: operand of the first product, in parts
  const int head = tile * kHeadTile + col;
  const bool live = head < group;
  typename M::Frag q[F::kParts][F::kKeyLoads];
  float scale = a.scale_log2;
  {
    const X* row = (const X*)((const char*)a.q + (int64_t)b * a.ldq) + ((int64_t)h * group + head) * D;
    float x[F::kKeyLoads][E];
    float top = 0.0f;
#pragma unroll
    for (int c = 0; c < F::kKeyLoads; ++c) {
      const int d = (4 * c + quad) * E;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        x[c][e] = live && d < D ? (float)row[d + e] : 0.0f;
        top = fmaxf(top, fabsf(x[c][e]));
      }
    }
    if (CT == MOSAIC_F16 && XT == MOSAIC_F32) {
      // by a power of two into the upper part of the range of f16
      top = head_max(top);
      const int up = top > 0.0f && top < INFINITY ? 14 - __builtin_amdgcn_frexp_expf(top) : 0;
      scale = ldexpf(scale, -up);
#pragma unroll
      for (int c = 0; c < F::kKeyLoads; ++c)
#pragma unroll
        for (int e = 0; e < E; ++e) x[c][e] = ldexpf(x[c][e], up);
    }
#pragma unroll
    for (int c = 0; c < F::kKeyLoads; ++c)
#pragma unroll
      for (int e = 0; e < E; ++e) {
        C part[F::kParts];
        split<C, F::kParts>(x[c][e], part);
#pragma unroll
        for (int s = 0; s < F::kParts; ++s) q[s][c][e] = part[s];
      }
  }

  // a lane's offsets within a block of 16 rows; columns past head_dim lie nowhere
  const int ts = (int)a.c.token_stride;
  int key_off[F::kKeyLoads], value_off[NV];
#pragma unroll
  for (int c = 0; c < F::kKeyLoads; ++c) key_off[c] = (4 * c + quad) * E < D ? col * ts + (4 * c + quad) * 16 : kNowhere;
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int d = (16 * v + col) * EV;
    value_off[v] = d < D ? 4 * quad * ts + d * (int)sizeof(C) : kNowhere;
  }

  // a block of 16 tokens: its first row's place in memory and how many there are
  struct Block {
    int64_t base;
    int valid;
  };
  const int page_mask = (1 << a.c.log2_page) - 1;
  auto block_at = [&](int slot) {
    Block k = {0, 0};
    if (slot < t1) {
      const int page = page_of_uniform(a.c, b, slot);
      if (page >= 0) {
        k.base = (int64_t)page * a.c.page_stride + (int64_t)h * a.c.head_stride + (slot & page_mask) * ts;
        k.valid = min(t1 - slot, 16);
      }
    }
    return k;
  };

  f32x4 acc[NV][EV];
#pragma unroll
  for (int v = 0; v < NV; ++v)
#pragma unroll
    for (int j = 0; j < EV; ++j) acc[v][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  float top = -INFINITY, base = 0.0f, sum = 0.0f;

  const int stride = F::kTokens * lanes_of_tokens;
  const int first_of_wave = t0 + F::kTokens * (wave / tiles_per_wg);

  // Scores go to memory through LDS, many steps at a time: a load that is
  // issued behind a store waits for it, and stores take longer than loads.
  float* scores = wk.scores + ((int64_t)b * a.heads + h * group) * wk.row + 16 * head + 4 * quad;
  const int tile_heads = min(max(group - tile * kHeadTile, 1), kHeadTile);
  f32x4* held = &shared.held[wave][quad * tile_heads + min(col, tile_heads - 1)];
  int holding = 0, held_from = first_of_wave;   // blocks of 16 tokens, and the first one's step
  auto release = [&]() {
    if (live)
      for (int k = 0; k < holding; ++k)
        *(f32x4*)(scores + (int64_t)(held_from + k / F::kSub * stride + k % F::kSub * 16) * group) = held[4 * tile_heads * k];
    held_from += holding / F::kSub * stride;
    holding = 0;
  };
  typename M::Frag key[F::kSub][F::kKeyLoads];
  Block cur[F::kSub];
  auto load_keys = [&](const Block* k) {
#pragma unroll
    for (int s = 0; s < F::kSub; ++s) {
      const __amdgpu_buffer_rsrc_t r = rows_rsrc(a.c.k + k[s].base, k[s].valid * ts);
#pragma unroll
      for (int c = 0; c < F::kKeyLoads; ++c)
        key[s][c] = __builtin_bit_cast(typename M::Frag,
                                       __builtin_amdgcn_raw_buffer_load_b128(r, key_off[c], 0, kStream));
    }
  };
#pragma unroll
  for (int s = 0; s < F::kSub; ++s) cur[s] = block_at(first_of_wave + 16 * s);
  load_keys(cur);

  for (int t = first_of_wave; t < t1; t += stride) {
    // values of these tokens, keys of the next ones: in flight during the arithmetic
    u32x4 value[F::kRows][NV];
#pragma unroll
    for (int s = 0; s < F::kSub; ++s) {
      const __amdgpu_buffer_rsrc_t r = rows_rsrc(a.c.v + cur[s].base, cur[s].valid * ts);
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int v = 0; v < NV; ++v) {
          if (EV * sizeof(C) == 16) {
            value[4 * s + i][v] =
                __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, value_off[v] + i * ts, 0, kStream));
          } else {
            const u32x2 w =
                __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(r, value_off[v] + i * ts, 0, kStream));
            value[4 * s + i][v] = u32x4{w[0], w[1], 0u, 0u};
          }
        }
    }
    Block next[F::kSub];
#pragma unroll
    for (int s = 0; s < F::kSub; ++s) next[s] = block_at(t + stride + 16 * s);

    float p[F::kRows];
    float tile_top = -INFINITY;
#pragma unroll
    for (int s = 0; s < F::kSub; ++s) {
      f32x4 dot = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int part = F::kParts - 1; part >= 0; --part)       // small terms first
#pragma unroll
        for (int c = 0; c < F::kKeyLoads; ++c) dot = M::mul(key[s][c], q[part][c], dot);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        p[4 * s + i] = 4 * quad + i < cur[s].valid ? dot[i] * scale : -INFINITY;
        tile_top = fmaxf(tile_top, p[4 * s + i]);
      }
    }
    load_keys(next);
    if (a.accumulate) {
      if (4 * tile_heads * (holding + F::kSub) > kHold) release();
#pragma unroll
      for (int s = 0; s < F::kSub; ++s)
        if (live) held[4 * tile_heads * (holding + s)] = f32x4{p[4 * s], p[4 * s + 1], p[4 * s + 2], p[4 * s + 3]};
      holding += F::kSub;
    }

    if (__any(tile_top > top + F::kSlack)) {
      const float now = fmaxf(top, head_max(tile_top));
      const float rescaled = now == -INFINITY ? 0.0f : now - F::kShift;
      const float f = top == -INFINITY ? 0.0f : exp2_fast(base - rescaled);
      sum *= f;
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int j = 0; j < EV; ++j) acc[v][j] *= f;
      top = now;
      base = rescaled;
    }
    typename M::Frag pf[F::kParts];
#pragma unroll
    for (int i = 0; i < F::kRows; ++i) {
      const float w = exp2_fast(p[i] - base);
      sum += w;
      C part[F::kParts];
      split<C, F::kParts>(w, part);
#pragma unroll
      for (int s = 0; s < F::kParts; ++s) pf[s][i] = part[s];
    }

#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int j = 0; j < EV; ++j) {
        typename M::Frag vf;
        if constexpr (F::kWide) {
#pragma unroll
          for (int i = 0; i < 4; ++i) vf[i] = __uint_as_float(value[i][v][j]);
        } else {
          u32x4 w;
#pragma unroll
          for (int i = 0; i < 4; ++i)
            w[i] = __builtin_amdgcn_perm(value[2 * i + 1][v][j / 2], value[2 * i][v][j / 2], j % 2 ? 0x07060302u : 0x05040100u);
          vf = __builtin_bit_cast(typename M::Frag, w);
        }
#pragma unroll
        for (int part = F::kParts - 1; part >= 0; --part) acc[v][j] = M::mul(vf, pf[part], acc[v][j]);
      }
#pragma unroll
    for (int s = 0; s < F::kSub; ++s) cur[s] = next[s];
  }

  if (a.accumulate) release();

  // join the waves that share heads
  sum = head_sum(sum);
  if (quad == 0) {
    stat[wave][col][0] = top == -INFINITY ? -INFINITY : base;
    stat[wave][col][1] = sum;
  }
  __syncthreads();
  {
    float common = -INFINITY;
    for (int w = wave % tiles_per_wg; w < kWaves; w += tiles_per_wg) common = fmaxf(common, stat[w][col][0]);
    const float f = stat[wave][col][0] == -INFINITY ? 0.0f : exp2_fast(base - common);
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < EV; j += 4)
          *(f32x4*)&slab[wave][col][(16 * v + 4 * quad + i) * EV + j] =
              f32x4{acc[v][j][i] * f, acc[v][j + 1][i] * f, acc[v][j + 2][i] * f, acc[v][j + 3][i] * f};
  }
  __syncthreads();
  const int chunks = D / 4;
  for (int u = tid; u < tiles_per_wg * kHeadTile * chunks; u += 64 * kWaves) {
    const int hd = u / chunks, c = u - hd * chunks, w0 = hd / kHeadTile, hc = hd % kHeadTile;
    const int g = ((blockIdx.x % tile_groups) * tiles_per_wg + w0) * kHeadTile + hc;
    if (g >= group) continue;
    f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
    float common = -INFINITY, total = 0.0f;
    for (int w = w0; w < kWaves; w += tiles_per_wg) {
      o += *(const f32x4*)&slab[w][hc][4 * c];
      common = fmaxf(common, stat[w][hc][0]);
    }
    for (int w = w0; w < kWaves; w += tiles_per_wg)
      total += stat[w][hc][1] * (stat[w][hc][0] == -INFINITY ? 0.0f : exp2_fast(stat[w][hc][0] - common));
    const int64_t row = (int64_t)b * a.heads + h * group + g;
    if (join) {
      *(f32x4*)(wk.part + (row * wk.pieces + piece) * D + 4 * c) = o;
      if (c == 0) {
        wk.stat[2 * (row * wk.pieces + piece)] = common;
        wk.stat[2 * (row * wk.pieces + piece) + 1] = total;
      }
    } else {
      X* dst = (X*)((char*)a.out + (int64_t)b * a.ldo) + (int64_t)(h * group + g) * D + 4 * c;
      const float inv = total == 0.0f ? 0.0f : 1.0f / total;
#pragma unroll
      for (int i = 0; i < 4; ++i) dst[i] = (X)(o[i] * inv);
    }
  }
}

// Base and sum of a head over its pieces, by one wave.
__device__ __forceinline__ void head_norm(const float* st, int pieces, int lane, float* common, float* sum) {
  float m = -INFINITY, l = 0.0f;
  for (int s = lane; s < pieces; s += 64) m = fmaxf(m, st[2 * s]);
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) m = fmaxf(m, __shfl_xor(m, off));
  for (int s = lane; s < pieces; s += 64) l += st[2 * s + 1] * (st[2 * s] == -INFINITY ? 0.0f : exp2_fast(st[2 * s] - m));
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) l += __shfl_xor(l, off);
  *common = m == -INFINITY ? 0.0f : m;
  *sum = l;
}

// Joins the pieces. The first `group` workgroups of a key/value head write one
// query head's output each: rows of 16-byte columns, the pieces dealt out to
// the rows of threads. The others add the weights of kJoinTokens tokens up,
// over the heads of the group.
constexpr int kJoinHeads = 16, kJoinTokens = 4 * 256;
template <int XT>
__global__ __launch_bounds__(256) void cache_join_kernel(AttendLaunch a, Work wk) {
  typedef typename FloatType<XT>::type X;
  __shared__ f32x4 rows[256];
  __shared__ float norm[kJoinHeads][2];           // common base, 1 / sum
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int h = blockIdx.x, b = blockIdx.y, group = a.heads / a.c.kv_heads, D = a.c.head_dim;
  const int n = held_tokens(a.lengths, b, a.max_len);
  const int pieces = n == 0 ? 1 : (n + wk.piece - 1) / wk.piece;
  if ((int)blockIdx.z < group) {
    const int64_t row = (int64_t)b * a.heads + h * group + blockIdx.z;
    const float* st = wk.stat + 2 * row * wk.pieces;
    float common, sum;
    head_norm(st, pieces, lane, &common, &sum);   // every wave for itself
    const int cols = D / 4, at_once = 256 / cols, c = tid % cols, s0 = tid / cols;
    f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
    if (s0 < at_once) {
      const float* part = wk.part + row * wk.pieces * D + 4 * c;
#pragma unroll 4
      for (int s = s0; s < pieces; s += at_once)
        o += *(const f32x4*)(part + (int64_t)s * D) * (st[2 * s] == -INFINITY ? 0.0f : exp2_fast(st[2 * s] - common));
    }
    rows[tid] = o;
    __syncthreads();
    if (tid >= cols) return;
    for (int s = 1; s < at_once; ++s) o += rows[s * cols + tid];
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    X* dst = (X*)((char*)a.out + (int64_t)b * a.ldo) + (int64_t)(h * group + blockIdx.z) * D + 4 * tid;
#pragma unroll
    for (int i = 0; i < 4; ++i) dst[i] = (X)(o[i] * inv);
    return;
  }
  const int t0 = ((int)blockIdx.z - group) * kJoinTokens;
  if (t0 >= n) return;
  const int t = t0 + 4 * tid;                     // four tokens of one page
  const float* scores = wk.scores + ((int64_t)b * a.heads + h * group) * wk.row + (int64_t)(t & ~15) * group + (t & 15);
  f32x4 w = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int g0 = 0; g0 < group; g0 += kJoinHeads) {
    const int count = min(group - g0, kJoinHeads);
    const int64_t row0 = (int64_t)b * a.heads + h * group + g0;
    __syncthreads();
    for (int g = wave; g < count; g += 4) {
      float common, sum;
      head_norm(wk.stat + 2 * (row0 + g) * wk.pieces, pieces, lane, &common, &sum);
      if (lane == 0) {
        norm[g][0] = common;
        norm[g][1] = sum == 0.0f ? 0.0f : 1.0f / sum;
      }
    }
    __syncthreads();
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
  if (page < 0) return;
  float* dst = a.c.weights + row_index(a.c, page, h, t);
  if (t + 4 <= n) {
    *(f32x4_any*)dst += w;
  } else {
#pragma unroll
    for (int i = 0; i < 3; ++i)
      if (t + i < n) dst[i] += w[i];
  }
}

template <int CT, int XT>
hipError_t launch_types(const AttendLaunch& a, hipStream_t s) {
  const Plan p = plan_of(a.c, a.heads, a.max_len, a.accumulate);
  Work w = {nullptr, nullptr, nullptr, padded_len(a.max_len), p.pieces, p.piece};
  if (p.join) {
    w.stat = (float*)a.workspace;
    w.part = w.stat + stat_floats(a.c, a.heads, p);
    w.scores = w.part + part_floats(a.c, a.heads, p);
  }
  const dim3 grid(a.c.kv_heads * ((p.head_tiles + p.tiles_per_wg - 1) / p.tiles_per_wg), a.c.batch, p.pieces);
  if (a.c.head_dim <= 64) cache_attend_kernel<CT, XT, 64><<<grid, 64 * kWaves, 0, s>>>(a, w, p.tiles_per_wg, p.join);
  else if (a.c.head_dim <= 128) cache_attend_kernel<CT, XT, 128><<<grid, 64 * kWaves, 0, s>>>(a, w, p.tiles_per_wg, p.join);
  else cache_attend_kernel<CT, XT, 256><<<grid, 64 * kWaves, 0, s>>>(a, w, p.tiles_per_wg, p.join);
  if (p.join) {
    const int64_t ranges = a.accumulate ? (a.max_len + kJoinTokens - 1) / kJoinTokens : 0;
    cache_join_kernel<XT><<<dim3(a.c.kv_heads, a.c.batch, (unsigned)(a.heads / a.c.kv_heads + ranges)), 256, 0, s>>>(a, w);
  }
  return hipGetLastError();
}

}  // namespace

int64_t cache_attend_workspace(const CacheView& c, int32_t heads, int64_t max_len, int32_t accumulate) {
  const Plan p = plan_of(c, heads, max_len, accumulate);
  if (!p.join) return 0;
  const int64_t scores = accumulate ? (int64_t)c.batch * heads * padded_len(max_len) : 0;
  return 4 * (stat_floats(c, heads, p) + part_floats(c, heads, p) + scores);
}

hipError_t launch_cache_attend(const AttendLaunch& a, hipStream_t s) {
  if (a.x_dtype == MOSAIC_F32 && a.c.dtype == MOSAIC_F32) return launch_types<MOSAIC_F32, MOSAIC_F32>(a, s);
  if (a.x_dtype == MOSAIC_F32 && a.c.dtype == MOSAIC_BF16) return launch_types<MOSAIC_BF16, MOSAIC_F32>(a, s);
  if (a.x_dtype == MOSAIC_F32) return launch_types<MOSAIC_F16, MOSAIC_F32>(a, s);
  if (a.c.dtype == MOSAIC_BF16) return launch_types<MOSAIC_BF16, MOSAIC_BF16>(a, s);
  return launch_types<MOSAIC_F16, MOSAIC_F16>(a, s);
}

}  // namespace mosaic
