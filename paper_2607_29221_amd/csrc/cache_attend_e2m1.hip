// Attention of one new token per sequence over its paged cache in 4 bits
// (mosaic_cache_attend; formulas, work of the matrix cores and division of the
// tokens as in cache_attend.hip).
//
// A cached element is a code times a power of two: two significant bits, which
// bf16 holds exactly, so keys and values become bf16 operands two at a time in
// one instruction each and nothing is lost to the 4 bits but what the cache
// itself lost. Queries and weights are split into bf16 parts: three of a float32
// query (24 bits) or of a weight for float32 outputs, two of an f16 query (11
// bits), one of a bf16 one, two of a weight for 16-bit outputs (at most 2^-17
// of it is left out, where the output's rounding takes 2^-12 or more).
//
// * Keys: the 16 lanes of a quarter take one token each, a quarter of its row:
//   dwords of codes and as many scale bytes lie side by side. The inner
//   dimension's order differs from the elements' by that, in the queries too.
// * Values: a lane takes the same 8 columns (4 where head_dim is at most 64) of
//   8 tokens, a dword of codes and a scale byte each, and turns them with byte
//   permutes once they are bf16.
#include <cfloat>

#include "cache_attend.h"
#include "e2m1.h"

namespace mosaic {
namespace {

template <int XT, int DP> struct Form {
  typedef typename FloatType<XT>::type X;
  static constexpr int kParts = XT == MOSAIC_F32 ? 3 : XT == MOSAIC_F16 ? 2 : 1;
  static constexpr int kWeightParts = XT == MOSAIC_F32 ? 3 : 2;
  static constexpr int kSub = 2;                            // blocks of 16 tokens
  static constexpr int kTokens = 16 * kSub;
  static constexpr int kKeyDwords = DP / 32;                // per lane and token
  static constexpr int kEach = DP == 64 ? 4 : 8;            // elements per lane of a value's piece
  static constexpr int kValuePieces = DP / 16 / kEach;
  static constexpr int kRows = 4 * kSub;                    // token rows per lane
  static constexpr float kSlack = 8.0f;
};

__device__ __forceinline__ f32x4 mul(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// A query's element as parts. Infinities and NaN are their first part; a number
// that rounds to infinity is the largest of bf16 and the rest.
template <int PARTS> __device__ __forceinline__ void split_query(float x, __bf16* part) {
#pragma unroll
  for (int s = 0; s < PARTS; ++s) {
    part[s] = (__bf16)x;
    if (s + 1 < PARTS) {
      const float most = __uint_as_float(0x7F7F0000u);
      if (fabsf(x) <= FLT_MAX && fabsf(x) > most) part[s] = (__bf16)copysignf(most, x);
      x = fabsf(x) <= FLT_MAX ? x - (float)part[s] : 0.0f;
    }
  }
}

constexpr int waves_of(int DP, int NT) { return DP == 256 ? 1 : NT == 2 ? 2 : 3; }

// NT: blocks of 16 query heads per wave; STREAM: past the caches (cache_attend.hip).
template <int XT, int DP, int NT, bool STREAM>
__global__ __launch_bounds__(64 * kWaves, waves_of(DP, NT)) void cache_attend_e2m1_kernel(AttendLaunch a, Work wk, int32_t workgroups) {
  typedef Form<XT, DP> F;
  typedef typename F::X X;
  typedef bf16x8 Frag;
  constexpr int KL = F::kKeyDwords, NV = F::kValuePieces, EV = F::kEach, PARTS = F::kParts, WPARTS = F::kWeightParts;
  constexpr int kPolicy = STREAM ? kStream : 0;
  constexpr int kHold = 8192 / 16;              // of a wave's scores, 16 bytes each
  union Shared {
    struct {
      Frag query[NT][PARTS][KL][64];            // operands of the first product, by lane
      f32x4 held[kWaves][kHold];                // scores on their way to memory
    } in;
    float slab[kWaves][kHeadTile][DP + 4];      // outputs of the waves, at the end
  };
  __shared__ Shared shared;
  __shared__ float stat[NT][kWaves][kHeadTile][2];

  const int tid = threadIdx.x, lane = tid & 63, col = lane & 15, quad = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const uint32_t share_of = blockIdx.y * kXcds + blockIdx.x % kXcds;
  const int u = share_of / (uint32_t)a.c.kv_heads, h = share_of - u * a.c.kv_heads;
  const int tile0 = blockIdx.x / kXcds * NT;
  if (u >= workgroups) return;
  const int group = a.heads / a.c.kv_heads, D = a.c.head_dim;

  int before;
  FirstSteps first64;
  const int total = all_steps(a, lane, &first64), share = (total + workgroups - 1) / workgroups;
  int at = u * share;
  const int stop = min(total, at + share);
  if (at >= stop) return;
  int b = sequence_at(a, lane, at, first64, &before);
  if (b < 0) return;
  while (true) {
    const int n = held_tokens_uniform(a.lengths, b, a.max_len), steps = (n + kStepTokens - 1) / kStepTokens;
    const int t0 = (at - before) * kStepTokens, t1 = min(n, min(stop - before, steps) * kStepTokens);

    // What only the start and the end of a part need is computed there.
    int own_lane = lane;
    asm volatile("" : "+v"(own_lane));

    // the queries, asked for first (loads come back in order); lanes without a
    // head or column read another's
    constexpr int QL = 8 * (int)sizeof(X) / 16;   // loads per chunk of 8
    u32x4 raw[NT][KL][QL];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int head = min((tile0 + nt) * kHeadTile + (own_lane & 15), group - 1);
      const char* row = (const char*)a.q + (int64_t)b * a.ldq + ((int64_t)h * group + head) * D * (int)sizeof(X);
#pragma unroll
      for (int c = 0; c < KL; ++c)
#pragma unroll
        for (int l = 0; l < QL; ++l)
          raw[nt][c][l] = *(const u32x4*)(row + min(((own_lane >> 4) * KL + c) * 8, D - 8) * (int)sizeof(X) + 16 * l);
    }

    // a lane's offsets within a block of 16 rows; columns past head_dim lie nowhere
    const int ts = (int)a.c.token_stride;
    const int key_off = quad * KL * 8 < D ? col * ts + quad * KL * 4 : kNowhere;
    const int key_scale = quad * KL * 8 < D ? col * ts + D / 2 + quad * KL : kNowhere;
    uint32_t there[KL];                         // all bits of the dwords of the row, none past it
#pragma unroll
    for (int c = 0; c < KL; ++c) there[c] = (quad * KL + c) * 8 < D ? ~0u : 0u;
    int value_off[NV], value_scale[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int d = (16 * v + col) * EV;
      value_off[v] = d < D ? 4 * quad * ts + d / 2 : kNowhere;
      value_scale[v] = d < D ? 4 * quad * ts + D / 2 + d / 8 : kNowhere;
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
    uint32_t key[F::kSub][KL], key_e[F::kSub][(KL + 3) / 4];
    auto load_keys = [&](const Block* k) {
#pragma unroll
      for (int s = 0; s < F::kSub; ++s) {
        const __amdgpu_buffer_rsrc_t r = rows_rsrc(a.c.k + k[s].base, k[s].valid * ts);
        if constexpr (KL == 2) {
          const u32x2 w = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(r, key_off, 0, kPolicy));
          key[s][0] = w[0];
          key[s][1] = w[1];
          key_e[s][0] = __builtin_amdgcn_raw_buffer_load_b16(r, key_scale, 0, kPolicy);
        } else {
#pragma unroll
          for (int c = 0; c < KL / 4; ++c) {
            // (of 256: the second 16 bytes may lie past the row)
            const bool in = quad * KL * 8 + 32 * c < D;
            const u32x4 w = __builtin_bit_cast(
                u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, c == 0 || in ? key_off + 16 * c : kNowhere, 0, kPolicy));
#pragma unroll
            for (int i = 0; i < 4; ++i) key[s][4 * c + i] = w[i];
            key_e[s][c] = __builtin_amdgcn_raw_buffer_load_b32(r, c == 0 || in ? key_scale + 4 * c : kNowhere, 0, kPolicy);
          }
        }
      }
    };
    constexpr int kStep = F::kTokens * kWaves;
    const int first = t0 + F::kTokens * wave;
    Block cur[F::kSub];
#pragma unroll
    for (int s = 0; s < F::kSub; ++s) cur[s] = block_at(first + 16 * s);
    uint32_t value[F::kRows][NV], value_e[F::kRows][NV];
    auto load_values = [&](const Block* k) {
#pragma unroll
      for (int s = 0; s < F::kSub; ++s) {
        const __amdgpu_buffer_rsrc_t r = rows_rsrc(a.c.v + k[s].base, k[s].valid * ts);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int v = 0; v < NV; ++v) {
            if constexpr (EV == 8) value[4 * s + i][v] = __builtin_amdgcn_raw_buffer_load_b32(r, value_off[v] + i * ts, 0, kPolicy);
            else value[4 * s + i][v] = __builtin_amdgcn_raw_buffer_load_b16(r, value_off[v] + i * ts, 0, kPolicy);
            value_e[4 * s + i][v] = __builtin_amdgcn_raw_buffer_load_b8(r, value_scale[v] + i * ts, 0, kPolicy);
          }
      }
    };
    load_keys(cur);
    load_values(cur);

    // Queries, in parts: every wave reads them and writes a share.
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int head = (tile0 + nt) * kHeadTile + (own_lane & 15);
#pragma unroll
      for (int c = 0; c < KL; ++c) {
        if (c % kWaves != wave) continue;
        const bool in = head < group && ((own_lane >> 4) * KL + c) * 8 < D;
        Frag f[PARTS];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          constexpr int PER = 16 / (int)sizeof(X);
          const Chunk<X> v = __builtin_bit_cast(Chunk<X>, raw[nt][c][e / PER]);
          __bf16 part[PARTS];
          split_query<PARTS>(in ? (float)v.e[e % PER] : 0.0f, part);
#pragma unroll
          for (int s = 0; s < PARTS; ++s) f[s][e] = part[s];
        }
#pragma unroll
        for (int s = 0; s < PARTS; ++s) shared.in.query[nt][s][c][own_lane] = f[s];
      }
    }
    lds_barrier();                                // leaves keys and values under way

    f32x4 acc[NT][NV][EV];
    float top[NT], base[NT], sum[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int j = 0; j < EV; ++j) acc[nt][v][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
      top[nt] = -INFINITY;
      base[nt] = sum[nt] = 0.0f;
    }

    // Scores go to memory through LDS, many steps at a time.
    float* scores = wk.scores + ((int64_t)b * a.heads + h * group) * wk.row + 4 * quad;
    const int held_heads = min(group - tile0 * kHeadTile, NT * kHeadTile);
    int holding = 0, held_from = first;           // blocks of 16 tokens, and the first one's step
    auto release = [&]() {
      for (int k = 0; k < holding; ++k)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          const int hd = nt * kHeadTile + col;
          if (hd < held_heads)
            *(f32x4*)(scores + (int64_t)(held_from + k / F::kSub * kStep + k % F::kSub * 16) * group +
                      16 * (tile0 * kHeadTile + hd)) = shared.in.held[wave][4 * held_heads * k + quad * held_heads + hd];
        }
      held_from += holding / F::kSub * kStep;
      holding = 0;
    };

    for (int t = first; t < t1; t += kStep) {
      asm volatile("" ::: "memory");              // the queries stay in LDS
      Block next[F::kSub];
#pragma unroll
      for (int s = 0; s < F::kSub; ++s) next[s] = block_at(t + kStep + 16 * s);

      Frag kf[F::kSub][KL];
#pragma unroll
      for (int s = 0; s < F::kSub; ++s)
#pragma unroll
        for (int c = 0; c < KL; ++c) {
          const uint32_t e = key_e[s][c / 4] >> 8 * (c % 4) & 0xFFu & there[c];
          u32x4 w;
          e2m1_decode(key[s][c] & there[c], e2m1_scale(e), (uint32_t*)&w);
          kf[s][c] = __builtin_bit_cast(Frag, w);
        }
      load_keys(next);

      float p[NT][F::kRows], tile_top[NT];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        f32x4 dot[F::kSub];
#pragma unroll
        for (int s = 0; s < F::kSub; ++s) dot[s] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int part = PARTS - 1; part >= 0; --part)             // small terms first
#pragma unroll
          for (int c = 0; c < KL; ++c) {
            const Frag q = shared.in.query[nt][part][c][lane];
#pragma unroll
            for (int s = 0; s < F::kSub; ++s) dot[s] = mul(kf[s][c], q, dot[s]);
          }
        tile_top[nt] = -INFINITY;
#pragma unroll
        for (int s = 0; s < F::kSub; ++s)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            p[nt][4 * s + i] = 4 * quad + i < cur[s].valid ? dot[s][i] * a.scale_log2 : -INFINITY;
            tile_top[nt] = fmaxf(tile_top[nt], p[nt][4 * s + i]);
          }
      }
      if (a.accumulate) {
        if (4 * held_heads * (holding + F::kSub) > kHold) release();
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int s = 0; s < F::kSub; ++s) {
            const int hd = nt * kHeadTile + col;
            if (hd < held_heads)
              shared.in.held[wave][4 * held_heads * (holding + s) + quad * held_heads + hd] =
                  f32x4{p[nt][4 * s], p[nt][4 * s + 1], p[nt][4 * s + 2], p[nt][4 * s + 3]};
          }
        holding += F::kSub;
      }

      Frag pf[NT][WPARTS];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        if (__any(tile_top[nt] > top[nt] + F::kSlack)) {
          const float now = fmaxf(top[nt], head_max(tile_top[nt]));
          const float rescaled = now == -INFINITY ? 0.0f : now;
          const float f = top[nt] == -INFINITY ? 0.0f : exp2_fast(base[nt] - rescaled);
          sum[nt] *= f;
#pragma unroll
          for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int j = 0; j < EV; ++j) acc[nt][v][j] *= f;
          top[nt] = now;
          base[nt] = rescaled;
        }
#pragma unroll
        for (int i = 0; i < F::kRows; ++i) {
          const float w = exp2_fast(p[nt][i] - base[nt]);
          sum[nt] += w;
          __bf16 part[WPARTS];
          split<__bf16, WPARTS>(w, part);
#pragma unroll
          for (int s = 0; s < WPARTS; ++s) pf[nt][s][i] = part[s];
        }
      }

#pragma unroll
      for (int v = 0; v < NV; ++v) {
        uint32_t x[F::kRows][EV / 2];               // pairs of a token's columns
#pragma unroll
        for (int i = 0; i < F::kRows; ++i) {
          const float s = e2m1_scale(value_e[i][v]);
          if constexpr (EV == 8) {
            e2m1_decode(value[i][v], s, x[i]);
          } else {
            x[i][0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(value[i][v], s, 0));
            x[i][1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(value[i][v], s, 1));
          }
        }
#pragma unroll
        for (int j = 0; j < EV; ++j) {
          u32x4 w;                                  // tokens of a column
#pragma unroll
          for (int i = 0; i < 4; ++i)
            w[i] = __builtin_amdgcn_perm(x[2 * i + 1][j / 2], x[2 * i][j / 2], j % 2 ? 0x07060302u : 0x05040100u);
          const Frag vf = __builtin_bit_cast(Frag, w);
#pragma unroll
          for (int part = WPARTS - 1; part >= 0; --part)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) acc[nt][v][j] = mul(vf, pf[nt][part], acc[nt][v][j]);
        }
      }
#pragma unroll
      for (int s = 0; s < F::kSub; ++s) cur[s] = next[s];
      load_values(cur);
    }
    if (a.accumulate) release();

    // join the waves
    asm volatile("" : "+v"(own_lane));
    const int own_col = own_lane & 15, own_quad = own_lane >> 4;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const float all = head_sum(sum[nt]);
      if (own_quad == 0) {
        stat[nt][wave][own_col][0] = top[nt] == -INFINITY ? -INFINITY : base[nt];
        stat[nt][wave][own_col][1] = all;
      }
    }
    const int chunks = D / 4;
    const int64_t slot = u + b;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      __syncthreads();
      {
        float common = -INFINITY;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) common = fmaxf(common, stat[nt][w][own_col][0]);
        const float f = top[nt] == -INFINITY ? 0.0f : exp2_fast(base[nt] - common);
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < EV; j += 4)
              *(f32x4*)&shared.slab[wave][own_col][(16 * v + 4 * own_quad + i) * EV + j] =
                  f32x4{acc[nt][v][j][i], acc[nt][v][j + 1][i], acc[nt][v][j + 2][i], acc[nt][v][j + 3][i]} * f;
      }
      __syncthreads();
      const int g0 = (tile0 + nt) * kHeadTile, live = min(group - g0, kHeadTile);
      for (int k = 64 * wave + own_lane; k < live * chunks; k += 64 * kWaves) {
        const int hd = k / chunks, c = k - hd * chunks;
        f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
        float common = -INFINITY, weight = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
          o += *(const f32x4*)&shared.slab[w][hd][4 * c];
          common = fmaxf(common, stat[nt][w][hd][0]);
        }
#pragma unroll
        for (int w = 0; w < kWaves; ++w)
          weight += stat[nt][w][hd][0] == -INFINITY ? stat[nt][w][hd][1]
                                                    : stat[nt][w][hd][1] * exp2_fast(stat[nt][w][hd][0] - common);
        const int64_t row = slot * a.heads + h * group + g0 + hd;
        *(f32x4*)(wk.part + row * D + 4 * c) = o;
        if (c == 0) {
          wk.stat[2 * row] = common;
          wk.stat[2 * row + 1] = weight;
        }
      }
    }

    // on to the next sequence of this share
    at = before + steps;
    if (at >= stop) return;
    __syncthreads();                              // the outputs are read
    before = at;
    do {
      if (++b >= a.c.batch) return;
    } while (held_tokens_uniform(a.lengths, b, a.max_len) == 0);
  }
}

template <int XT, int DP>
void launch_tiles(const AttendLaunch& a, const Work& w, const Plan& p, hipStream_t s) {
  const int64_t shares = (int64_t)a.c.kv_heads * p.workgroups;
  const dim3 grid(kXcds * p.tile_groups, (unsigned)((shares + kXcds - 1) / kXcds)), block(64 * kWaves);
  if constexpr (DP < 256) {
    if (p.wave_tiles == 2) {
      if (p.tile_groups == 1) cache_attend_e2m1_kernel<XT, DP, 2, true><<<grid, block, 0, s>>>(a, w, p.workgroups);
      else cache_attend_e2m1_kernel<XT, DP, 2, false><<<grid, block, 0, s>>>(a, w, p.workgroups);
      return;
    }
  } else if (p.tile_groups > 1) {
    cache_attend_e2m1_kernel<XT, DP, 1, false><<<grid, block, 0, s>>>(a, w, p.workgroups);
    return;
  }
  cache_attend_e2m1_kernel<XT, DP, 1, true><<<grid, block, 0, s>>>(a, w, p.workgroups);
}

template <int XT>
hipError_t launch_types(const AttendLaunch& a, hipStream_t s) {
  const Plan p = plan_of(a.c, a.heads, a.max_len);
  const Work w = work_of(a, p);
  if (a.c.head_dim <= 64) launch_tiles<XT, 64>(a, w, p, s);
  else if (a.c.head_dim <= 128) launch_tiles<XT, 128>(a, w, p, s);
  else launch_tiles<XT, 256>(a, w, p, s);
  launch_join<XT>(a, w, p, s);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_cache_attend_e2m1(const AttendLaunch& a, hipStream_t s) {
  if (a.x_dtype == MOSAIC_F32) return launch_types<MOSAIC_F32>(a, s);
  if (a.x_dtype == MOSAIC_BF16) return launch_types<MOSAIC_BF16>(a, s);
  return launch_types<MOSAIC_F16>(a, s);
}

}  // namespace mosaic
