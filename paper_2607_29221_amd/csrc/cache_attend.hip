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
// * Over a 16-bit cache, float32 queries and all weights are split into 16-bit
//   parts that are multiplied one after the other into the same sums. Three of
//   bf16 (float32 activations) hold all 24 bits. Two of f16, the range centred,
//   leave out at most 2^-23 of a number, less than the sums' own rounding, and two
//   of bf16 (16-bit activations) at most 2^-17 of a weight: a five hundredth
//   of what rounding the output to bf16 leaves out of it.
//   The matrix cores have room for it (busy 14% of the time at full bandwidth
//   with three parts): 64 sequences take 165 us with bf16, 164 us with float32.
// * M is raised, and O rescaled, only when a score passes it by more than
//   kSlack: sums of up to 2^kSlack are as exact as sums of up to 1.
// * All tokens of a key/value head, one sequence after the other, are cut into
//   equal shares, one per workgroup, from the lengths that the device holds: a
//   workgroup takes part of one sequence or several. A second kernel joins the
//   parts, and adds up attention weights from the scores that the first one
//   left in the workspace.
#include <cfloat>
#include <type_traits>

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

template <class T> struct Chunk { T e[16 / sizeof(T)]; };

// Every wave's writes to LDS before every wave's reads after; memory accesses
// go on (a __syncthreads waits for those too).
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// What the types of cache and activations make of a wave's step. DP: head_dim
// padded to 64, 128 or 256 (columns beyond head_dim are zeros).
template <int CT, int XT, int DP> struct Form {
  typedef typename FloatType<CT>::type C;
  typedef typename FloatType<XT>::type X;
  static constexpr bool kWide = CT == MOSAIC_F32;
  // 16-bit numbers that make up a query's element (one if it is one) and a
  // weight (16-bit activations: enough that the output's rounding is the larger)
  static constexpr int kParts = kWide || XT != MOSAIC_F32 ? 1 : CT == MOSAIC_BF16 ? 3 : 2;
  static constexpr int kWeightParts = kWide ? 1 : XT != MOSAIC_F32 || CT == MOSAIC_F16 ? 2 : 3;
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

// Two 16-bit numbers of a cache, 0 in place of an infinity or NaN.
template <int CT> __device__ __forceinline__ uint32_t finite_pair(uint32_t w) {
  constexpr uint32_t kExponent = CT == MOSAIC_BF16 ? 0x7F80u : 0x7C00u;
  return ((w & kExponent) == kExponent ? 0u : w & 0xFFFFu) |
         ((w & kExponent << 16) == kExponent << 16 ? 0u : w & 0xFFFF0000u);
}

// x as the sum of PARTS 16-bit numbers, each rounded from what the ones before leave.
template <class T, int PARTS>
__device__ __forceinline__ void split(float x, T* part) {
#pragma unroll
  for (int s = 0; s < PARTS; ++s) {
    part[s] = (T)x;
    x -= (float)part[s];
  }
}

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

Plan plan_of(const CacheView& c, int32_t heads, int64_t max_len) {
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
  // would idle (71 heads: 217 us with 213, 186 us with 497).
  int32_t slots = p.tile_groups > 1 && c.head_dim <= 128 ? 512 : 256;
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

// Steps of sequence i, 0 beyond the batch.
__device__ __forceinline__ int steps_of(const AttendLaunch& a, int i) {
  return i < a.c.batch ? (held_tokens(a.lengths, i, a.max_len) + kStepTokens - 1) / kStepTokens : 0;
}
// Steps of the first 64 sequences, a lane each: its own, and all up to it.
struct FirstSteps {
  int own, upto;
};
// Steps of all sequences, by one wave.
__device__ __forceinline__ int all_steps(const AttendLaunch& a, int lane, FirstSteps* first) {
  first->own = steps_of(a, lane);
  first->upto = wave_scan(first->own);
  int total = __builtin_amdgcn_readlane(first->upto, 63);
  for (int i0 = 64; i0 < a.c.batch; i0 += 64) total += __builtin_amdgcn_readlane(wave_scan(steps_of(a, i0 + lane)), 63);
  return total;
}
// Steps of the sequences before b.
__device__ __forceinline__ int steps_before(const AttendLaunch& a, int lane, int b, const FirstSteps& first) {
  if (b < 64) return __builtin_amdgcn_readlane(first.upto - first.own, b);
  int carry = __builtin_amdgcn_readlane(first.upto, 63);
  for (int i0 = 64; ; i0 += 64) {
    const int own = steps_of(a, i0 + lane), upto = wave_scan(own);
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
    own = steps_of(a, i0 + lane);
    upto = wave_scan(own);
  }
}

// Waves per SIMD that the registers are held to: one is enough for a call of
// its own, more let it share the chip.
constexpr int waves_of(int DP, int NT) { return DP == 256 ? 1 : (DP == 128 ? 3 : 4) - (NT - 1); }

// NT: blocks of 16 query heads per wave (64 query heads on one key/value head
// of 128 elements, 64 sequences: 111 us with one, 75 us with two; four would
// leave the registers one wave per SIMD).
// STREAM: no other workgroup reads the same keys and values, so they pass by
// the caches (131072 tokens: 92 us through them, 80 us past them); where
// several do (groups of more than 32 heads) they go through (the 64 heads: 75
// us, 88 us past).
// Measured on an MI355X, this kernel alone, heads of 128 elements, 64 query
// and 8 key/value heads: 131072 tokens of one sequence 80 us (6.7 TB/s of keys
// and values); 64 sequences of 512 to 7168 tokens 161 us (6.4 TB/s); 32 heads
// of each, float32 cache, 122 us (6.2 TB/s); 1024 tokens 7 us, the latency of
// its chain of loads. With weights the 64 sequences take 217 us: storing 63 MB
// of scores costs several times their share of the traffic, whether one
// step's or many steps' are stored at a time, past the caches or through them.
// Loads that wait behind a wave's stores, with one wave per SIMD and nothing
// to cover the wait, would explain it; that is not shown.
template <int CT, int XT, int DP, int NT, bool STREAM>
__global__ __launch_bounds__(64 * kWaves, waves_of(DP, NT)) void cache_attend_kernel(AttendLaunch a, Work wk, int32_t workgroups) {
  typedef Form<CT, XT, DP> F;
  typedef typename F::C C;
  typedef typename F::X X;
  typedef Matrix<CT> M;
  typedef typename M::Frag Frag;
  constexpr int E = F::kWide ? 4 : 8;           // elements of a 16-byte key chunk
  constexpr int KL = F::kKeyLoads, NV = F::kValueLoads, EV = F::kEach, PARTS = F::kParts, WPARTS = F::kWeightParts;
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

    // What only the start and the end of a part need is computed there: kept
    // in registers through the steps it would cost a wave per SIMD.
    int own_lane = lane;
    asm volatile("" : "+v"(own_lane));

    // the queries, asked for first (loads come back in order); lanes without a
    // head or column read another's
    constexpr int QL = E * (int)sizeof(X) / 16;   // loads per chunk
    u32x4 raw[NT][KL][QL];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int head = min((tile0 + nt) * kHeadTile + (own_lane & 15), group - 1);
      const char* row = (const char*)a.q + (int64_t)b * a.ldq + ((int64_t)h * group + head) * D * (int)sizeof(X);
#pragma unroll
      for (int c = 0; c < KL; ++c)
#pragma unroll
        for (int l = 0; l < QL; ++l)
          raw[nt][c][l] = *(const u32x4*)(row + min((4 * c + (own_lane >> 4)) * E, D - E) * (int)sizeof(X) + 16 * l);
    }

    // a lane's offsets within a block of 16 rows; columns past head_dim lie nowhere
    const int ts = (int)a.c.token_stride;
    int key_off[KL], value_off[NV];
#pragma unroll
    for (int c = 0; c < KL; ++c) key_off[c] = (4 * c + quad) * E < D ? col * ts + (4 * c + quad) * 16 : kNowhere;
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
    Frag key[F::kSub][KL];
    auto load_keys = [&](const Block* k) {
#pragma unroll
      for (int s = 0; s < F::kSub; ++s) {
        const __amdgpu_buffer_rsrc_t r = rows_rsrc(a.c.k + k[s].base, k[s].valid * ts);
#pragma unroll
        for (int c = 0; c < KL; ++c)
          key[s][c] = __builtin_bit_cast(Frag, __builtin_amdgcn_raw_buffer_load_b128(r, key_off[c], 0, kPolicy));
      }
    };
    constexpr int kStep = F::kTokens * kWaves;
    const int first = t0 + F::kTokens * wave;
    Block cur[F::kSub];
#pragma unroll
    for (int s = 0; s < F::kSub; ++s) cur[s] = block_at(first + 16 * s);
    // values of these tokens
    u32x4 value[F::kRows][NV];
    auto load_values = [&](const Block* k) {
#pragma unroll
      for (int s = 0; s < F::kSub; ++s) {
        const __amdgpu_buffer_rsrc_t r = rows_rsrc(a.c.v + k[s].base, k[s].valid * ts);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int v = 0; v < NV; ++v) {
            if (EV * sizeof(C) == 16) {
              value[4 * s + i][v] =
                  __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, value_off[v] + i * ts, 0, kPolicy));
            } else {
              const u32x2 w =
                  __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(r, value_off[v] + i * ts, 0, kPolicy));
              value[4 * s + i][v] = u32x4{w[0], w[1], 0u, 0u};
            }
          }
      }
    };
    load_keys(cur);
    load_values(cur);

    // Queries, in parts: every wave reads them (the scale is a lane's own) and
    // writes a share.
    float scale[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int head = (tile0 + nt) * kHeadTile + (own_lane & 15);
      float x[KL][E];
      float top = 0.0f;
#pragma unroll
      for (int c = 0; c < KL; ++c) {
        const bool there = head < group && (4 * c + (own_lane >> 4)) * E < D;
#pragma unroll
        for (int e = 0; e < E; ++e) {
          constexpr int PER = 16 / (int)sizeof(X);
          const Chunk<X> v = __builtin_bit_cast(Chunk<X>, raw[nt][c][e / PER]);
          x[c][e] = there ? (float)v.e[e % PER] : 0.0f;
          top = fmaxf(top, fminf(fabsf(x[c][e]), FLT_MAX));
        }
      }
      int up = 0;
      if (CT == MOSAIC_F16 && XT == MOSAIC_F32) {
        // by a power of two into the upper part of the range of f16
        top = head_max(top);
        up = top > 0.0f ? 14 - __builtin_amdgcn_frexp_expf(top) : 0;
      }
      scale[nt] = ldexpf(a.scale_log2, -up);
#pragma unroll
      for (int c = 0; c < KL; ++c) {
        if (c % kWaves != wave) continue;
        Frag f[PARTS];
#pragma unroll
        for (int e = 0; e < E; ++e) {
          C part[PARTS];
          split<C, PARTS>(CT == MOSAIC_F16 && XT == MOSAIC_F32 ? ldexpf(x[c][e], up) : x[c][e], part);
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

    // Scores go to memory through LDS, many steps at a time: a load that is
    // issued behind a store waits for it, and stores take longer than loads.
    float* scores = wk.scores + ((int64_t)b * a.heads + h * group) * wk.row + 4 * quad;
    const int held_heads = min(group - tile0 * kHeadTile, NT * kHeadTile);
    int holding, held_from;                       // blocks of 16 tokens, and the first one's step
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

    // All steps of the part. Where a key, query or value holds an infinity, its
    // products with the parts of the other (small ones of either sign, and zeros)
    // can add up to NaN although the sum is infinite: `careful` takes such a score
    // from the first parts alone, which have the signs of the whole, and gives
    // such a value to the first parts only. That is a second pass, for waves that
    // found NaN: no step of the first has a check for it.
    auto pass = [&](auto careful) __attribute__((always_inline)) {
      constexpr bool kCareful = decltype(careful)::value;
      holding = 0;
      held_from = first;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
          for (int j = 0; j < EV; ++j) acc[nt][v][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        top[nt] = -INFINITY;
        base[nt] = sum[nt] = 0.0f;
      }
      for (int t = first; t < t1; t += kStep) {
        asm volatile("" ::: "memory");              // the queries stay in LDS
        Block next[F::kSub];
#pragma unroll
        for (int s = 0; s < F::kSub; ++s) next[s] = block_at(t + kStep + 16 * s);

        float p[NT][F::kRows], tile_top[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          f32x4 dot[F::kSub];
#pragma unroll
          for (int s = 0; s < F::kSub; ++s) dot[s] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
          for (int part = PARTS - 1; part >= 0; --part)           // small terms first
#pragma unroll
            for (int c = 0; c < KL; ++c) {
              const Frag q = shared.in.query[nt][part][c][lane];
#pragma unroll
              for (int s = 0; s < F::kSub; ++s) dot[s] = M::mul(key[s][c], q, dot[s]);
            }
          if constexpr (kCareful && PARTS > 1) {
            f32x4 first_part[F::kSub];
#pragma unroll
            for (int s = 0; s < F::kSub; ++s) first_part[s] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int c = 0; c < KL; ++c)
#pragma unroll
              for (int s = 0; s < F::kSub; ++s)
                first_part[s] = M::mul(key[s][c], shared.in.query[nt][0][c][lane], first_part[s]);
#pragma unroll
            for (int s = 0; s < F::kSub; ++s)
#pragma unroll
              for (int i = 0; i < 4; ++i) dot[s][i] = dot[s][i] == dot[s][i] ? dot[s][i] : first_part[s][i];
          }
          tile_top[nt] = -INFINITY;
#pragma unroll
          for (int s = 0; s < F::kSub; ++s)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              p[nt][4 * s + i] = 4 * quad + i < cur[s].valid ? dot[s][i] * scale[nt] : -INFINITY;
              tile_top[nt] = fmaxf(tile_top[nt], p[nt][4 * s + i]);
            }
        }
        load_keys(next);
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
            const float rescaled = now == -INFINITY ? 0.0f : now - F::kShift;
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
            C part[WPARTS];
            split<C, WPARTS>(w, part);
            if constexpr (kCareful && CT == MOSAIC_F16) {
              // a weight that no part holds is none for a finite value, but not for an infinite one
              constexpr float kLeast = 0x1p-24f;
              if (w > 0.0f && part[0] == (C)0.0f) {
                part[0] = (C)kLeast;
                part[1] = (C)-kLeast;
              }
            }
#pragma unroll
            for (int s = 0; s < WPARTS; ++s) pf[nt][s][i] = part[s];
          }
        }

#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
          for (int j = 0; j < EV; ++j) {
            Frag vf, rest;                          // for the first part of the weights, and for the others
            if constexpr (F::kWide) {
#pragma unroll
              for (int i = 0; i < 4; ++i) vf[i] = __uint_as_float(value[i][v][j]);
              rest = vf;
            } else {
              u32x4 w;
#pragma unroll
              for (int i = 0; i < 4; ++i)
                w[i] = __builtin_amdgcn_perm(value[2 * i + 1][v][j / 2], value[2 * i][v][j / 2],
                                             j % 2 ? 0x07060302u : 0x05040100u);
              vf = __builtin_bit_cast(Frag, w);
              if constexpr (kCareful) {
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] = finite_pair<CT>(w[i]);
              }
              rest = __builtin_bit_cast(Frag, w);
            }
#pragma unroll
            for (int part = WPARTS - 1; part >= 0; --part)
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) acc[nt][v][j] = M::mul(part > 0 ? rest : vf, pf[nt][part], acc[nt][v][j]);
          }
#pragma unroll
        for (int s = 0; s < F::kSub; ++s) cur[s] = next[s];
        load_values(cur);
      }
      if (a.accumulate) release();
    };
    pass(std::false_type());
    if constexpr (WPARTS > 1) {
      f32x4 most = acc[0][0][0];                    // NaN if any is
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        most[0] = __builtin_elementwise_maximum(most[0], sum[nt]);
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
          for (int j = 0; j < EV; ++j) most = __builtin_elementwise_maximum(most, acc[nt][v][j]);
      }
      if (__any(__builtin_isunordered(most[0], most[1]) || __builtin_isunordered(most[2], most[3]))) {
#pragma unroll
        for (int s = 0; s < F::kSub; ++s) cur[s] = block_at(first + 16 * s);
        load_keys(cur);
        load_values(cur);
        pass(std::true_type());
      }
    }

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
  const int total = all_steps(a, lane, &first64), share = max((total + workgroups - 1) / workgroups, 1);
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

template <int CT, int XT, int DP>
void launch_tiles(const AttendLaunch& a, const Work& w, const Plan& p, hipStream_t s) {
  const int64_t shares = (int64_t)a.c.kv_heads * p.workgroups;
  const dim3 grid(kXcds * p.tile_groups, (unsigned)((shares + kXcds - 1) / kXcds)), block(64 * kWaves);
  if constexpr (DP < 256) {
    if (p.wave_tiles == 2) {
      if (p.tile_groups == 1) cache_attend_kernel<CT, XT, DP, 2, true><<<grid, block, 0, s>>>(a, w, p.workgroups);
      else cache_attend_kernel<CT, XT, DP, 2, false><<<grid, block, 0, s>>>(a, w, p.workgroups);
      return;
    }
  } else if (p.tile_groups > 1) {
    cache_attend_kernel<CT, XT, DP, 1, false><<<grid, block, 0, s>>>(a, w, p.workgroups);
    return;
  }
  cache_attend_kernel<CT, XT, DP, 1, true><<<grid, block, 0, s>>>(a, w, p.workgroups);
}

template <int CT, int XT>
hipError_t launch_types(const AttendLaunch& a, hipStream_t s) {
  const Plan p = plan_of(a.c, a.heads, a.max_len);
  Work w;
  w.stat = (float*)a.workspace;
  w.part = w.stat + stat_floats(a.c, a.heads, p);
  w.scores = w.part + part_floats(a.c, a.heads, p);
  w.row = padded_len(a.max_len);
  if (a.c.head_dim <= 64) launch_tiles<CT, XT, 64>(a, w, p, s);
  else if (a.c.head_dim <= 128) launch_tiles<CT, XT, 128>(a, w, p, s);
  else launch_tiles<CT, XT, 256>(a, w, p, s);
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
  return hipGetLastError();
}

}  // namespace

int64_t cache_attend_workspace(const CacheView& c, int32_t heads, int64_t max_len, int32_t accumulate) {
  const Plan p = plan_of(c, heads, max_len);
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
