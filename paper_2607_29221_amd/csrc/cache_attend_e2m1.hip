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
// * Rows of 80 bytes (of 128 elements) make small pieces of codes and scales. They
//   come to LDS whole, 16 bytes per lane, past the caches: read piece by piece from
//   memory, the same lines were asked for several times (131072 tokens 45 us, 40 us
//   through the caches, 35 us by way of LDS). A wave has two stages of 32 tokens
//   and waits for its own loads only.
// * Keys: the 16 lanes of a quarter take one token each, a quarter of its row:
//   dwords of codes and as many scale bytes lie side by side. The inner
//   dimension's order differs from the elements' by that, in the queries too.
// * Values: a lane takes the same 8 columns (4 where head_dim is at most 64) of
//   8 tokens, a dword of codes and a scale byte each, and turns them with byte
//   permutes once they are bf16.
//
// Measured on an MI355X with the join, heads of 128 elements: 131072 tokens of one
// sequence, 32 query and 8 key/value heads, bf16, 35 us, 29 to 31 us in this kernel
// (168 MB: 5.4 to 5.8 TB/s); 64 sequences of 512 to 7168 tokens, 64 and 8 heads,
// bf16 61 us, float32 67 to 75 us (315 MB: 5.6 and 4.5 to 4.8 TB/s in this kernel).
// What is left above the bandwidth: without the arithmetic the 64 sequences (float32)
// take 62 of 75 us, without the rows past a part's first steps 68; a part of a sequence
// starts with 3.5 to 5.5 us of dependent loads, and about 200 vector instructions
// per 32 tokens and wave leave the two waves of a SIMD little room.
#include <cfloat>
#include <type_traits>

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

// Rows come to LDS as they lie, 16 bytes per lane and load: lane l of the wave
// writes LDS bytes [to + 16 l, to + 16 l + 16), zeros for what lies past the
// descriptor's range. In assembly, so that the compiler does not wait for all
// loads before each read of LDS; a wave waits for its own with landed().
// Nothing else in this kernel uses M0.
typedef int v4i __attribute__((ext_vector_type(4)));
template <bool STREAM> __device__ __forceinline__ void row_load(v4i rsrc, uint32_t to, int off) {
  if constexpr (STREAM)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen nt lds" ::"s"(to), "v"(off), "s"(rsrc) : "memory");
  else
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(to), "v"(off), "s"(rsrc) : "memory");
}
// At most N of the wave's vector-memory accesses are under way.
template <int N> __device__ __forceinline__ void landed() {
  static_assert(N < 64, "the counter's range");
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

constexpr int waves_of(int DP) { return DP == 256 ? 1 : 2; }

// Weights as bf16 parts, two to a dword.
template <int PARTS> __device__ __forceinline__ void split_pair(float x, float y, uint32_t* part) {
#pragma unroll
  for (int s = 0; s < PARTS; ++s) {
    bf16x2 r;
    r[0] = (__bf16)x;
    r[1] = (__bf16)y;
    part[s] = __builtin_bit_cast(uint32_t, r);
    x -= __uint_as_float(part[s] << 16);
    y -= __uint_as_float(part[s] & 0xFFFF0000u);
  }
}

// The value N columns further on, of 16 that come round.
template <int N> __device__ __forceinline__ float other_column(float v) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), 0x120 + N, 0xF, 0xF, true));
}

// Bytes of LDS: operands of the first product by lane; the waves' stages of rows;
// where weights are added up, scores on their way to memory. The waves' outputs
// come over these at the end.
template <int XT, int DP, int NT, int W> struct Lds {
  typedef Form<XT, DP> F;
  static constexpr int kSlots = kHeadTile / W;  // parts of a head, side by side
  static constexpr int kPasses = (F::kParts + kSlots - 1) / kSlots, kWeightPasses = (F::kWeightParts + kSlots - 1) / kSlots;
  static constexpr int kStages = 2;             // of a wave, kTokens rows of keys and of values each
  static constexpr int kStageBytes = 2 * F::kTokens * MOSAIC_E2M1_ROW_BYTES(DP);
  static constexpr int kQuery = NT * kPasses * F::kKeyDwords * 64 * 16;
  static constexpr int kRows = kWaves * kStages * kStageBytes;
  static constexpr int kPast = 256;             // columns past head_dim are read from what follows a row
  static constexpr int kHold = 128 * NT;        // of a wave's scores, 16 bytes each: one step's at least
  static constexpr int kSlab = kWaves * kHeadTile * (DP + 4) * 4;
  static constexpr int bytes(bool accumulate) {
    const int in = kQuery + kRows + kPast + (accumulate ? kWaves * kHold * 16 : 0);
    return in > kSlab ? in : kSlab;
  }
  static constexpr int kStat = NT * kWaves * kHeadTile * 8;
  static constexpr bool two_fit(bool accumulate) { return 2 * (bytes(accumulate) + kStat) <= 160 * 1024; }
};

// Whether a unit holds two workgroups of a call (parts side by side take less LDS).
template <int XT, int DP> bool two_fit(const AttendLaunch& a) {
  return a.heads / a.c.kv_heads > kHeadTile ? Lds<XT, DP, 2, 16>::two_fit(a.accumulate) : Lds<XT, DP, 1, 16>::two_fit(a.accumulate);
}

// NT: blocks of 16 query heads per wave. W: where a group has at most 8 or 4
// heads, columns W, 2W, ... of a block hold further parts of the heads in the first
// W, so that a product takes several parts at a time. FULL: head_dim is DP.
// STREAM: past the caches, as no other workgroup reads the same rows.
template <int XT, int DP, int NT, int W, bool FULL, bool STREAM>
__global__ __launch_bounds__(64 * kWaves, waves_of(DP)) void cache_attend_e2m1_kernel(AttendLaunch a, Work wk, int32_t workgroups) {
  typedef Form<XT, DP> F;
  typedef Lds<XT, DP, NT, W> S;
  typedef typename F::X X;
  typedef bf16x8 Frag;
  constexpr int KL = F::kKeyDwords, NV = F::kValuePieces, EV = F::kEach, PARTS = F::kParts, WPARTS = F::kWeightParts;
  constexpr int R = S::kSlots, PASSES = S::kPasses, WPASSES = S::kWeightPasses;
  constexpr int kHold = S::kHold, kStages = S::kStages, kStageBytes = S::kStageBytes;
  constexpr int kMostLoads = (2 * MOSAIC_E2M1_ROW_BYTES(DP) / 16 + 3) / 4;   // per 32 rows
  extern __shared__ __attribute__((aligned(16))) char lds[];
  __shared__ float stat[NT][kWaves][kHeadTile][2];
  Frag(*query)[PASSES][KL][64] = (Frag(*)[PASSES][KL][64])lds;
  float(*slab)[kHeadTile][DP + 4] = (float(*)[kHeadTile][DP + 4])lds;

  const int tid = threadIdx.x, lane = tid & 63, col = lane & 15, quad = lane >> 4, slot_of_col = col / W;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const char* const rows = lds + S::kQuery + wave * kStages * kStageBytes;
  f32x4* const held = (f32x4*)(lds + S::kQuery + S::kRows + S::kPast) + wave * kHold;
  const uint32_t share_of = blockIdx.y * kXcds + blockIdx.x % kXcds;
  const int u = share_of / (uint32_t)a.c.kv_heads, h = share_of - u * a.c.kv_heads;
  const int tile0 = blockIdx.x / kXcds * NT;
  if (u >= workgroups) return;
  const int group = a.heads / a.c.kv_heads, D = FULL ? DP : a.c.head_dim;

  int before, total;
  FirstSteps first64;
  const int share = share_of_steps(a, lane, workgroups, true, &first64, &total);
  int at = u * share;
  const int stop = min(total, at + share);
  if (at >= stop) return;
  int b = sequence_at(a, lane, at, first64, &before);
  if (b < 0) return;
  while (true) {
    const int n = held_tokens_uniform(a.lengths, b, a.max_len), steps = (n + kStepTokens - 1) / kStepTokens;
    if (at - before >= steps) {                   // the share begins behind the sequence's own steps: nothing of it
      at = before + steps + first64.extra;
      if (at >= stop) return;
      before = at;
      do {
        if (++b >= a.c.batch) return;
      } while (held_tokens_uniform(a.lengths, b, a.max_len) == 0);
      continue;
    }
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
      const int head = min((tile0 + nt) * kHeadTile + (own_lane & (W - 1)), group - 1);
      const char* row = (const char*)a.q + (int64_t)b * a.ldq + ((int64_t)h * group + head) * D * (int)sizeof(X);
#pragma unroll
      for (int c = 0; c < KL; ++c)
#pragma unroll
        for (int l = 0; l < QL; ++l)
          raw[nt][c][l] = *(const u32x4*)(row + min(((own_lane >> 4) * KL + c) * 8, D - 8) * (int)sizeof(X) + 16 * l);
    }

    // Offsets of the lane's 16 bytes of a block's rows. 32 rows are a block where
    // they lie in one page, 16 otherwise.
    const int ts = (int)a.c.token_stride, row_bytes = MOSAIC_E2M1_ROW_BYTES(D), pieces = row_bytes / 16;
    const bool wide = a.c.log2_page > 4;
    const int row_loads = wide ? (2 * pieces + 3) / 4 : (pieces + 3) / 4;
    int row_off[kMostLoads];
#pragma unroll
    for (int j = 0; j < kMostLoads; ++j) row_off[j] = (64 * j + lane) / pieces * ts + (64 * j + lane) % pieces * 16;
    // a scale's exponent bits, none of those past the row (codes there meet queries of 0)
    uint32_t there[KL];
#pragma unroll
    for (int c = 0; c < KL; ++c) there[c] = (quad * KL + c) * 8 < D ? 0x7F800000u : 0u;

    // the page of a slot, as the table has it (of a later one than the last, the
    // last one's), and how many tokens of 16 or 32 from there on there are
    const int page_mask = (1 << a.c.log2_page) - 1;
    const uniform_i32 pages = (uniform_i32)(uintptr_t)a.c.table + b * a.c.ldt;
    auto page_at = [&](int slot) { return pages[min(slot, t1 - 1) >> a.c.log2_page]; };
    auto valid_at = [&](int slot, int page, int most) {
      return (uint32_t)page < (uint32_t)a.c.pages ? max(min(t1 - slot, most), 0) : 0;
    };
    const char *const head_k = a.c.k + (int64_t)h * a.c.head_stride, *const head_v = a.c.v + (int64_t)h * a.c.head_stride;
    constexpr int kStep = F::kTokens * kWaves;
    const int first = t0 + F::kTokens * wave;
    // stage after stage into its slot; one without tokens counts as loaded all the same
    const uint32_t stage0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char*)rows;
    // keys and values of `valid` rows from slot t on
    auto load_block = [&](int t, int page, int valid, int count, uint32_t to) {
      const int64_t at = valid > 0 ? (int64_t)page * a.c.page_stride + (t & page_mask) * ts : 0;
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const uint64_t base = (uint64_t)((s == 0 ? head_k : head_v) + at);
        const v4i rsrc = {__builtin_amdgcn_readfirstlane((int)(uint32_t)base),
                          __builtin_amdgcn_readfirstlane((int)((uint32_t)(base >> 32) & 0xFFFFu)),
                          __builtin_amdgcn_readfirstlane(valid * ts), 0x00020000};
#pragma unroll
        for (int j = 0; j < kMostLoads; ++j)
          if (j < row_loads && 64 * j + lane < count * pieces) row_load<STREAM>(rsrc, to + s * F::kTokens * row_bytes + 1024 * j, row_off[j]);
      }
    };
    auto load_rows = [&](int t, const int* page, const int* valid, int slot) {
      const uint32_t to = stage0 + slot * kStageBytes;
      if (wide) {
        load_block(t, page[0], valid[0] + valid[1], 32, to);
      } else {
        load_block(t, page[0], valid[0], 16, to);
        load_block(t + 16, page[1], valid[1], 16, to + 16 * row_bytes);
      }
    };
    auto landed_but_last = [&]() {
      const int n = wide ? 2 * row_loads : 4 * row_loads;
      if (n <= 2) landed<2>();
      else if (n <= 4) landed<4>();
      else if (n <= 6) landed<6>();
      else if (n <= 8) landed<8>();
      else if (n <= 10) landed<10>();
      else landed<12>();
    };
    int page[F::kSub];                          // of the stage after those under way
    int valid[F::kSub], valid_next[F::kSub];    // tokens of the current stage and the one after
    auto pages_at = [&](int t) {
      page[0] = page_at(t);
      page[1] = wide ? page[0] : page_at(t + 16);
    };
    auto count_at = [&](int t, int* n) {
      n[0] = valid_at(t, page[0], 16);
      n[1] = valid_at(t + 16, page[1], 16);
    };
    pages_at(first);
    count_at(first, valid);
    // the queries are waited for here, so that turning them into operands does
    // not wait for rows (loads are counted in order)
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int c = 0; c < KL; ++c)
#pragma unroll
        for (int l = 0; l < QL; ++l) asm volatile("" : "+v"(raw[nt][c][l]));
    load_rows(first, page, valid, 0);
    pages_at(first + kStep);

    // Queries, in parts: every wave reads them and writes a share.
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int head = (tile0 + nt) * kHeadTile + (own_lane & (W - 1)), part0 = (own_lane & 15) / W;
#pragma unroll
      for (int c = 0; c < KL; ++c) {
        if (c % kWaves != wave) continue;
        const bool in = head < group && ((own_lane >> 4) * KL + c) * 8 < D;
        Frag f[PASSES];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          constexpr int PER = 16 / (int)sizeof(X);
          const Chunk<X> v = __builtin_bit_cast(Chunk<X>, raw[nt][c][e / PER]);
          __bf16 part[PARTS];
          const float x = (float)v.e[e % PER];
          split_query<PARTS>(in ? (a.scale_log2 < 0.0f ? -x : a.scale_log2 > 0.0f ? x : x * 0.0f) : 0.0f, part);
#pragma unroll
          for (int s = 0; s < PASSES; ++s) {
            f[s][e] = PARTS == 1 ? part[0] : (__bf16)0.0f;       // one part: the same in all columns of a head
#pragma unroll
            for (int i = 0; i < PARTS; ++i)
              if (PARTS > 1 && s * R + part0 == i) f[s][e] = part[i];
          }
        }
#pragma unroll
        for (int s = 0; s < PASSES; ++s) query[nt][s][c][own_lane] = f[s];
      }
    }
    lds_barrier();                                // leaves rows under way

    // the sign of the scale, or that it is 0, is in the queries
    const float scale = a.scale_log2 == 0.0f ? 1.0f : fabsf(a.scale_log2);
    constexpr bool kKeep = PASSES * KL * NT <= 4; // the queries' operands in registers
    Frag kept[kKeep ? NT * PASSES * KL : 1];
    if constexpr (kKeep) {
#pragma unroll
      for (int i = 0; i < NT * PASSES * KL; ++i) kept[i] = (&query[0][0][0][0])[64 * i + lane];
    }
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
                      16 * (tile0 * kHeadTile + hd)) = held[4 * held_heads * k + quad * held_heads + hd];
        }
      held_from += holding / F::kSub * kStep;
      holding = 0;
    };

    auto step = [&](int t, auto slot_of) __attribute__((always_inline)) {
      constexpr int kSlot = decltype(slot_of)::value;
      asm volatile("" ::: "memory");              // the queries stay in LDS
      // Of two waves on a SIMD the older one goes first and would end long before the
      // other: raised in every second step, neither runs ahead (64 sequences 75.0 and
      // 74.5 us, one of 65536 tokens 26.4 and 25.2 us).
      __builtin_amdgcn_s_setprio(kSlot == 0 ? 2 : 0);
      const char* const stage = rows + kSlot * kStageBytes;
      count_at(t + kStep, valid_next);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // what the slot held is read
      load_rows(t + kStep, page, valid_next, 1 - kSlot);
      pages_at(t + 2 * kStep);
      landed_but_last();

      uint32_t key[F::kSub][KL], key_e[F::kSub][(KL + 3) / 4], value[F::kRows][NV], value_e[F::kRows][NV];
#pragma unroll
      for (int s = 0; s < F::kSub; ++s) {
        const char* row = stage + (16 * s + col) * row_bytes + quad * KL * 4;
        const char* scales = stage + (16 * s + col) * row_bytes + D / 2 + quad * KL;
#pragma unroll
        for (int c = 0; c < KL; ++c) key[s][c] = ((const uint32_t*)row)[c];
        if constexpr (KL == 2) {
          key_e[s][0] = *(const uint16_t*)scales;
        } else {
#pragma unroll
          for (int c = 0; c < KL / 4; ++c) key_e[s][c] = ((const uint32_t*)scales)[c];
        }
      }
#pragma unroll
      for (int i = 0; i < F::kRows; ++i) {
        const char* row = stage + (F::kTokens + i / 4 * 16 + 4 * quad + i % 4) * row_bytes;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
          const int d = (16 * v + col) * EV;
          if constexpr (EV == 8) value[i][v] = *(const uint32_t*)(row + d / 2);
          else value[i][v] = *(const uint16_t*)(row + d / 2);
          value_e[i][v] = *(const uint8_t*)(row + D / 2 + d / 8);
        }
      }
      __builtin_amdgcn_sched_barrier(0);          // all asked for before the first is used

      Frag kf[F::kSub][KL];
#pragma unroll
      for (int s = 0; s < F::kSub; ++s)
#pragma unroll
        for (int c = 0; c < KL; ++c) {
          const uint32_t e = key_e[s][c / 4];
          const uint32_t at = c % 4 < 3 ? e << (23 - 8 * (c % 4)) : e >> 1;
          u32x4 w;
          e2m1_decode(key[s][c], __uint_as_float(FULL ? at : at & there[c]), (uint32_t*)&w);   // of a scale, the exponent counts
          kf[s][c] = __builtin_bit_cast(Frag, w);
        }

      float dot[NT][F::kRows], tile_top[NT];
      // the largest score of a lane, NaN if one is NaN
      auto tops = [&](int nt) {
        tile_top[nt] = dot[nt][0];
#pragma unroll
        for (int i = 1; i < F::kRows; ++i) tile_top[nt] = __builtin_elementwise_maximum(tile_top[nt], dot[nt][i]);
        tile_top[nt] *= scale;
      };
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        f32x4 d[F::kSub];
#pragma unroll
        for (int s = 0; s < F::kSub; ++s) d[s] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int part = PASSES - 1; part >= 0; --part)            // small terms first
#pragma unroll
          for (int c = 0; c < KL; ++c) {
            const Frag q = kKeep ? kept[kKeep ? (nt * PASSES + part) * KL + c : 0] : query[nt][part][c][lane];
#pragma unroll
            for (int s = 0; s < F::kSub; ++s) d[s] = mul(kf[s][c], q, d[s]);
          }
#pragma unroll
        for (int i = 0; i < F::kRows; ++i) {
          float x = d[i / 4][i % 4];
          if (PARTS > 1 && R > 1) x += other_column<8>(x);       // the parts' scores: the same sum in all columns
          if (PARTS > 1 && R > 2) x += other_column<4>(x);
          dot[nt][i] = x;
        }
      }
      if (valid[0] + valid[1] < F::kTokens) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int i = 0; i < F::kRows; ++i) dot[nt][i] = 4 * quad + i % 4 < valid[i / 4] ? dot[nt][i] : -INFINITY;
      }
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        tops(nt);
        // The products of two parts of a query may overflow to infinities of both
        // signs and add up to NaN although the sum is infinite: such a score is taken
        // from the first parts alone, which have the sign of the whole.
        if (PARTS > 1 && __any(tile_top[nt] != tile_top[nt])) {
          f32x4 d[F::kSub];
#pragma unroll
          for (int s = 0; s < F::kSub; ++s) d[s] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
          for (int c = 0; c < KL; ++c)
#pragma unroll
            for (int s = 0; s < F::kSub; ++s) d[s] = mul(kf[s][c], query[nt][0][c][lane], d[s]);
#pragma unroll
          for (int i = 0; i < F::kRows; ++i) {
            const float x = R > 1 ? __shfl(d[i / 4][i % 4], 16 * quad + col % W) : d[i / 4][i % 4];
            dot[nt][i] = dot[nt][i] == dot[nt][i] ? dot[nt][i] : x;
          }
          tops(nt);
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
              held[4 * held_heads * (holding + s) + quad * held_heads + hd] =
                  f32x4{dot[nt][4 * s], dot[nt][4 * s + 1], dot[nt][4 * s + 2], dot[nt][4 * s + 3]} * scale;
          }
        holding += F::kSub;
      }

      u32x4 pf[NT][WPASSES];
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
        for (int i = 0; i < F::kRows; i += 2) {
          const float w0 = exp2_fast(fmaf(dot[nt][i], scale, -base[nt])), w1 = exp2_fast(fmaf(dot[nt][i + 1], scale, -base[nt]));
          sum[nt] += w0 + w1;                     // all of them, whatever their parts leave out
          uint32_t part[WPARTS];
          split_pair<WPARTS>(w0, w1, part);
#pragma unroll
          for (int s = 0; s < WPASSES; ++s) {
            pf[nt][s][i / 2] = s * R < WPARTS ? part[s * R] : 0u;
#pragma unroll
            for (int o = 1; o < R; ++o)
              if (slot_of_col == o) pf[nt][s][i / 2] = s * R + o < WPARTS ? part[s * R + o < WPARTS ? s * R + o : 0] : 0u;
          }
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
        for (int j = 0; j < EV; j += 2) {
          u32x4 w[2];                               // tokens of two columns
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            w[0][i] = __builtin_amdgcn_perm(x[2 * i + 1][j / 2], x[2 * i][j / 2], 0x05040100u);
            w[1][i] = __builtin_amdgcn_perm(x[2 * i + 1][j / 2], x[2 * i][j / 2], 0x07060302u);
          }
#pragma unroll
          for (int part = WPASSES - 1; part >= 0; --part)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int o = 0; o < 2; ++o)
                acc[nt][v][j + o] = mul(__builtin_bit_cast(Frag, w[o]), __builtin_bit_cast(Frag, pf[nt][part]), acc[nt][v][j + o]);
        }
      }
#pragma unroll
      for (int s = 0; s < F::kSub; ++s) {
        valid[s] = valid_next[s];
      }
    };
    for (int t = first; t < t1; t += 2 * kStep) {
      step(t, std::integral_constant<int, 0>());
      if (t + kStep >= t1) break;
      step(t + kStep, std::integral_constant<int, 1>());
    }
    landed<0>();                                  // the outputs come where rows were
    if (a.accumulate) release();

    // join the waves
    asm volatile("" : "+v"(own_lane));
    const int own_col = own_lane & 15, own_quad = own_lane >> 4;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const float all = head_sum(sum[nt]);        // the same in all columns of a head
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
              *(f32x4*)&slab[wave][own_col][(16 * v + 4 * own_quad + i) * EV + j] =
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
#pragma unroll
          for (int i = (R < WPARTS ? R : WPARTS) - 1; i >= 0; --i) o += *(const f32x4*)&slab[w][hd + i * W][4 * c];
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
    at = before + steps + first64.extra;
    if (at >= stop) return;
    __syncthreads();                              // the outputs are read
    before = at;
    do {
      if (++b >= a.c.batch) return;
    } while (held_tokens_uniform(a.lengths, b, a.max_len) == 0);
  }
}

template <int XT, int DP, int NT, int W, bool FULL, bool STREAM>
void launch_kernel(const AttendLaunch& a, const Work& w, const Plan& p, hipStream_t s) {
  const int64_t shares = (int64_t)a.c.kv_heads * p.workgroups;
  const dim3 grid(kXcds * p.tile_groups, (unsigned)((shares + kXcds - 1) / kXcds)), block(64 * kWaves);
  const int bytes = Lds<XT, DP, NT, W>::bytes(a.accumulate);
  cache_attend_e2m1_kernel<XT, DP, NT, W, FULL, STREAM><<<grid, block, bytes, s>>>(a, w, p.workgroups);
}

template <int XT, int DP, bool FULL>
void launch_tiles(const AttendLaunch& a, const Work& w, const Plan& p, hipStream_t s) {
  const int32_t group = a.heads / a.c.kv_heads;
  // Parts side by side, 64 sequences and 8 key/value heads, without and with, us:
  //   heads of                 128         96        64        256 (up to 4096 tokens)
  //   float32, groups of 4  71.5, 64.5  74.6, 69.4  52.6, 50.4  101.0, 92.6
  //   float32, groups of 8  75.5, 74.4  75.1, 72.9  54.1, 52.9  106.0, 102.3
  //   f16, groups of 4      62.3, 59.5  63.4, 59.3  45.8, 44.5  85.9, 83.4
  //   f16, groups of 8      64.6, 62.2  64.6, 61.1  47.8, 47.3  90.2, 87.1
  //   bf16, groups of 4     59.4, 59.2  56.6, 55.8  42.3, 41.3  78.5, 81.3
  //   bf16, groups of 8     61.7, 61.5  57.9, 58.8  44.5, 43.3  82.2, 83.8
  // (a bf16 query is one part: only its weights' two are taken together).
  if constexpr (DP < 256 || Form<XT, DP>::kParts > 1) {
    if (group <= 4) return launch_kernel<XT, DP, 1, 4, FULL, true>(a, w, p, s);
    if (group <= 8) return launch_kernel<XT, DP, 1, 8, FULL, true>(a, w, p, s);
  }
  if constexpr (DP < 256) {
    if (p.wave_tiles == 1) launch_kernel<XT, DP, 1, 16, FULL, true>(a, w, p, s);
    else if (p.tile_groups == 1) launch_kernel<XT, DP, 2, 16, FULL, true>(a, w, p, s);
    else launch_kernel<XT, DP, 2, 16, FULL, false>(a, w, p, s);
  } else {
    if (p.tile_groups == 1) launch_kernel<XT, DP, 1, 16, FULL, true>(a, w, p, s);
    else launch_kernel<XT, DP, 1, 16, FULL, false>(a, w, p, s);
  }
}

template <int XT, int DP>
void launch_dim(const AttendLaunch& a, const Work& w, const Plan& p, hipStream_t s) {
  if (a.c.head_dim == DP) launch_tiles<XT, DP, true>(a, w, p, s);
  else launch_tiles<XT, DP, false>(a, w, p, s);
}

template <int XT>
Plan plan_for(const AttendLaunch& a) {
  return plan_of(a.c, a.heads, a.max_len, a.c.head_dim <= 64 ? two_fit<XT, 64>(a) : a.c.head_dim <= 128 && two_fit<XT, 128>(a));
}

template <int XT>
hipError_t launch_types(const AttendLaunch& a, hipStream_t s) {
  const Plan p = plan_for<XT>(a);
  const Work w = work_of(a, p);
  if (a.c.head_dim <= 64) launch_dim<XT, 64>(a, w, p, s);
  else if (a.c.head_dim <= 128) launch_dim<XT, 128>(a, w, p, s);
  else launch_dim<XT, 256>(a, w, p, s);
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
