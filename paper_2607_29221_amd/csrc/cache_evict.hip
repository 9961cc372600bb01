// Eviction by accumulated weight (mosaic_cache_evict).
//
// The rank of a token is a 32-bit key, and the budget-th largest key of a
// key/value head is found digit by digit (11, 11 and 10 bits): counts of a
// digit's values in LDS, integers, so no order of the atomics shows. Counting
// the survivors over the slots in their order then settles ties and numbers
// both sides of the move: the r-th slot that came free below the budget takes
// the r-th survivor from beyond it. Sources lie at or beyond the budget and
// destinations below it, so a last kernel copies rows along these pairs in any
// order.
//
// Up to kShortSlots slots one workgroup takes a head: its keys stay in
// registers through all the steps. Beyond, a workgroup takes kChunk slots and
// the steps are launches: counts of the first, second and third digit (each
// finds the digit before it from the counts of all chunks), then the numbering.
//
// Measured on an MI355X, 8 key/value heads: 64 sequences of 2049 tokens to
// 2048: 8.9 us for the selection (21 MB of weights, order and slots in and
// out: 2.4 TB/s, half of it latency) and 3.4 us for one row per head; four of up
// to 7168 to 1024: 12 us, the latency of its steps on 32 workgroups, and
// 11.6 us for 50 MB of float32 rows; one of 131072 to 8192: 7.6 + 6.3 + 6.8 +
// 8.8 us, and 15.3 us for 62 MB of rows.
#include "cache.h"
#include "device_common.h"
#include "dispatch.h"

namespace mosaic {
namespace {

constexpr int kBins = 2048;
constexpr int kShortSlots = 8192;
constexpr int kChunk = 8192, kChunkThreads = 1024, kChunkKeys = kChunk / kChunkThreads;
// Evictions that are found one by one: a loop at its budget has one per step
// (64 sequences of 2049 to 2048: 8.9 us, 13.8 us by digits).
constexpr int kFew = 4;

// Rank of a slot; a larger key stays before a smaller one. The latest tokens
// come first, then weights as numbers (0 and -0 alike), then NaN. A slot whose
// page is not there holds nothing. Below the budget nothing can be moved to it
// either: it stays, before everything else, as one of the budget's slots, so
// the tokens that are there have that many fewer (ties go to the lowest slot,
// so slots below the budget with the largest key always stay). Beyond the budget it
// goes first; the slots that are there are never fewer than what is left of the
// budget, so none such is among the survivors.
constexpr uint32_t kHole = 0xFFFFFFFFu, kLatest = 0xFFFFFFFEu, kNan = 1u, kAbsent = 0u;
__device__ __forceinline__ uint32_t rank_key(float w, bool latest) {
  if (latest) return kLatest;
  if (w != w) return kNan;
  const uint32_t u = __float_as_uint(w + 0.0f);
  return (u >> 31) != 0u ? ~u : u | 0x80000000u;
}

// Of one (sequence, head): the slots that came free below the budget, in
// order; the survivors beyond it, from the last to the first; how many.
// Beyond kShortSlots also keys by slot, the counts of the three digits by
// chunk, the digits found so far with the number still needed below them, and
// the survivors of each chunk that are above the digits found so far.
struct Lists {
  int32_t *free_slots, *movers, *count;
  uint32_t *keys, *counts[3], *found, *above;
  int64_t chunks;
};
int64_t most_moves(int64_t max_len, int64_t budget) {
  const int64_t beyond = max_len - budget;
  return beyond <= 0 ? 0 : beyond < budget ? beyond : budget;
}
__host__ __device__ inline int64_t chunks_of(int64_t max_len) {
  return max_len <= kShortSlots ? 0 : (max_len + kChunk - 1) / kChunk;
}
// words of the workspace per (sequence, head)
int64_t list_words(int64_t max_len, int64_t budget) {
  const int64_t moves = most_moves(max_len, budget), chunks = chunks_of(max_len);
  return moves == 0 ? 0 : 2 * moves + 1 + (chunks > 0 ? max_len + 3 * kBins * chunks + 4 + chunks : 0);
}
__device__ __forceinline__ Lists lists_of(const EvictLaunch& a, int64_t moves, int64_t bh) {
  const int64_t all = (int64_t)a.c.batch * a.c.kv_heads;
  Lists l;
  l.chunks = chunks_of(a.max_len);
  uint32_t* p = (uint32_t*)a.workspace;
  for (int d = 0; d < 3; ++d) {
    l.counts[d] = p + bh * l.chunks * kBins;
    p += all * l.chunks * kBins;
  }
  if (l.chunks > 0) {
    l.found = p + 4 * bh;
    l.above = p + 4 * all + bh * l.chunks;
    l.keys = p + (4 + l.chunks) * all + bh * a.max_len;
    p += all * (4 + l.chunks + a.max_len);
  }
  l.free_slots = (int32_t*)p + bh * moves;
  l.movers = (int32_t*)p + (all + bh) * moves;
  l.count = (int32_t*)p + 2 * all * moves + bh;
  return l;
}

// Digit d of the key: its lowest bit and its width.
__device__ __forceinline__ int digit_shift(int d) { return d == 0 ? 21 : d == 1 ? 10 : 0; }
__device__ __forceinline__ uint32_t digit_of(uint32_t key, int d) {
  return (key >> digit_shift(d)) & (d == 2 ? 1023u : 2047u);
}
// whether a key agrees with the digits before d
__device__ __forceinline__ bool agrees(uint32_t key, uint32_t prefix, int d) {
  return d == 0 || (key >> digit_shift(d - 1)) == prefix;
}

// From counts of a digit (thread t holds those of values BINS - 1 - PER t
// downwards in own[0 ..]): the value at which the running sum from the top
// reaches `need`, and what is still needed within it. All threads.
template <int THREADS, int BINS>
__device__ __forceinline__ void find_digit(const uint32_t (&own)[BINS / THREADS], uint32_t need, uint32_t* part,
                                           uint32_t* found) {
  constexpr int PER = BINS / THREADS;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  uint32_t total = 0;
#pragma unroll
  for (int k = 0; k < PER; ++k) total += own[k];
  const uint32_t sum = (uint32_t)wave_scan((int)total);
  if (lane == 63) part[wave] = sum;
  __syncthreads();
  uint32_t before = sum - total;
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) before += w < wave ? part[w] : 0u;
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    if (before < need && before + own[k] >= need) {
      found[0] = (uint32_t)(BINS - 1 - PER * tid - k);
      found[1] = need - before;
    }
    before += own[k];
  }
  __syncthreads();
}

// The numbers of a token that stays in its slot, to wherever they are wanted.
// there: the slot has a page; row: its place in the arrays, or -1 if nothing is to be written.
__device__ __forceinline__ void stay(const EvictLaunch& a, int32_t* kept, bool apart, bool there, int64_t row,
                                     int32_t slot, float w, int32_t o) {
  if (apart && row >= 0) {
    a.new_weights[row] = w;
    a.new_order[row] = o;
  }
  if (kept != nullptr) kept[slot] = there ? slot : -1;
}

// A workgroup's slots first + THREADS r + tid: keys, and what they come from.
template <int R> struct Tokens {
  uint32_t key[R];
  float w[R];
  int32_t o[R];
  int64_t row[R];         // index into weights and order, -1 if there is none
};
template <int THREADS, int R>
__device__ __forceinline__ void load_tokens(const EvictLaunch& a, int b, int h, int32_t first, int32_t n, int64_t latest,
                                            Tokens<R>& t) {
  const float* weights = a.c.pages > 0 ? a.c.weights : (const float*)a.state;
  const int32_t* order = a.c.pages > 0 ? a.c.order : a.state;
  int32_t page[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int32_t i = first + THREADS * r + (int)threadIdx.x;
    page[r] = page_of(a.c, b, min(i, n - 1));
  }
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int32_t i = min(first + THREADS * r + (int)threadIdx.x, n - 1);
    t.row[r] = page[r] >= 0 ? row_index(a.c, page[r], h, i) : -1;
    const int64_t safe = page[r] >= 0 ? t.row[r] : 0;     // a load that every lane can make
    t.w[r] = weights[safe];
    t.o[r] = order[safe];
  }
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const bool below = first + THREADS * r + (int)threadIdx.x < a.budget;
    t.key[r] = t.row[r] >= 0 ? rank_key(t.w[r], t.o[r] >= latest) : below ? kHole : kAbsent;
  }
}

// Numbers the slots first .. of a workgroup, of which `above` lower ones have
// a key over `least` and `equal` a key like it (of those `need` stay), and
// writes the lists. cnt: THREADS / 64 * R words.
template <int THREADS, int R>
__device__ __forceinline__ void number_slots(const EvictLaunch& a, int b, int h, const Lists& l, int32_t* kept,
                                             bool apart, int32_t first, int32_t n, uint32_t least, uint32_t need, uint32_t above,
                                             uint32_t equal, const Tokens<R>& t, uint32_t* cnt) {
  constexpr int NW = THREADS / 64, ENTRIES = NW * R, EACH = (ENTRIES + 63) / 64;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int32_t budget = (int32_t)a.budget;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const bool in = first + THREADS * r + tid < n;
    const uint32_t g = (uint32_t)__popcll(__ballot(in && t.key[r] > least));
    const uint32_t e = (uint32_t)__popcll(__ballot(in && t.key[r] == least));
    if (lane == 0) cnt[NW * r + wave] = g << 16 | e;        // at most kShortSlots of each
  }
  __syncthreads();
  if (wave == 0) {
    uint32_t v[EACH], sum = 0;
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
      const int at = EACH * lane + k;
      v[k] = at < ENTRIES ? cnt[at] : 0u;
      sum += v[k];
    }
    uint32_t run = (uint32_t)wave_scan((int)sum) - sum;
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
      if (EACH * lane + k < ENTRIES) cnt[EACH * lane + k] = run;
      run += v[k];
    }
  }
  __syncthreads();
  const uint64_t under = ((uint64_t)1 << lane) - 1;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int32_t i = first + THREADS * r + tid;
    const bool in = i < n, gt = in && t.key[r] > least, eq = in && t.key[r] == least;
    const uint64_t mg = __ballot(gt), me = __ballot(eq);
    const uint32_t base = cnt[NW * r + wave];
    const uint32_t g = above + (base >> 16) + (uint32_t)__popcll(mg & under);
    const uint32_t e = equal + (base & 0xFFFFu) + (uint32_t)__popcll(me & under);
    const int32_t rank = (int32_t)(g + (e < need ? e : need));    // survivors in lower slots
    const bool stays = gt || (eq && e < need);
    if (i == budget) *l.count = budget - rank;
    if (i < budget && in) {
      if (!stays) {
        l.free_slots[i - rank] = i;
      } else {
        stay(a, kept, apart, t.key[r] != kHole, t.row[r], i, t.w[r], t.o[r]);
      }
    } else if (stays) {
      l.movers[budget - 1 - rank] = i;
    }
  }
}

__device__ __forceinline__ int64_t first_latest(const EvictLaunch& a, int b) {
  return (int64_t)a.state[a.c.batch + b] - a.recent;
}
__device__ __forceinline__ bool apart_of(const EvictLaunch& a) {
  return a.new_weights != a.c.weights || a.new_order != a.c.order;
}

// One head, all its keys in registers.
template <int THREADS, int R>
__global__ __launch_bounds__(THREADS) void cache_select_kernel(EvictLaunch a, int64_t moves) {
  constexpr int NW = THREADS / 64, PER = kBins / THREADS;
  __shared__ uint32_t bins[3][kBins];             // a digit's each, so that none waits to be cleared
  __shared__ uint32_t part[3][NW], found[3][2], cnt[NW * R];
  __shared__ uint64_t worst[NW];
  const int h = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t bh = (int64_t)b * a.c.kv_heads + h;
  const int32_t n = held_tokens(a.state, b, a.max_len);
  int32_t* kept = a.kept != nullptr ? a.kept + bh * a.budget : nullptr;
  const bool apart = apart_of(a);
  const Lists l = lists_of(a, moves, bh);
  if (n <= a.budget && moves > 0 && tid == 0) *l.count = 0;
  if (kept != nullptr)
    for (int64_t i = n + tid; i < a.budget; i += THREADS) kept[i] = -1;
  if (n == 0) return;
  Tokens<R> t;
  load_tokens<THREADS, R>(a, b, h, 0, n, first_latest(a, b), t);
  if (n <= a.budget) {
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (THREADS * r + tid < n) stay(a, kept, apart, t.row[r] >= 0, t.row[r], THREADS * r + tid, t.w[r], t.o[r]);
    return;
  }
  const int32_t budget = (int32_t)a.budget;

  if (n - budget <= kFew) {
    // a step of a loop at its budget: the smallest key goes, of equal ones the
    // last, once or a few times
    uint32_t gone = 0;                            // of this thread's slots, by bits
    int32_t out[kFew];
    const int32_t evicted = n - budget;
#pragma unroll
    for (int k = 0; k < kFew; ++k) {
      out[k] = n;                                 // none
      if (k >= evicted) continue;
      uint64_t m = ~(uint64_t)0;
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const int32_t i = THREADS * r + tid;
        const uint64_t v = (uint64_t)t.key[r] << 32 | (uint32_t)~i;
        if (i < n && ((gone >> r) & 1u) == 0u && v < m) m = v;
      }
#pragma unroll
      for (int off = 32; off > 0; off >>= 1) {
        const uint64_t o = __shfl_xor(m, off);
        m = o < m ? o : m;
      }
      if (lane == 0) worst[wave] = m;
      __syncthreads();
#pragma unroll
      for (int w = 0; w < NW; ++w) m = worst[w] < m ? worst[w] : m;
      __syncthreads();
      out[k] = (int32_t)~(uint32_t)m;
      if (out[k] % THREADS == tid) gone |= 1u << (out[k] / THREADS);
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int32_t i = THREADS * r + tid;
      if (i >= n) continue;
      const bool stays = ((gone >> r) & 1u) == 0u;
      if (i < budget && stays) {
        stay(a, kept, apart, t.row[r] >= 0, t.row[r], i, t.w[r], t.o[r]);
      } else if (i < budget || stays) {
        int32_t lower = 0, lower_within = 0;      // evicted slots below i, and those within the budget
#pragma unroll
        for (int k = 0; k < kFew; ++k) {
          lower += k < evicted && out[k] < i ? 1 : 0;
          lower_within += k < evicted && out[k] < budget ? 1 : 0;
        }
        if (i < budget) l.free_slots[lower] = i;
        else l.movers[lower_within - 1 - (i - budget - (lower - lower_within))] = i;
      }
      if (i == budget) {
        int32_t count = 0;
#pragma unroll
        for (int k = 0; k < kFew; ++k) count += k < evicted && out[k] < budget ? 1 : 0;
        *l.count = count;
      }
    }
    return;
  }

  uint32_t prefix = 0, need = (uint32_t)budget;
#pragma unroll
  for (int d = 0; d < 3; ++d)
#pragma unroll
    for (int k = 0; k < PER; ++k) bins[d][THREADS * k + tid] = 0u;
  __syncthreads();
#pragma unroll
  for (int d = 0; d < 3; ++d) {
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (THREADS * r + tid < n && agrees(t.key[r], prefix, d)) atomicAdd(&bins[d][digit_of(t.key[r], d)], 1u);
    __syncthreads();
    uint32_t own[PER];
#pragma unroll
    for (int k = 0; k < PER; ++k) own[k] = bins[d][kBins - 1 - PER * tid - k];
    find_digit<THREADS, kBins>(own, need, part[d], found[d]);
    prefix = prefix << (d == 2 ? 10 : 11) | found[d][0];
    need = found[d][1];
  }
  number_slots<THREADS, R>(a, b, h, l, kept, apart, 0, n, prefix, need, 0u, 0u, t, cnt);
}

// Long sequences: the counts of digit D, in chunks of slots.
template <int D>
__global__ __launch_bounds__(kChunkThreads) void cache_count_kernel(EvictLaunch a, int64_t moves) {
  constexpr int PER = kBins / kChunkThreads;
  __shared__ uint32_t bins[kBins];
  __shared__ uint32_t part[kChunkThreads / 64], found[2];
  const int chunk = blockIdx.x, h = blockIdx.y, b = blockIdx.z, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t bh = (int64_t)b * a.c.kv_heads + h;
  const int32_t n = held_tokens(a.state, b, a.max_len), first = chunk * kChunk;
  if (n <= a.budget || first >= n) return;
  const Lists l = lists_of(a, moves, bh);
  uint32_t key[kChunkKeys];
  if (D == 0) {
    Tokens<kChunkKeys> t;
    load_tokens<kChunkThreads, kChunkKeys>(a, b, h, first, n, first_latest(a, b), t);
#pragma unroll
    for (int r = 0; r < kChunkKeys; ++r) {
      const int32_t i = first + kChunkThreads * r + tid;
      key[r] = t.key[r];
      if (i < n) l.keys[i] = key[r];
    }
  } else {
#pragma unroll
    for (int r = 0; r < kChunkKeys; ++r) key[r] = l.keys[min(first + kChunkThreads * r + tid, n - 1)];
  }
  uint32_t prefix = 0;
  if (D > 0) {
    const int chunks = (n + kChunk - 1) / kChunk;
    uint32_t own[PER] = {};
#pragma unroll 16
    for (int c = 0; c < chunks; ++c)
#pragma unroll
      for (int k = 0; k < PER; ++k) own[k] += l.counts[D - 1][(int64_t)c * kBins + kBins - 1 - PER * tid - k];
    const uint32_t before = D > 1 ? l.found[0] : 0u;
    find_digit<kChunkThreads, kBins>(own, D > 1 ? l.found[1] : (uint32_t)a.budget, part, found);
    prefix = before << 11 | found[0];
    if (chunk == 0 && tid == 0) {
      l.found[2 * (D - 1)] = prefix;
      l.found[2 * (D - 1) + 1] = found[1];
    }
  }
  if (D == 2) {
    // this chunk's survivors by the digits found so far
    uint32_t above = 0;
#pragma unroll
    for (int r = 0; r < kChunkKeys; ++r)
      above += (uint32_t)__popcll(__ballot(first + kChunkThreads * r + tid < n && (key[r] >> digit_shift(D - 1)) > prefix));
    __syncthreads();
    if (lane == 0) part[wave] = above;
    __syncthreads();
    if (tid == 0) {
      above = 0;
      for (int w = 0; w < kChunkThreads / 64; ++w) above += part[w];
      l.above[chunk] = above;
    }
  }
#pragma unroll
  for (int k = 0; k < PER; ++k) bins[kChunkThreads * k + tid] = 0u;
  __syncthreads();
#pragma unroll
  for (int r = 0; r < kChunkKeys; ++r)
    if (first + kChunkThreads * r + tid < n && agrees(key[r], prefix, D)) atomicAdd(&bins[digit_of(key[r], D)], 1u);
  __syncthreads();
#pragma unroll
  for (int k = 0; k < PER; ++k)
    l.counts[D][(int64_t)chunk * kBins + kChunkThreads * k + tid] = bins[kChunkThreads * k + tid];
}

// The numbering, kNumberKeys rounds of slots per workgroup (a chunk's take more
// instructions than one compute unit should issue): rounds before its own in
// the chunk are counted again.
constexpr int kNumberKeys = 4, kNumberParts = kChunkKeys / kNumberKeys, kLastBins = 1024;
__global__ __launch_bounds__(kChunkThreads) void cache_number_kernel(EvictLaunch a, int64_t moves) {
  constexpr int NW = kChunkThreads / 64;
  __shared__ uint32_t part[NW], part_equal[NW], found[2], cnt[NW * kNumberKeys], lower[2], lower_bin;
  const int chunk = blockIdx.x / kNumberParts, round0 = blockIdx.x % kNumberParts * kNumberKeys;
  const int h = blockIdx.y, b = blockIdx.z, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t bh = (int64_t)b * a.c.kv_heads + h;
  const int32_t n = held_tokens(a.state, b, a.max_len), chunk0 = chunk * kChunk, first = chunk0 + kChunkThreads * round0;
  int32_t* kept = a.kept != nullptr ? a.kept + bh * a.budget : nullptr;
  const bool apart = apart_of(a);
  const Lists l = lists_of(a, moves, bh);
  if (kept != nullptr)
    for (int64_t i = n + (int64_t)blockIdx.x * kChunkThreads + tid; i < a.budget; i += (int64_t)gridDim.x * kChunkThreads)
      kept[i] = -1;
  if (n <= a.budget) {
    if (blockIdx.x == 0 && tid == 0 && moves > 0) *l.count = 0;
    for (int32_t i = first + tid; i < min(n, first + kNumberKeys * kChunkThreads); i += kChunkThreads) {
      const int32_t page = page_of(a.c, b, i);
      const int64_t row = page >= 0 ? row_index(a.c, page, h, i) : -1;
      stay(a, kept, apart, row >= 0, row, i, row >= 0 ? a.c.weights[row] : 0.0f, row >= 0 ? a.c.order[row] : 0);
    }
    return;
  }
  if (first >= n) return;
  uint32_t key[kChunkKeys - kNumberKeys];
#pragma unroll
  for (int r = 0; r < kChunkKeys - kNumberKeys; ++r) key[r] = r < round0 ? l.keys[chunk0 + kChunkThreads * r + tid] : 0u;
  Tokens<kNumberKeys> t;
  int32_t page[kNumberKeys];
  const bool copies = apart && first < a.budget;
#pragma unroll
  for (int r = 0; r < kNumberKeys; ++r) {
    const int32_t i = min(first + kChunkThreads * r + tid, n - 1);
    t.key[r] = l.keys[i];
    page[r] = copies ? page_of(a.c, b, i) : -1;
  }
  // the last digit, and how many of its values lie in the chunks before
  const int chunks = (n + kChunk - 1) / kChunk;
  uint32_t own[1] = {0}, earlier = 0, above = 0;
#pragma unroll 8
  for (int c = 0; c < chunks; ++c) {
    const uint32_t v = l.counts[2][(int64_t)c * kBins + kLastBins - 1 - tid];
    own[0] += v;
    earlier += c < chunk ? v : 0u;
  }
  for (int c = tid; c < chunk; c += kChunkThreads) above += l.above[c];
#pragma unroll
  for (int r = 0; r < kNumberKeys; ++r) {         // under way while the digit is found
    t.row[r] = page[r] >= 0 ? row_index(a.c, page[r], h, min(first + kChunkThreads * r + tid, n - 1)) : -1;
    t.w[r] = page[r] >= 0 ? a.c.weights[t.row[r]] : 0.0f;
    t.o[r] = page[r] >= 0 ? a.c.order[t.row[r]] : 0;
  }
  find_digit<kChunkThreads, kLastBins>(own, l.found[3], part, found);
  const uint32_t digit = found[0], need = found[1], least = l.found[2] << 10 | digit;
  const uint32_t value = (uint32_t)(kLastBins - 1 - tid);
  if (value > digit) above += earlier;
  if (value == digit) lower_bin = earlier;
  uint32_t equal = 0;
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) above += __shfl_xor(above, off);
#pragma unroll
  for (int r = 0; r < kChunkKeys - kNumberKeys; ++r)
    if (r < round0) {
      above += (uint32_t)__popcll(__ballot(key[r] > least));
      equal += (uint32_t)__popcll(__ballot(key[r] == least));
    }
  __syncthreads();
  if (lane == 0) {
    part[wave] = above;
    part_equal[wave] = equal;
  }
  __syncthreads();
  if (tid == 0) {
    above = 0;
    equal = lower_bin;
    for (int w = 0; w < NW; ++w) {
      above += part[w];
      equal += part_equal[w];
    }
    lower[0] = above;
    lower[1] = equal;
  }
  __syncthreads();
  number_slots<kChunkThreads, kNumberKeys>(a, b, h, l, kept, apart, first, n, least, need, lower[0], lower[1], t, cnt);
}

// Copies rows along the pairs of slots, 16 bytes per thread. Bound by the rows'
// traffic: 63 MB in and out in 15.4 us for the 131072 -> 8192 case, in 15.7 us
// with 64 moves per workgroup (more rounds of dependent loads for a thread).
// A launch takes less than 2^32 threads along an axis, so beyond kMostBlocks
// workgroups they go on to further moves.
constexpr int32_t kMovesPerBlock = 16, kMostBlocks = 1 << 16;
__global__ __launch_bounds__(256) void cache_move_kernel(EvictLaunch a, int64_t moves) {
  const int h = blockIdx.y, b = blockIdx.z;
  const int64_t bh = (int64_t)b * a.c.kv_heads + h;
  if (blockIdx.x == 0 && h == 0 && threadIdx.x == 0) {
    const int32_t n = held_tokens(a.state, b, a.max_len);
    const int32_t seen = a.state[a.c.batch + b];
    a.new_state[b] = n < a.budget ? n : (int32_t)a.budget;
    a.new_state[a.c.batch + b] = seen;
  }
  if (moves == 0) return;
  const Lists l = lists_of(a, moves, bh);
  const int32_t all = *l.count;
  const int32_t chunks = a.c.head_dim * (a.c.dtype == MOSAIC_F32 ? 4 : 2) / 16;
  for (int32_t first = (int32_t)blockIdx.x * kMovesPerBlock; first < all; first += (int32_t)gridDim.x * kMovesPerBlock) {
    const int32_t count = min(all - first, kMovesPerBlock);
    for (int32_t w = threadIdx.x; w < count * chunks; w += 256) {
      const int32_t m = w / chunks, c = w - m * chunks;
      const int32_t from = l.movers[all - 1 - (first + m)], to = l.free_slots[first + m];
      const int32_t pf = page_of(a.c, b, from), pt = page_of(a.c, b, to);   // both are there: see rank_key
      const int64_t of = row_offset(a.c, pf, h, from) + 16 * c, ot = row_offset(a.c, pt, h, to) + 16 * c;
      const u32x4 k = *(const u32x4*)(a.c.k + of), v = *(const u32x4*)(a.c.v + of);
      *(u32x4*)(a.c.k + ot) = k;
      *(u32x4*)(a.c.v + ot) = v;
      if (c == 0) {
        const int64_t rf = row_index(a.c, pf, h, from), rt = row_index(a.c, pt, h, to);
        a.new_weights[rt] = a.c.weights[rf];
        a.new_order[rt] = a.c.order[rf];
        if (a.kept != nullptr) a.kept[bh * a.budget + to] = from;
      }
    }
  }
}

}  // namespace

int64_t cache_evict_workspace(const CacheView& c, int64_t max_len, int64_t budget) {
  return (int64_t)c.batch * c.kv_heads * list_words(max_len, budget) * 4;
}

hipError_t launch_cache_evict(const EvictLaunch& a, hipStream_t s) {
  const int64_t moves = most_moves(a.max_len, a.budget);
  const dim3 heads(a.c.kv_heads, a.c.batch);
  if (a.max_len <= 1024) {
    cache_select_kernel<256, 4><<<heads, 256, 0, s>>>(a, moves);
  } else if (a.max_len <= 4096) {
    cache_select_kernel<512, 8><<<heads, 512, 0, s>>>(a, moves);
  } else if (a.max_len <= kShortSlots) {
    cache_select_kernel<1024, 8><<<heads, 1024, 0, s>>>(a, moves);
  } else {
    const dim3 grid((unsigned)chunks_of(a.max_len), a.c.kv_heads, a.c.batch);
    if (moves > 0) {
      cache_count_kernel<0><<<grid, kChunkThreads, 0, s>>>(a, moves);
      cache_count_kernel<1><<<grid, kChunkThreads, 0, s>>>(a, moves);
      cache_count_kernel<2><<<grid, kChunkThreads, 0, s>>>(a, moves);
    }
    cache_number_kernel<<<dim3(grid.x * kNumberParts, grid.y, grid.z), kChunkThreads, 0, s>>>(a, moves);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int64_t blocks = moves > 0 ? (moves + kMovesPerBlock - 1) / kMovesPerBlock : 1;
  cache_move_kernel<<<dim3((unsigned)(blocks < kMostBlocks ? blocks : kMostBlocks), a.c.kv_heads, a.c.batch), 256, 0, s>>>(a, moves);
  return hipGetLastError();
}

}  // namespace mosaic
