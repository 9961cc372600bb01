// Eviction by accumulated weight (mosaic_cache_evict).
//
// One workgroup selects for one key/value head of one sequence: the rank of a
// token is a 32-bit key, the budget-th largest key is found digit by digit
// (counts of the digits' values in LDS, integers, so no order of the atomics
// shows), and a scan over the slots in their order numbers the survivors,
// which settles ties and pairs the r-th survivor beyond the budget with the
// r-th slot that came free below it. A second kernel copies rows along these
// pairs: sources lie at or beyond the budget and destinations below it, so
// the copies are independent.
#include "cache.h"
#include "dispatch.h"

namespace mosaic {
namespace {

constexpr int kSelectThreads = 1024;
constexpr int kWaves = kSelectThreads / 64;

// Rank of a token; a larger key stays before a smaller one. The latest come
// first, then weights as numbers (0 and -0 alike), then NaN, then slots whose
// page is not there.
constexpr uint32_t kLatest = 0xFFFFFFFFu, kNan = 1u, kAbsent = 0u;
__device__ __forceinline__ uint32_t rank_key(float w, bool latest) {
  if (latest) return kLatest;
  if (w != w) return kNan;
  const uint32_t u = __float_as_uint(w + 0.0f);
  return (u >> 31) != 0u ? ~u : u | 0x80000000u;
}

// Lists of one (sequence, head): keys by slot, then pairs of slots.
struct Lists {
  uint32_t* keys;
  int32_t* holes;
  int32_t* movers;
  int32_t* count;
};
int64_t most_moves(int64_t max_len, int64_t budget) {
  const int64_t beyond = max_len - budget;
  return beyond <= 0 ? 0 : beyond < budget ? beyond : budget;
}
__device__ __forceinline__ Lists lists_of(const EvictLaunch& a, int64_t moves, int64_t bh, int64_t all) {
  uint32_t* keys = (uint32_t*)a.workspace;
  int32_t* holes = (int32_t*)(keys + all * a.max_len);
  int32_t* movers = holes + all * moves;
  return {keys + bh * a.max_len, holes + bh * moves, movers + bh * moves, movers + all * moves + bh};
}

__device__ __forceinline__ void copy_numbers(const EvictLaunch& a, int64_t from, int64_t to) {
  a.new_weights[to] = a.c.weights[from];
  a.new_order[to] = a.c.order[from];
}

__global__ __launch_bounds__(kSelectThreads) void cache_select_kernel(EvictLaunch a, int64_t moves) {
  __shared__ uint32_t bins[2048];
  __shared__ uint32_t part[2 * kWaves];
  __shared__ uint32_t found[2];
  const int h = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t bh = (int64_t)b * a.c.kv_heads + h, all = (int64_t)a.c.batch * a.c.kv_heads;
  const Lists l = lists_of(a, moves, bh, all);
  const int32_t n = held_tokens(a.state, b, a.max_len);
  const int64_t latest = (int64_t)a.state[a.c.batch + b] - a.recent;
  int32_t* kept = a.kept != nullptr ? a.kept + bh * a.budget : nullptr;
  const bool apart = a.new_weights != a.c.weights || a.new_order != a.c.order;

  if (n <= a.budget) {
    for (int64_t i = tid; i < n; i += kSelectThreads) {
      const int32_t page = page_of(a.c, b, i);
      if (apart && page >= 0) copy_numbers(a, row_index(a.c, page, h, i), row_index(a.c, page, h, i));
    }
    if (kept != nullptr)
      for (int64_t i = tid; i < a.budget; i += kSelectThreads) kept[i] = i < n ? (int32_t)i : -1;
    if (tid == 0 && moves > 0) *l.count = 0;
    return;
  }
  const int32_t budget = (int32_t)a.budget;

  // the budget-th largest key, from its upper digits to its lower ones
  uint32_t prefix = 0, need = (uint32_t)budget;
  for (int shift = 21, bits = 11; ; shift -= bits) {
    const int width = shift == 0 ? 10 : 11;
    for (int i = tid; i < 2048; i += kSelectThreads) bins[i] = 0u;
    __syncthreads();
    for (int i = tid; i < n; i += kSelectThreads) {
      uint32_t key;
      if (shift == 21) {
        const int32_t page = page_of(a.c, b, i);
        key = kAbsent;
        if (page >= 0) {
          const int64_t r = row_index(a.c, page, h, i);
          key = rank_key(a.c.weights[r], a.c.order[r] >= latest);
        }
        l.keys[i] = key;
      } else {
        key = l.keys[i];
      }
      if (shift == 21 || (key >> (shift + width)) == prefix) atomicAdd(&bins[(key >> shift) & ((1u << width) - 1)], 1u);
    }
    __syncthreads();
    // thread t holds bins 2047 - 2t and 2046 - 2t: sums from the top
    const uint32_t hi = bins[2047 - 2 * tid], lo = bins[2046 - 2 * tid];
    uint32_t sum = hi + lo;
    for (int off = 1; off < 64; off <<= 1) {
      const uint32_t o = __shfl_up(sum, off);
      if (lane >= off) sum += o;
    }
    if (lane == 63) part[wave] = sum;
    __syncthreads();
    uint32_t before = sum - hi - lo;
    for (int w = 0; w < wave; ++w) before += part[w];
    if (before < need && before + hi + lo >= need) {
      const bool upper = before + hi >= need;
      found[0] = upper ? 2047 - 2 * tid : 2046 - 2 * tid;
      found[1] = need - before - (upper ? 0u : hi);
    }
    __syncthreads();
    prefix = (prefix << width) | found[0];
    need = found[1];
    __syncthreads();
    if (shift == 0) break;
    bits = shift == 21 ? 11 : 10;
  }
  const uint32_t least = prefix;                 // keys above stay, and the first `need` equal to it

  uint32_t above = 0, equal = 0;                 // in the slots before this round's
  int32_t kept_low = 0;
  for (int64_t i0 = 0; i0 < n; i0 += kSelectThreads) {
    const int64_t i = i0 + tid;
    const uint32_t key = i < n ? l.keys[i] : 0u;
    const bool gt = i < n && key > least, eq = i < n && key == least;
    const uint64_t mg = __ballot(gt), me = __ballot(eq);
    if (lane == 0) {
      part[2 * wave] = (uint32_t)__popcll(mg);
      part[2 * wave + 1] = (uint32_t)__popcll(me);
    }
    __syncthreads();
    const uint64_t under = ((uint64_t)1 << lane) - 1;
    uint32_t g = above + (uint32_t)__popcll(mg & under), e = equal + (uint32_t)__popcll(me & under);
    for (int w = 0; w < kWaves; ++w) {
      if (w < wave) {
        g += part[2 * w];
        e += part[2 * w + 1];
      }
      above += part[2 * w];
      equal += part[2 * w + 1];
    }
    const bool stays = gt || (eq && e < need);
    const int32_t rank = (int32_t)(g + (e < need ? e : need));    // survivors in lower slots
    if (i == budget) found[0] = (uint32_t)rank;
    __syncthreads();
    if (i0 + kSelectThreads > budget && i0 <= budget) kept_low = (int32_t)found[0];
    if (i < budget) {
      if (!stays) l.holes[i - rank] = (int32_t)i;
      else {
        const int32_t page = page_of(a.c, b, i);
        if (apart && page >= 0) copy_numbers(a, row_index(a.c, page, h, i), row_index(a.c, page, h, i));
        if (kept != nullptr) kept[i] = (int32_t)i;
      }
    } else if (i < n && stays) {
      l.movers[rank - kept_low] = (int32_t)i;
    }
  }
  if (tid == 0) *l.count = budget - kept_low;
}

// Copies rows along the pairs of slots, 16 bytes per thread.
__global__ __launch_bounds__(256) void cache_move_kernel(EvictLaunch a, int64_t moves, int32_t per_block) {
  const int h = blockIdx.y, b = blockIdx.z;
  const int64_t bh = (int64_t)b * a.c.kv_heads + h, all = (int64_t)a.c.batch * a.c.kv_heads;
  if (blockIdx.x == 0 && h == 0 && threadIdx.x == 0) {
    const int32_t n = held_tokens(a.state, b, a.max_len);
    const int32_t seen = a.state[a.c.batch + b];
    a.new_state[b] = n < a.budget ? n : (int32_t)a.budget;
    a.new_state[a.c.batch + b] = seen;
  }
  if (moves == 0) return;
  const Lists l = lists_of(a, moves, bh, all);
  const int32_t first = (int32_t)blockIdx.x * per_block;
  int32_t count = *l.count - first;
  count = count < per_block ? count : per_block;
  const int32_t chunks = a.c.head_dim * (a.c.dtype == MOSAIC_F32 ? 4 : 2) / 16;
  for (int32_t w = threadIdx.x; w < count * chunks; w += 256) {
    const int32_t m = w / chunks, c = w - m * chunks;
    const int32_t from = l.movers[first + m], to = l.holes[first + m];
    const int32_t pf = page_of(a.c, b, from), pt = page_of(a.c, b, to);
    if (pf < 0 || pt < 0) continue;
    const int64_t of = row_offset(a.c, pf, h, from) + 16 * c, ot = row_offset(a.c, pt, h, to) + 16 * c;
    const uint4 k = *(const uint4*)(a.c.k + of), v = *(const uint4*)(a.c.v + of);
    *(uint4*)(a.c.k + ot) = k;
    *(uint4*)(a.c.v + ot) = v;
    if (c == 0) {
      copy_numbers(a, row_index(a.c, pf, h, from), row_index(a.c, pt, h, to));
      if (a.kept != nullptr) a.kept[bh * a.budget + to] = from;
    }
  }
}

}  // namespace

int64_t cache_evict_workspace(const CacheView& c, int64_t max_len, int64_t budget) {
  const int64_t moves = most_moves(max_len, budget);
  return moves == 0 ? 0 : (int64_t)c.batch * c.kv_heads * (max_len + 2 * moves + 1) * 4;
}

hipError_t launch_cache_evict(const EvictLaunch& a, hipStream_t s) {
  const int64_t moves = most_moves(a.max_len, a.budget);
  cache_select_kernel<<<dim3(a.c.kv_heads, a.c.batch), kSelectThreads, 0, s>>>(a, moves);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int32_t per_block = 64;
  const unsigned blocks = moves > 0 ? (unsigned)((moves + per_block - 1) / per_block) : 1u;
  cache_move_kernel<<<dim3(blocks, a.c.kv_heads, a.c.batch), 256, 0, s>>>(a, moves, per_block);
  return hipGetLastError();
}

}  // namespace mosaic
