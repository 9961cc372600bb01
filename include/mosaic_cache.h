/*
 * mosaic_cache.h -- C ABI of the trusted client's cached decoding.
 *
 * Attention, and the keys and values it reads, stay with the client (the
 * paper's Section 5.1: non-linear layers are evaluated locally in floating
 * point). Between the masked q|k|v product of a new token and the masked
 * output projection the client does three things, one entry point each:
 *   mosaic_cache_append  rotates the new query and key by the token's
 *                        position and writes key and value into the cache,
 *   mosaic_cache_attend  attends from the query over the cached tokens, and
 *                        adds up how much weight each of them got,
 *   mosaic_cache_evict   drops the tokens that got least.
 *
 * Conventions are those of mosaic.h (device pointers owned by the caller,
 * asynchronous on ``stream``, arguments validated before anything is
 * launched, nothing allocated or kept between calls, empty calls do nothing).
 * Workspaces are the caller's too: their sizes come from the *_workspace
 * functions, their contents have no meaning between calls, and two calls that
 * may run at the same time need one each. 16-byte alignment is required
 * where it is said.
 *
 * The cache. Sequence b (0 <= b < batch) holds tokens in slots 0 .. n-1.
 * Slot i lies in page block_table[b * ldt + i / page_size], at place
 * i mod page_size; the row of key/value head h there starts at element
 *     page * page_stride + h * head_stride + place * token_stride
 * of ``k`` and of ``v`` and has head_dim elements. Strides are in elements.
 * Both orders, (page, head, place) and (page, place, head), and gaps are
 * fine, as long as the rows of a page do not overlap and pages do not.
 * Alongside every row two numbers may be kept, in contiguous arrays of
 * pages x kv_heads x page_size: ``weights``, the attention weight that the
 * token has got from the queries of this head's group so far, and ``order``,
 * the token's number in its sequence (0, 1, ...). The heads of a sequence
 * hold equally many tokens but, once tokens were evicted, not the same ones
 * and in no particular order of slots.
 *
 * A block-table entry outside [0, pages) is a page that is not there: its
 * tokens are not read, not written and not evicted to. Sequences share no
 * page that a call writes to (through append, accumulated weights or
 * eviction). ``ldt`` 0 is one row of the table that all sequences share; only
 * attention without accumulated weights takes it.
 *
 * ``state`` is an int32 array [2][batch]: the number of tokens that sequence
 * b holds (a negative one counts as 0, and one beyond the block table's
 * max_blocks * page_size slots as that), then the number that it has seen
 * since its start, evicted ones among them. Calls that change it write
 * ``new_state``, which may be ``state`` itself and may not overlap it
 * otherwise.
 */
#ifndef MOSAIC_CACHE_H
#define MOSAIC_CACHE_H

#include <stdint.h>

#include "mosaic.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum mosaic_ftype {
  MOSAIC_F32 = 0,
  MOSAIC_BF16 = 1,
  MOSAIC_F16 = 2
} mosaic_ftype;

typedef struct mosaic_kv_cache {
  void* k;                    /* 16-byte aligned */
  void* v;                    /* 16-byte aligned; strides as k's */
  float* weights;             /* NULL if not kept */
  int32_t* order;             /* NULL if not kept */
  const int32_t* block_table; /* batch rows of max_blocks entries */
  int64_t ldt;
  int64_t pages;
  int64_t page_stride;        /* strides: multiples of 16 bytes */
  int64_t head_stride;
  int64_t token_stride;
  int32_t dtype;              /* mosaic_ftype of k and v */
  int32_t batch;
  int32_t max_blocks;
  int32_t kv_heads;
  int32_t head_dim;           /* a multiple of 8, at most 256 */
  int32_t page_size;          /* a power of two, 16 to 4096 */
} mosaic_kv_cache;

/* Rotary positions. Pair j of a head (j < P, P the sum of the naxes entries
 * of ``sections``, 2 P <= head_dim) are its elements j and P + j, or 2j and
 * 2j + 1 if ``interleaved``; the elements from 2P on stay as they are. Pairs
 * belong to the axes in order, sections[a] of them to axis a (for pictures
 * and video: time, height, width). With the token's place p on the pair's
 * axis, c = table[p][j] and s = table[p][P + j], the pair (x, y) becomes
 * (x c - y s, y c + x s), computed in float32 and rounded once to the
 * output's type. */
typedef struct mosaic_rotary {
  const float* table;         /* rows x 2P: cosines, then sines */
  int64_t rows;               /* at least 1 */
  const int32_t* positions;   /* naxes x ldp, a token's place on every axis
                                 (one outside the table counts as its nearest
                                 row); NULL: its number in its sequence */
  int64_t ldp;                /* at least the tokens, or 0: all axes share one
                                 row of places */
  int32_t naxes;              /* 1 to 4 */
  int32_t sections[4];
  int32_t interleaved;
} mosaic_rotary;

/* New tokens. Row t of ``qkv`` (rows x (heads + 2 kv_heads) * head_dim:
 * queries, keys, values, as the fused projection gives them) is a token of
 * sequence b for starts[b] <= t < starts[b + 1] (starts: batch + 1 ascending
 * entries, the first 0 and the last ``rows``; NULL: rows == batch and row b
 * is sequence b's). The i-th new token of a sequence that holds n goes to
 * slot n + i. Writes the rotated queries to q_out (rows x heads * head_dim,
 * the type of qkv, not overlapping it), rotated keys and the values into the
 * cache (rounded to its type), 0 to ``weights`` and the token's number, seen
 * + i, to ``order`` where the cache has them, and new_state = (n, seen) plus
 * the new tokens. Tokens beyond the last slot are not kept (their queries
 * are still written). ``rotary`` NULL: nothing is rotated. x_dtype is
 * MOSAIC_F32 or the cache's type; qkv, q_out 16-byte aligned, ldx and ldq
 * multiples of 16 bytes; heads a multiple of kv_heads. */
mosaic_status mosaic_cache_append(const mosaic_kv_cache* cache, const void* qkv, int64_t ldx, int32_t x_dtype,
                                  int64_t rows, const int32_t* starts, int32_t heads, const mosaic_rotary* rotary,
                                  void* q_out, int64_t ldq, const int32_t* state, int32_t* new_state, void* stream);

/* One new token per sequence attends over its first n = min(lengths[b],
 * max_len) slots: for every query head g (key/value head h = g / (heads /
 * kv_heads))
 *     p_i = exp(scale q_g . k_i) / sum_j exp(scale q_g . k_j),
 *     out_g = sum_i p_i v_i,
 * zeros for a sequence without tokens. Infinities and NaN among the tokens act
 * as in these formulas (a score of -inf is no weight; zeros if there is no
 * other). Scores, softmax sums and outputs are accumulated in float32, outputs
 * before the division and with weights of up to 2^8: a value above 2^119 over
 * the number of tokens may overflow there. ``accumulate`` nonzero adds p_i of
 * every head of the group to ``weights`` of slot i and head h (without atomics:
 * two runs give the same bits). q and out are batch x heads * head_dim of
 * x_dtype (MOSAIC_F32 or the cache's type), 16-byte aligned, ldq and ldo
 * multiples of 16 bytes, not overlapping. lengths: batch entries, e.g. the
 * first row of the state. The workspace of a call that accumulates holds every
 * score, batch x heads x max_len floats: there max_len should be no larger than
 * it has to be. */
mosaic_status mosaic_cache_attend_workspace(const mosaic_kv_cache* cache, int32_t heads, int64_t max_len,
                                            int32_t accumulate, int64_t* bytes);
mosaic_status mosaic_cache_attend(const mosaic_kv_cache* cache, const void* q, int64_t ldq, int32_t x_dtype,
                                  int32_t heads, const int32_t* lengths, int64_t max_len, float scale,
                                  int32_t accumulate, void* out, int64_t ldo, void* workspace,
                                  int64_t workspace_bytes, void* stream);

/* Every sequence that holds n > budget tokens (n counted up to max_len) keeps
 * ``budget`` of them, for each key/value head by itself: first those of the
 * ``recent`` latest that its sequence has seen (order >= seen - recent), then
 * those of the largest weight (a NaN comes after every number), ties going to
 * the lowest slot. A slot below the budget whose page is not there can hold
 * none of them: as many fewer are kept, and the slot counts on as one in use
 * that holds nothing. Survivors in slots below the budget stay where they are;
 * the others, in the order of their slots, go to the slots below the budget
 * that came free, in theirs, with their weight and order. Pages from
 * ceil(budget / page_size) on then hold nothing. Weights and order of all
 * slots in use are written to new_weights and new_order, which may be the
 * cache's own arrays (then the survivors that stay are not rewritten) and may
 * not overlap them otherwise; new_state = (min(n, budget), seen). ``kept``
 * (batch x kv_heads x budget, or NULL) gets for every slot the slot that its
 * token had before, -1 for a slot without one or without a page. 1 <= budget, 0 <= recent <=
 * budget; the cache has weights and order. workspace 16-byte aligned. */
mosaic_status mosaic_cache_evict_workspace(const mosaic_kv_cache* cache, int64_t max_len, int64_t budget,
                                           int64_t* bytes);
mosaic_status mosaic_cache_evict(const mosaic_kv_cache* cache, const int32_t* state, int32_t* new_state,
                                 int64_t max_len, int64_t budget, int64_t recent, float* new_weights,
                                 int32_t* new_order, int32_t* kept, void* workspace, int64_t workspace_bytes,
                                 void* stream);

#ifdef __cplusplus
}
#endif

#endif /* MOSAIC_CACHE_H */
