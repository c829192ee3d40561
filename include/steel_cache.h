/*
 * steel_cache.h — C ABI of the paged 4-bit key/value cache that stands beside the prefill attention of
 * steel_attn.h: tokens are quantised into pages (append), given back in bf16 in the layout that
 * steel_attn_run takes (read), attended to by the few new tokens of a step (attend), and the pages are
 * shared, copied, given back and moved on the device (extend, fork, free, compact).
 *
 * Everything that a step changes lives in device memory — table, lengths, reference counts — so that a
 * step needs no host synchronisation and can be captured into a CUDA graph and replayed while
 * sequences grow.
 *
 * Quantiser.  The head_dim channels of a token's key (equally value) of one head form groups of 64.  With x
 * clamped to +-65504, of each group:
 *
 *     zero = f16(min x)      scale = f16(f32((max x - min x) / 15))
 *     code = clamp(round_half_even((x - zero) / scale), 0, 15), 0 where scale = 0
 *     value = scale * code + zero
 *
 * 4.5 bits a value.  The quotient is rounded as if it were exact.  A group that holds a NaN gets scale = zero =
 * NaN: its token's values read as NaN, as they would in a cache that is not quantised.
 *
 * Memory, all of it the caller's.  `pool` is [layers][pages][heads_kv][page_tokens / 16][unit]; a unit holds 16
 * tokens of one head in the order in which the tensor cores take them, so that a lane's operands are 16 bytes
 * side by side.  With n = head_dim / 64 groups a unit is, in bytes: 512 n of K codes, 512 n of V codes, 64 n of
 * K scales, 64 n of V scales:
 *
 *     K codes   32-bit words [group n][g 8][t 4][c 2][h 2]: token 8h + g, nibble i = channel 64 group + 32c + 8t + i
 *     V codes   16-bit words [group n][g 8][t 4][h 2][y 2][f 2]: token 8h + 2t + f, nibble i = channel 64 group + 8g + 4y + i
 *     K scales  fp16 pairs (scale, zero) [g 8][h 2][group n]: token 8h + g;     V scales  the same
 *
 * `table` int32 [slots][max_pages]: page of token j of a slot at column j / page_tokens, -1 behind the last.
 * `lens` int32 [slots]: tokens of each slot; it holds ceil(lens / page_tokens) pages.
 * `refs` int32 [pages]: how many table entries name the page; 0 = free.
 * `status` int32: what went wrong on the device (below).   `scratch`: working memory of the calls that change pages.
 *
 * Batches.  `slots` (DEVICE int32 [batch], NULL = 0, 1, 2, ...) says which slots a call is about.  The calls that
 * write want distinct slots; read and attend take a slot several times, in batches of up to 65535 (beyond: STEEL_ERR_UNSUPPORTED).
 *
 * Errors on the device.  A slot outside the cache, a count or length that cannot be, a slot named twice where they
 * have to be distinct, a table entry outside the pool: the status word is set to STEEL_ERR_INVALID_ARG; too few free
 * pages: STEEL_ERR_NO_PAGES; an expired wait: STEEL_ERR_TIMEOUT.  extend, fork and free then change nothing at all (fork and free: but for a
 * table entry outside the pool, which is not counted); append, read and attend leave out the sequences concerned (attend: their output is
 * undefined).  No memory outside the tensors is touched, nothing traps.  steel_cache_last_status reads and clears the word.
 *
 * Streams.  Every call is asynchronous on `cuda_stream`.  Calls that change pages (extend, fork, free, compact, reset) or write
 * tokens (append) must be ordered with each other and with the calls that read what they change; they share
 * `scratch`.  attend and read may overlap with each other on several streams; attend takes a workspace per
 * call.  The object is bound to the device that is current at create; a call with another current device is refused.
 * All functions return a status code; nothing throws, aborts or traps.
 */
#ifndef STEEL_CACHE_H_
#define STEEL_CACHE_H_

#include <stdint.h>

#include "steel_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct steel_cache steel_cache_t; /* opaque, owned by the library */

typedef struct {
  int32_t layers;      /* 1 ... 4096                                                     */
  int32_t pages;       /* 1 ... 2^20; one page holds page_tokens tokens, all KV heads, of every layer */
  int32_t page_tokens; /* 16, 32, 64 or 128                                              */
  int32_t heads_kv;    /* 1 ... 1024                                                     */
  int32_t head_dim;    /* 64 or 128                                                      */
  int32_t slots;       /* 1 ... 8192 sequences                                           */
  int32_t max_pages;   /* 1 ... 2^20 pages a sequence; max_pages * page_tokens <= 2^30, and * heads_kv / 16 < 2^30 */
} steel_cache_params_t;

typedef struct {
  int64_t pool_bytes, table_bytes, lens_bytes, refs_bytes, status_bytes, scratch_bytes;
  int64_t unit_bytes, page_bytes; /* of one layer */
} steel_cache_sizes_t;

typedef struct { /* DEVICE pointers; pool, scratch and status 128-byte aligned */
  void *pool;
  int32_t *table, *lens, *refs, *status;
  void *scratch;
} steel_cache_memory_t;

/* A bf16 tensor [batch, heads, seq, head_dim] of the caller: base (16-byte aligned) and strides in elements
 * (multiples of 8, at most 2^40); the last dimension is contiguous. */
typedef struct {
  void *data;
  int64_t stride_batch, stride_head, stride_seq;
} steel_cache_tensor_t;

/* Bytes of each part of the memory that the caller provides. */
steel_status_t steel_cache_sizes(const steel_cache_params_t *params, steel_cache_sizes_t *sizes);

/* Checks the arguments and binds the memory; nothing is allocated on the device and nothing is written there:
 * call steel_cache_reset, or bring table, lens and refs of an earlier cache and a status of 0.  *out is NULL on failure. */
steel_status_t steel_cache_create(const steel_cache_params_t *params, const steel_cache_memory_t *memory,
                                  steel_cache_t **out);
/* destroy(NULL) is STEEL_OK.  The memory stays the caller's. */
steel_status_t steel_cache_destroy(steel_cache_t *cache);

/* An empty cache: table -1, lens, refs and status 0. */
steel_status_t steel_cache_reset(steel_cache_t *cache, void *cuda_stream);

/*
 * Room for counts[i] more tokens (DEVICE int32 [batch], >= 0) of each slot: lens grows by counts[i], pages are taken where needed,
 * the lowest free page first in the order of the batch and of the tokens.  Where a slot's last page is partly filled and has
 * refs > 1 when the call begins, and counts[i] > 0, the slot gets a page of its own in its place, into which the 16-token units that hold
 * tokens are copied in every layer.  All or nothing: with too few free pages, or a length beyond max_pages, nothing changes.
 * The contents of new tokens are undefined until append writes them.
 */
steel_status_t steel_cache_extend(steel_cache_t *cache, int32_t batch, const int32_t *slots, const int32_t *counts,
                                  void *cuda_stream);

/*
 * Quantise the last counts[i] tokens (NULL = seq) of each slot, for which extend has made room: token j < counts[i] of the
 * batch's sequence i (0 <= counts[i] <= seq <= 2^30) goes to position lens[slot] - counts[i] + j.  Of k and v only those rows are read.
 * A token whose page other table entries name too (refs > 1: the slot was forked and not extended) is not written, and reported.
 */
steel_status_t steel_cache_append(steel_cache_t *cache, int32_t layer, int32_t batch, const int32_t *slots,
                                  const int32_t *counts, int32_t seq, const steel_cache_tensor_t *k,
                                  const steel_cache_tensor_t *v, void *cuda_stream);

/*
 * Keys and values in bf16: token begin[i] + j (NULL = j), for j < seq and as far as the slot has tokens, goes to row j of the batch's
 * sequence i.  Rows behind are left as they were.  k and v as steel_attn_run takes them, or with strides.
 */
steel_status_t steel_cache_read(steel_cache_t *cache, int32_t layer, int32_t batch, const int32_t *slots,
                                const int32_t *begin, int32_t seq, const steel_cache_tensor_t *k,
                                const steel_cache_tensor_t *v, void *cuda_stream);

typedef struct {
  int32_t layer, batch, heads_q, seq_q; /* heads_q a multiple of heads_kv; query head h reads KV head h / (heads_q / heads_kv) */
  const int32_t *slots;                 /* DEVICE [batch] or NULL                                                      */
  const int32_t *counts;                /* DEVICE [batch] or NULL: queries of each sequence, 0 ... seq_q (NULL: seq_q)  */
  uint32_t flags;                       /* STEEL_MASK_CAUSAL, STEEL_MASK_WINDOW or both, or 0                           */
  float scale;                          /* finite, > 0                                                                 */
  int64_t window;                       /* > 0, used iff WINDOW                                                        */
  steel_cache_tensor_t q;               /* [batch, heads_q, seq_q, head_dim]                                           */
  void *o;                              /* bf16 [batch, heads_q, seq_q, head_dim], contiguous, 16-byte aligned, not q   */
  float *lse;                           /* float32 [batch, heads_q, seq_q] or NULL                                     */
  void *workspace;                      /* 128-byte aligned, of steel_cache_attend_workspace bytes; not shared between  */
  int64_t workspace_bytes;              /* calls that may overlap (graphs captured with it included)                   */
} steel_cache_attend_t;

/*
 * Attention of each sequence's newest tokens over the cache.  Query i < counts[b] of sequence b stands at position
 * p = lens - counts[b] + i; key j is visible iff j < lens and, with CAUSAL, j <= p, with WINDOW, p - j < window (the predicate of
 * steel_attn.h with seq_q = counts[b], seq_kv = lens).
 *     O = softmax_j(scale q . k_j) V,  LSE = ln sum_j exp(scale q . k_j);  no visible key: O = 0, LSE = -inf.
 * Scores are meant to be below 2^26 in magnitude: beyond, a weight may leave the range of 32 bits.
 * What is rounded: a weight times the scale of a group of V to fp16 (2^-11 of it; the power of two beside it is the row's own), O to bf16 (2^-8).
 * Scores, weights, LSE and all sums are in 32 bits.  Codes are summed apart from zeros for up to 512 tokens at a time, so the first rounding counts
 * about 2.5 times; that is a third of the second or less.  Matrix products cut their sums off by 2^-23.4 each, one way: 0.02 % of O for each
 * 32768 tokens that one warp goes through (the whole call's steps are dealt out evenly to about 2400 warps).
 * Rows i >= counts[b] are left as they were.  A key that a query does not see has no influence on it but by rounding, whatever its
 * contents, NaN among them.  For a few queries a sequence: 8 rows (queries times query heads of a KV head) go through the cache together,
 * more rows several times; a long chunk of a prompt is better served by steel_cache_read and steel_attn_run.
 * The result does not depend on what else is in the batch but by rounding, and is the same for the same call each time.
 * STEEL_ERR_UNSUPPORTED: more than 2^24 rows (seq_q times the query heads of a KV head), or about 2^30 and more pairs of (8 rows,
 * 32 tokens) if every sequence of the batch were as long as the cache has room for.
 */
steel_status_t steel_cache_attend(steel_cache_t *cache, const steel_cache_attend_t *args, void *cuda_stream);

/* Bytes of workspace that attend wants for these sizes (a negative number: bad arguments). */
int64_t steel_cache_attend_workspace(const steel_cache_t *cache, int32_t batch, int32_t heads_q, int32_t seq_q);

/*
 * Slot dst[i] gives up its pages and holds the same pages as src[i] did when the call began (DEVICE int32 [n], n <= slots): beams
 * that take over their parents, prompts that share a prefix.  src may name a slot several times, and slots of dst too; dst are distinct.
 */
steel_status_t steel_cache_fork(steel_cache_t *cache, int32_t n, const int32_t *src, const int32_t *dst,
                                void *cuda_stream);

/* Keep the first keep[i] tokens of each slot (NULL = none; 0 <= keep[i] <= lens) and give back the pages behind them. */
steel_status_t steel_cache_free(steel_cache_t *cache, int32_t batch, const int32_t *slots, const int32_t *keep,
                                void *cuda_stream);

/*
 * Move pages so that the pages in use are 0 ... live - 1: the k-th page in use from `live` up goes into the k-th free one
 * below, in every layer; table and refs follow.  `live` (DEVICE int32, may be NULL) receives the number of pages in use.
 * A table entry whose page has no count, or lies outside the pool, stays as it is; it is reported if any page moves.
 */
steel_status_t steel_cache_compact(steel_cache_t *cache, int32_t *live, void *cuda_stream);

/*
 * Test hook for attend's bounded wait of one CTA for the others' parts of a sequence: in this cache's following calls it ends after
 * `cycles` SM cycles (0: after one look; < 0: the default, about two seconds; at most 2^46).  The kernel then returns normally, the output is
 * undefined and steel_cache_last_status reports STEEL_ERR_TIMEOUT.  A captured call keeps the bound that it was captured with.
 */
steel_status_t steel_cache_debug_wait(steel_cache_t *cache, int64_t cycles);

/* Synchronise `cuda_stream`, then report and clear the status word. */
steel_status_t steel_cache_last_status(steel_cache_t *cache, void *cuda_stream);

#ifdef __cplusplus
}
#endif
#endif /* STEEL_CACHE_H_ */
