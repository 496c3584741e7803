/* freekv_cache.h -- a paged cache in 4 bits for many sequences, and the attention over it.
 *
 * Beside the retrieval contexts of freekv.h (one context length for all requests, pages in 16 bits that belong to one
 * request), a cache of this kind holds sequences of any lengths in one pool of pages, in 4 bits:
 *   - a page is 32 consecutive tokens of a sequence, their keys and values in all layers and KV heads.  Pages are shared:
 *     a page belongs to every sequence whose page table names it, and goes back to the pool with the last of them.
 *   - a sequence's last, partial page is open: its tokens are kept in 16 bits, per sequence.  With its 32nd token a page
 *     becomes full: it is put into the pool in 4 bits and never changes again, so sequences share full pages as they are.
 *
 * The 4 bits.  For every layer, KV head and page, keys and values apart; x_tc is token t's channel c, T the storage type:
 *     lo_c   = min_t x_tc                          in T (exact)
 *     w_c    = (max_t x_tc - lo_c) / 15            rounded to fp32
 *     E      = floor(log2(max_c w_c)), at least -126; 0 if every w_c is 0
 *     step_c = fp16(w_c 2^-E) 2^E                  one exponent for the 128 channels, so that any range of T fits
 *     code   = round((x_tc - lo_c) / step_c)       of the exact quotient, ties to even, held to 0..15; 0 where step_c is 0
 * and the cache stands for lo_c + step_c code.  A scale per channel, because keys and values have a few channels that are
 * larger than the others at every token.  A channel that holds a NaN or an infinity in a page stands for NaN at all 32 tokens.
 * A page of a KV head is 5120 bytes and an exponent, 16384 bytes in T.
 *
 * State lives on the device.  Lengths, page tables, reference counts and the free pages are in the arena, and the calls
 * below only enqueue kernels that read and change them, but for those that say that they are blocking: page ids never pass through
 * the host, and captured into a graph every replay does the work again on the state of that time.  What only the device can see
 * to be wrong (a slot that does not exist, a pool without room) makes no access: the entry, or the whole call where it says so,
 * does nothing, and fkv_cache_health reports it.
 *
 * Conventions are those of freekv.h: 0 or a negative FKV_E* code, fkv_cache_last_error for the text, `stream` a hipStream_t,
 * device pointers.  A call launches on the cache's device, whichever is current.  The calls on one cache (on either, for
 * fkv_cache_copy) have to follow each other: on one stream, or ordered by the caller.  The same goes for graphs that
 * hold such calls: two graphs of one cache must not run at once.
 *
 * Rows.  `seqs` is a device array of n_rows slot numbers, 0 <= slot < max_seqs; -1 is a row of padding, which is passed over.
 * Tokens of rows lie behind each other: `cu` is a device array of n_rows + 1 ascending token offsets that starts at 0, row i
 * has tokens cu[i] to cu[i + 1] - 1.  cu == NULL: one token a row.
 */
#ifndef FREEKV_CACHE_H
#define FREEKV_CACHE_H

#include "freekv.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct fkv_cache fkv_cache;

typedef struct {
  int32_t n_layers;
  int32_t n_q_heads;
  int32_t n_kv_heads;      /* G = n_q_heads / n_kv_heads, 1 <= G <= 16              */
  int32_t head_dim;        /* must be 128                                           */
  int32_t page_size;       /* must be 32                                            */
  int32_t max_seqs;        /* sequence slots, 1 to 4096; also the most rows of a call */
  int32_t max_ctx;         /* most tokens of a sequence, a multiple of page_size    */
  int32_t n_pages;         /* pages of the pool                                     */
  int32_t dtype;           /* FKV_DTYPE_*: of q, K, V and the outputs                */
} fkv_cache_config;        /* n_layers * max_seqs * n_kv_heads: at most 8388608      */

/* Bytes of device memory that such a cache needs: the pool, 16 KiB per layer, slot and KV head for open pages, tables,
 * and the workspace of attention. */
int fkv_cache_arena_bytes(const fkv_cache_config* cfg, size_t* dev_bytes);
/* An empty cache on the current device.  dev_arena: device memory, 256-byte aligned, >= dev_bytes; the caller's, to be kept
 * as long as the cache.  Blocking. */
int fkv_cache_create(const fkv_cache_config* cfg, void* dev_arena, size_t dev_bytes, fkv_cache** out);
/* Blocking: the arena may be freed behind it. */
int fkv_cache_destroy(fkv_cache* cache);
/* Text of the last error of this cache (cache == NULL: of this thread's last failed create or arena_bytes). */
const char* fkv_cache_last_error(const fkv_cache* cache);

/* What the device refused since the last call: FKV_ENOMEM (a fkv_cache_extend or fkv_cache_copy found too few free pages
 * and did nothing), FKV_ERANGE (a row would have grown past max_ctx and did not), FKV_EINVAL (a slot out of range or twice
 * in one call, tokens that do not match the row's last fkv_cache_extend, a target slot that was not empty), in this order;
 * clears it.  Blocking: synchronises the device. */
int fkv_cache_health(fkv_cache* cache);
/* Pages in use, or a negative code.  Blocking. */
int fkv_cache_used_pages(fkv_cache* cache);

/* Room for new tokens: row i's sequence becomes cu[i + 1] - cu[i] tokens longer, once for all layers, and gets a page of the
 * pool for every page that these tokens fill: the lowest free ones, in the order of the rows and of their pages.  A row
 * that would pass max_ctx stays as it is; if the pool has too few pages for the others, all stay as they are.  Until a layer's
 * fkv_cache_append, the new tokens hold anything in that layer. */
int fkv_cache_extend(fkv_cache* cache, const int32_t* seqs_dev, int32_t n_rows, const int32_t* cu_dev, void* stream);

/* The new tokens' keys and values in one layer: k, v dev [n_tokens, n_kv, d], 16-byte aligned, row i's being the tokens that its
 * last fkv_cache_extend made room for (same rows, same cu).  Pages that they fill are put into the pool in 4 bits, the
 * rest into the open page.  Once per layer after each extend; a row for which that does not hold is dropped, and so is one whose
 * extend was refused.  Between an extend and the last layer's append the sequences must not be forked, copied or freed. */
int fkv_cache_append(fkv_cache* cache, int32_t layer, const int32_t* seqs_dev, int32_t n_rows, const int32_t* cu_dev,
                     const void* k_dev, const void* v_dev, int32_t n_tokens, void* stream);

/* o_h = softmax(q_h K^T / sqrt(d)) V over what the cache holds of row i's sequence, one query token a row:
 * q, out dev [n_rows, n_q, d] of T, 16-byte aligned.  Several rows may name one sequence.
 *   pages_dev  NULL: every token.  Otherwise dev [n_rows, n_kv, n_list] i32, per KV head the positions (page 0 holds tokens
 *              0 to 31) of the full pages to attend, in the form of fkv_page_select's lists, next to the first sink_tokens and the
 *              last window_tokens tokens' full pages (both multiples of page_size, the sink first if they overlap) and the
 *              open page, which are attended always.  Entries that are not a full page between sink and window
 *              (-1, say) are passed over; one that is listed twice counts twice.  n_list: 0 to 131072.
 * Branches read pages that they shared at their last fork together, 16 / G rows at most at a time, whatever the rows' order, in
 * calls without lists of 2 to 64 rows with G <= 8, where they share 8 pages or more and the rows have more than 4096 / n_kv pages in
 * all.  The cache must have been forked by then: a graph that was captured before its first fork reads each row's pages for itself, as does
 * every other call.  The result is the same up to rounding.
 * Logits, softmax and sums are in fp32, the output is rounded once.  bf16 outputs of less than 2^-98 lose digits; values of any size
 * do not overflow up to 2^22 tokens that weigh about the same.  A row that has nothing to attend (padding, an empty sequence,
 * an empty list), or whose logits are all minus infinity, gets zeros.  An infinite value in the open page gives an infinity, NaN where
 * its token weighs less than 2^-30 of the largest. */
int fkv_cache_attn(fkv_cache* cache, int32_t layer, const int32_t* seqs_dev, int32_t n_rows, const void* q_dev,
                   const int32_t* pages_dev, int32_t n_list, int32_t sink_tokens, int32_t window_tokens, void* out_dev,
                   void* stream);

/* What the cache stands for of row i's first cu[i + 1] - cu[i] tokens in one layer, rounded to T: k, v dev
 * [n_tokens, n_kv, d], 16-byte aligned.  Places behind a sequence's end are left as they are. */
int fkv_cache_read(fkv_cache* cache, int32_t layer, const int32_t* seqs_dev, int32_t n_rows, const int32_t* cu_dev,
                   void* k_dev, void* v_dev, int32_t n_tokens, void* stream);

/* Sequence dst[i] becomes what src[i] is, for i < n: it shares src's full pages and gets a copy of its open page.  dst[i] must be
 * empty when the call begins; a slot may be the source of many.  An entry whose source or target is -1 is padding. */
int fkv_cache_fork(fkv_cache* cache, const int32_t* src_dev, const int32_t* dst_dev, int32_t n, void* stream);

/* The same with pages of its own: sequence src[i] of `from` is copied to the empty slot dst[i] of `to`, into the lowest free
 * pages of to's pool, in order.  from and to may be one cache; otherwise they are of one device, and layers,
 * heads and types are the same (a larger pool takes over a smaller one's sequences so).  A sequence longer than to's max_ctx
 * is passed over; if `to` has too few pages, nothing is copied.  Refusals are reported by `to`'s health. */
int fkv_cache_copy(fkv_cache* from, const int32_t* src_dev, fkv_cache* to, const int32_t* dst_dev, int32_t n, void* stream);

/* The sequences become empty; pages that no other sequence shares go back to the pool. */
int fkv_cache_free(fkv_cache* cache, const int32_t* seqs_dev, int32_t n, void* stream);

/* Moves the used pages with the highest numbers to the lowest free places, in order, until the pages in use are the first
 * ones of the pool.  Page tables follow; what the sequences hold stays the same. */
int fkv_cache_compact(fkv_cache* cache, void* stream);

/* For each row its sequence's length and page ids: lens_dev dev [n_rows] i32, pages_dev dev [n_rows, max_ctx / page_size] i32,
 * -1 behind the last full page, or NULL: the lengths alone.  Padding: length 0. */
int fkv_cache_tables(fkv_cache* cache, const int32_t* seqs_dev, int32_t n_rows, int32_t* lens_dev, int32_t* pages_dev,
                     void* stream);

#ifdef __cplusplus
}
#endif
#endif /* FREEKV_CACHE_H */
