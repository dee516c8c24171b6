/*
 * ssq_cache.h -- C ABI of libssq, third part: a paged cache held in 4 bits, and what is done with the
 * pages of any cache, for serving on AMD Instinct MI355X (gfx950).
 *
 * Beside the operators of ssq_attention.h, whose layouts and conventions these share (rows of heads and
 * their strides, tables, slots, alignment, checks on the host before any launch, nothing allocated or
 * kept):  with a cache in 4 bits, ssq_kv4_store follows ssq_qk_norm_rope (which then stores nothing) and
 * ssq_attention_decode_kv4 reads it.  Between steps, ssq_page_fork continues requests in others (beams,
 * samples), ssq_page_collect and ssq_page_compact find the free pages, and ssq_page_copy carries out
 * what they list.
 *
 * The cache in 4 bits -- the same pages, in 4.5 bits an element instead of 16 or 32: keys and
 * values on the signed absmax grid of ssq_quantize (q = 4), in groups of 32 elements along the
 * head, one binary16 scale each.  For groups w of a row,
 *   M = max|w|;  s = -M / 8 if max w > -min w, else M / 8   (binary32; +0 if M = 0)
 *   c = clip(rne(fl32(w / s)), -8, 7), 0 if M = 0;  held value = c * binary16(s).
 * (In binary32 rows of M <= 2^-147, s rounds to zero; there w = 0 has c = -8, as in ssq_quantize_f32.)
 * A group that holds an infinity or a NaN, or whose s binary16 does not reach (M >= 524160), has the
 * codes c = 0 and the scale NaN: all of it reads as NaN.
 *   cache  uint8 [pages, kv_heads, 2, page_size * (D/2 + D/16)], D = head_dim: for each page
 *          and head the keys, then the values, each page_size tokens' codes (D/2 bytes a
 *          token) and behind them their scales [page_size, D/32].  With u = c + 8, G = D/32:
 *          keys    word (4 bytes, little endian) h G + g of a token's codes holds elements
 *                  32 g + 8 h + (0..7), lowest in the lowest 4 bits
 *          values  byte 4 (x G + g) + i of four tokens' 2 D bytes holds, of the i-th, element
 *                  32 g + x in the low half and 32 g + 16 + x in the high half (x < 16).
 * Scales are finite or NaN; of others (nothing here writes them) only this is said, that
 * queries that do not see their key are not touched by them.
 */
#ifndef SSQ_CACHE_H
#define SSQ_CACHE_H

#include "ssq_attention.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * ssq_kv4_store -- keys and values of new tokens into their slots of a 4-bit cache, and, where
 * asked for, the values that the cache now holds for them (rounded to the rows' type, once).
 * With those a prompt's own attention sees what later steps will see.
 *
 *   k, v            device, bf16 [tokens, kv_heads, head_dim] (keys as ssq_qk_norm_rope
 *                   rotates them)
 *   tokens          >= 0; ceil(tokens * head_dim / 2048) * kv_heads < 2^24
 *   slots           device, int32 [tokens]: page * page_size + offset; a slot outside
 *                   [0, pages * page_size) is not stored.  Two tokens of a call must not have
 *                   the same slot (what it then holds is a mixture of both).  Bytes of other
 *                   slots stay as they are.
 *   cache, pages, page_size   the cache; at most 2^31 - 1 slots
 *   k_held, v_held  device, bf16, written, or NULL; may be k and v themselves with their
 *                   strides, and where k and v are the same rows, the same rows too
 * No other array that is written, the cache among them, may overlap another argument's.  Rows may lie
 * between those of another array, as in the rows of one projection.
 */
int ssq_kv4_store(const uint16_t* k, int64_t k_stride, const uint16_t* v, int64_t v_stride,
                  int64_t tokens, int kv_heads, int head_dim, const int32_t* slots, uint8_t* cache,
                  int64_t pages, int page_size, uint16_t* k_held, int64_t k_held_stride,
                  uint16_t* v_held, int64_t v_held_stride, hipStream_t stream);

/* ssq_kv4_store for binary32 rows; the cache is the same. */
int ssq_kv4_store_f32(const float* k, int64_t k_stride, const float* v, int64_t v_stride,
                      int64_t tokens, int kv_heads, int head_dim, const int32_t* slots, uint8_t* cache,
                      int64_t pages, int page_size, float* k_held, int64_t k_held_stride,
                      float* v_held, int64_t v_held_stride, hipStream_t stream);

/*
 * ssq_attention_decode_kv4 -- ssq_attention_decode over a 4-bit cache; arguments, positions, the
 * shared prefix, absent pages and the workspace are those of ssq_attention_decode, but
 * requests * (fresh * q_heads + 16 kv_heads) < 2^28.
 * Codes enter the products exactly and scales in binary32.  In bf16, weight times value scale is
 * rounded to bf16 for the product with the codes, each of a row's D/32 groups for itself; the sum that
 * divides them is that of the unrounded weights.  Codes enter bf16 products with an offset that is taken
 * out again in binary32: queries of magnitude 2^114 and above may overflow there and give NaN.  In binary32 nothing is rounded to fewer bits.
 */
int ssq_attention_decode_kv4(const uint16_t* q, int64_t q_stride, int64_t requests, int fresh,
                             int q_heads, int kv_heads, int head_dim, float scale, const uint8_t* cache,
                             int64_t pages, int page_size, const int32_t* table, int64_t table_stride,
                             const int32_t* lens, int64_t max_len, int64_t prefix, uint16_t* out,
                             int64_t out_stride, void* workspace, size_t workspace_bytes,
                             hipStream_t stream);

/* ssq_attention_decode_kv4 for binary32 q and out; the cache is the same. */
int ssq_attention_decode_kv4_f32(const float* q, int64_t q_stride, int64_t requests, int fresh,
                                 int q_heads, int kv_heads, int head_dim, float scale, const uint8_t* cache,
                                 int64_t pages, int page_size, const int32_t* table, int64_t table_stride,
                                 const int32_t* lens, int64_t max_len, int64_t prefix, float* out,
                                 int64_t out_stride, void* workspace, size_t workspace_bytes,
                                 hipStream_t stream);

/* Bytes of workspace for ssq_attention_decode_kv4 and its _f32 form with these sizes; 0 where
 * nothing would be split, or for invalid sizes. */
size_t ssq_attention_decode_kv4_workspace_size(int64_t requests, int fresh, int q_heads, int kv_heads,
                                               int head_dim, int64_t max_len, int64_t prefix);

/*
 * ssq_page_fork -- the tables of requests that continue others: beams after a step's selection,
 * several samples of one prompt, the rows that stay when others leave, in any order.
 * Request i continues row p = parents[i] of the table, whose lens[p] tokens lie in
 * n = ceil(lens[p] / page_size) pages:
 *   table_out[i, j] = table[p, j]                     for j < n, -1 behind
 *   lens_out[i]     = lens[p]
 * Whole pages are shared.  The last page, where it is not full, stays with the first request that
 * continues p; every other gets a new page in its place, from entry *taken of the list of free
 * pages on, request after request, and
 *   src[i] = the page that p has there,  dst[i] = the new page
 * say what has to be copied into it (ssq_page_copy, once for all layers); both are -1 where nothing has.
 * *taken_after = *taken plus the new pages.  Rows that nobody continues are dropped: their pages
 * are those that ssq_page_collect then finds free.
 *
 *   parents     device, int32 [requests]; outside [0, rows): an empty row of length 0
 *   requests, rows   0 to 2^14
 *   lens        device, int32 [rows]; negative values count as 0
 *   table       device, int32 [rows, table_stride]
 *   free_pages  device, int32 [free_count]; may be NULL if free_count is 0
 *   taken       device, int32 [1], or NULL for 0
 *   table_out   device, int32 [requests, table_out_stride], all of it written
 *   lens_out, src, dst   device, int32 [requests], written
 *   taken_after device, int32 [1], written
 * No array that is written may overlap another argument's.  Pages past the end of the list are the
 * entry -1, nothing to copy (then *taken_after > free_count).  A last page that a row has no room
 * for, or whose entry is negative, is neither replaced nor counted.
 */
int ssq_page_fork(const int32_t* parents, int64_t requests, const int32_t* lens, const int32_t* table,
                  int64_t rows, int64_t table_stride, const int32_t* free_pages, int64_t free_count,
                  const int32_t* taken, int page_size, int32_t* table_out, int64_t table_out_stride,
                  int32_t* lens_out, int32_t* src, int32_t* dst, int32_t* taken_after,
                  hipStream_t stream);

/*
 * ssq_page_collect -- the list of free pages: those of [0, pages) that no request's row names among its
 * first ceil(lens / page_size) entries and that are not pinned, ascending, then -1.  Requests
 * that have ended are left out, or have the length 0.  The list is one for ssq_page_tables and
 * ssq_page_fork, from entry 0 on.
 *
 *   requests    0 to 2^20 (up to 2048, and up to 131072 pages, in one or three launches instead of four or seven)
 *   lens        device, int32 [requests]; negative values count as 0.  lens and table may be NULL if
 *               requests or table_stride is 0
 *   table       device, int32 [requests, table_stride]; entries outside [0, pages) name none;
 *               requests * ceil(table_stride / 1024) < 2^24
 *   pages       pages of the pool; pages * page_size < 2^31
 *   pinned      device, uint8 [pages], or NULL: pages with a value other than 0 are held whether
 *               a request names them or not (a system prompt kept without a user)
 *   free_pages  device, int32 [pages], written
 *   count       device, int32 [1], written: free pages
 *   workspace   device, 256-byte aligned, ssq_page_collect_workspace_size(pages, 0) bytes, in any state
 * No array that is written may overlap another argument's.  Two calls that may run concurrently must
 * not share a workspace.
 */
int ssq_page_collect(const int32_t* lens, int64_t requests, const int32_t* table, int64_t table_stride,
                     int page_size, int64_t pages, const uint8_t* pinned, int32_t* free_pages,
                     int32_t* count, void* workspace, size_t workspace_bytes, hipStream_t stream);

/*
 * ssq_page_compact -- ssq_page_collect with the held pages brought to the front of the pool: with U held
 * pages, those at or above U that are not pinned move, ascending, into the free pages below U,
 * ascending.
 *   src[k] -> dst[k]   the moves, -1 behind them (ssq_page_copy, for every layer, before the cache is next used)
 *   table_out          the table with the pages' new numbers; entries that name none (see
 *                      ssq_page_collect) stay as they are
 *   free_pages, count  the free pages after the moves
 *
 *   table_out   device, int32 [requests, table_stride], written; may be `table` itself
 *   src, dst    device, int32 [pages / 2], written
 *   moved       device, int32 [1], written: moves
 *   workspace   of ssq_page_collect_workspace_size(pages, 1) bytes
 */
int ssq_page_compact(const int32_t* lens, int64_t requests, const int32_t* table, int64_t table_stride,
                     int page_size, int64_t pages, const uint8_t* pinned, int32_t* table_out,
                     int32_t* free_pages, int32_t* count, int32_t* src, int32_t* dst, int32_t* moved,
                     void* workspace, size_t workspace_bytes, hipStream_t stream);

/* Bytes of workspace for ssq_page_collect (compact 0) or ssq_page_compact; 0 for invalid sizes. */
size_t ssq_page_collect_workspace_size(int64_t pages, int compact);

/*
 * ssq_page_copy -- page src[i] of every cache into its page dst[i], for all i at once.
 *
 *   caches      host array of `count` (0 to 2^16) device pointers, 16-byte aligned, each
 *               [pages, page_bytes]: a layer's k_pages and v_pages, or its 4-bit cache
 *   page_bytes  multiple of 16, at most 2^30
 *   src, dst    device, int32 [entries], in none of the caches; an entry of which either is outside
 *               [0, pages) is skipped, as is one of a page to itself
 *   entries     0 to 2^30
 * No page may be named twice in dst, or both in src and in dst (those of ssq_page_fork and
 * ssq_page_compact are not): it would hold a mixture.  No two caches may overlap, but one may be named twice.
 */
int ssq_page_copy(void* const* caches, int count, int64_t page_bytes, int64_t pages, const int32_t* src,
                  const int32_t* dst, int64_t entries, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* SSQ_CACHE_H */
