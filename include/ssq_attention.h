/*
 * ssq_attention.h -- C ABI of libssq, second part: what a transformer layer computes
 * between its q/k/v and o projections (ssq_matmul of ssq.h), for serving on AMD
 * Instinct MI355X (gfx950).
 *
 * A step of a serving loop runs, per layer,
 *   ssq_matmul (q, k, v) -> ssq_qk_norm_rope -> ssq_attention_prompt or
 *   ssq_attention_decode -> ssq_matmul (o)
 * and once per step, before the first layer, ssq_page_tables.
 *
 * Layouts (shared by every entry point)
 * --------------------------------------
 *   q, out    [tokens, q_heads, head_dim]   rows of one token contiguous, consecutive
 *   k, v      [tokens, kv_heads, head_dim]  tokens `*_stride` elements apart, so that
 *                                           the rows of one fused projection can be
 *                                           passed as they are
 *   k_pages,  [pages, kv_heads, page_size, head_dim]
 *   v_pages                                 the paged cache: page_size tokens a page
 *   slots     int32: page * page_size + offset, the place of one token in the cache
 *   table     int32 [requests, table_stride]: the pages of each request, in order
 *   q_heads = group * kv_heads: query heads h * group ... h * group + group - 1 read
 *   key/value head h.  head_dim is 64 or 128, page_size a power of two from 16 to 1024.
 *
 * Conventions are those of ssq.h: device pointers owned by the caller, bf16 as uint16_t
 * bits, arguments validated on the host before any launch, calls asynchronous on
 * `stream`, nothing allocated and nothing kept.  Besides:
 *   - q, k, v, outputs, caches, gains and rotation tables must be 16-byte aligned and
 *     their strides multiples of 16 bytes; integer arrays 4-byte aligned.
 *   - What lies in device memory cannot be validated on the host: lengths, page numbers,
 *     slots and positions outside their range are handled as each entry point says, and
 *     never cause an access outside the arrays that were passed.
 *   - Keys that a query does not see have no influence on its result, whatever their
 *     bits (infinities and NaN included): it is the same to the last bit.  A query that
 *     sees no key gives zeros; one whose scores are all -infinity gives NaN.
 *   - Up to 2^20 requests are taken, but the calls are made for some thousands: each
 *     workgroup of ssq_attention_prompt and ssq_page_tables walks the requests' starts or
 *     lengths (64 and 1024 at a time) up to its own, so their time grows with the square.
 */
#ifndef SSQ_ATTENTION_H
#define SSQ_ATTENTION_H

#include "ssq.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * ssq_page_tables -- the page table, slots and positions of one step's new tokens.
 *
 * Request r holds `held[r]` tokens in ceil(held[r] / page_size) pages, the first entries
 * of its table row, and adds `added[r]`.  Pages it needs beyond those come from the list
 * of free pages, request after request, starting at entry *taken:
 *   first[r]    = *taken + sum_{i < r} (want[i] - have[i]),
 *   have, want  = ceil(held / page_size), ceil((held + added) / page_size)
 *   table[r, j] = free_pages[first[r] + j - have[r]]        for have[r] <= j < want[r]
 *   starts[r]   = sum_{i < r} added[i];  lens[r] = held[r] + added[r]
 * and for token t = starts[r] + i of request r (i < added[r])
 *   positions[t] = held[r] + i
 *   slots[t]     = table[r, positions[t] / page_size] * page_size + positions[t] % page_size.
 * Tokens t >= starts[requests] are padding: position 0, slot -1.
 *
 *   held, added  device, int32 [requests]; negative values count as 0
 *   requests     0 to 2^20
 *   free_pages   device, int32 [free_count]; may be NULL if free_count is 0
 *   taken        device, int32 [1], or NULL for 0: entries of the list used up before
 *   page_size    power of two, 16 to 1024
 *   table        device, int32 [requests, table_stride], read, and written where pages
 *                are added; a row's other entries stay
 *   table_stride pages that a row has room for
 *   tokens       length of positions and slots
 *   starts       device, int32 [requests + 1], written
 *   lens         device, int32 [requests], written
 *   positions    device, int32 [tokens], written
 *   slots        device, int32 [tokens], written
 *   taken_after  device, int32 [1], written: *taken plus all pages needed
 * No array that is written (`table` among them) may overlap another argument's, which
 * workgroups still read: the `lens` and *taken_after of one call are `held` and *taken of
 * a later one, in buffers of their own, not in the same call's.
 * Pages past the end of the list get the entry -1 and their tokens the slot -1 (then
 * *taken_after > free_count); so do tokens past a row's table_stride pages, whose pages
 * are counted and not stored.  Sums are those of 32-bit two's complement: fewer than
 * 2^31 tokens and pages in all.
 */
int ssq_page_tables(const int32_t* held, const int32_t* added, int64_t requests,
                    const int32_t* free_pages, int64_t free_count, const int32_t* taken,
                    int page_size, int32_t* table, int64_t table_stride, int64_t tokens,
                    int32_t* starts, int32_t* lens, int32_t* positions, int32_t* slots,
                    int32_t* taken_after, hipStream_t stream);

/*
 * ssq_qk_norm_rope -- for each token and head of q and k, in one pass:
 *   n = x / sqrt(mean(x^2) + eps) * gain          (gain given; else n = x)
 *   out[i]       = n[i] cos - n[i + D/2] sin,      i < D/2 = head_dim / 2
 *   out[i + D/2] = n[i + D/2] cos + n[i] sin,      cos, sin = rope[position][i], rope[position][i + D/2]
 * in binary32, rounded once at the end; the rotated k and v as it is also go to their
 * slots of the paged cache, where one is given.
 *
 *   q, k, v         device, bf16; v is read only if a cache is given (else it may be NULL)
 *   *_stride        elements between two tokens' rows
 *   tokens          >= 0; tokens * (q_heads + 2 kv_heads) * head_dim elements of at most 127 GiB
 *   q_gain, k_gain  device, bf16 [head_dim], or NULL: no norm for those heads
 *   eps             >= 0
 *   positions       device, int32 [tokens]
 *   rope            device, binary32 [rope_rows, head_dim]: cosines, then sines; a
 *                   position outside [0, rope_rows) gives NaN
 *   q_out, k_out    device, bf16, written; may be q and k themselves with their strides
 *                   (no other array that is written may overlap one that is read);
 *                   k_out may be NULL if a cache is given
 *   slots           device, int32 [tokens], or NULL (then so are the caches); a slot outside
 *                   [0, pages * page_size) is not stored
 *   k_pages, v_pages, pages, page_size   the cache; at most 2^31 - 1 slots
 */
int ssq_qk_norm_rope(const uint16_t* q, int64_t q_stride, const uint16_t* k, int64_t k_stride,
                     const uint16_t* v, int64_t v_stride, int64_t tokens, int q_heads, int kv_heads,
                     int head_dim, const uint16_t* q_gain, const uint16_t* k_gain, float eps,
                     const int32_t* positions, const float* rope, int64_t rope_rows,
                     uint16_t* q_out, int64_t q_out_stride, uint16_t* k_out, int64_t k_out_stride,
                     const int32_t* slots, uint16_t* k_pages, uint16_t* v_pages, int64_t pages,
                     int page_size, hipStream_t stream);

/* ssq_qk_norm_rope for binary32 heads, gains and caches; otherwise identical. */
int ssq_qk_norm_rope_f32(const float* q, int64_t q_stride, const float* k, int64_t k_stride,
                         const float* v, int64_t v_stride, int64_t tokens, int q_heads, int kv_heads,
                         int head_dim, const float* q_gain, const float* k_gain, float eps,
                         const int32_t* positions, const float* rope, int64_t rope_rows,
                         float* q_out, int64_t q_out_stride, float* k_out, int64_t k_out_stride,
                         const int32_t* slots, float* k_pages, float* v_pages, int64_t pages,
                         int page_size, hipStream_t stream);

/*
 * ssq_attention_prompt -- causal attention over whole prompts, packed one after another:
 * for token i of a sequence and query head h of key/value head h / group,
 *   out_i = sum_{j <= i} w_j v_j,   w = softmax_j(scale q_i . k_j),   j in the same sequence.
 * Scores, maxima, sums and outputs are held in binary32; the weights are rounded to bf16
 * for the product with v (as the values are), relative to a running reference, and divided by
 * the sum of the rounded ones.  Weights are up to 2^8 before that division, so that a result
 * may be infinite where 2^8 sum_j |v_j| reaches 2^128.
 *
 *   starts    device, int32 [requests + 1], ascending from 0: sequence r holds the
 *             tokens starts[r] ... starts[r + 1] - 1 (none is valid); values are clamped to
 *             [0, tokens]; tokens from starts[requests] on are padding and give zeros
 *   requests  0 to 2^20
 *   tokens    rows of q, k, v and out; tokens * q_heads + 128 (requests + 1) kv_heads < 2^31
 *   scale     finite, > 0 (1 / sqrt(head_dim) in these models)
 *   out       device, bf16, written; must not overlap q, k or v
 */
int ssq_attention_prompt(const uint16_t* q, int64_t q_stride, const uint16_t* k, int64_t k_stride,
                         const uint16_t* v, int64_t v_stride, const int32_t* starts, int64_t requests,
                         int64_t tokens, int q_heads, int kv_heads, int head_dim, float scale,
                         uint16_t* out, int64_t out_stride, hipStream_t stream);

/* ssq_attention_prompt for binary32 q, k, v and out (weights in binary32 too);
 * tokens * q_heads + 32 (requests + 1) kv_heads < 2^29. */
int ssq_attention_prompt_f32(const float* q, int64_t q_stride, const float* k, int64_t k_stride,
                             const float* v, int64_t v_stride, const int32_t* starts, int64_t requests,
                             int64_t tokens, int q_heads, int kv_heads, int head_dim, float scale,
                             float* out, int64_t out_stride, hipStream_t stream);

/*
 * ssq_attention_decode -- attention of `fresh` new tokens of each request over the paged
 * cache (1 in plain decoding; a drafted run's length where drafts are verified).  With
 * len = min(lens[r], max_len, table_stride * page_size), token i of request r stands at
 * position p = len - fresh + i and sees the keys 0 ... p, its own (already stored)
 * among them; a token with p < 0 sees none.
 *   The first `prefix` tokens are shared: their keys and values are read from the pages of
 * request 0's table row, once for all requests (one matrix product over all queries), and
 * only what lies behind them from each request's own pages.  So the first
 * ceil(prefix / page_size) entries of every row must stand for the same tokens; where the
 * prefix ends inside a page, each request may hold its own copy of that page.  prefix = 0
 * is ordinary decoding.
 *   A table entry outside [0, pages) stands for a page that is absent: its keys are not
 * seen.
 *
 *   q, out     device, bf16 [requests * fresh, q_heads, head_dim]: the tokens of request r
 *              are rows r * fresh ... r * fresh + fresh - 1; out must not overlap q
 *   requests   0 to 2^20;  fresh >= 1;  requests * (fresh * q_heads + 32 kv_heads) < 2^29
 *   lens       device, int32 [requests]: tokens in the cache, the new ones among them
 *   max_len    host bound of lens (it sizes the launch): 0 to 2^30
 *   prefix     >= 0
 *   workspace  device, 256-byte aligned scratch of ssq_attention_decode_workspace_size()
 *              bytes, in any state; with less, or NULL, nothing is split or shared: the
 *              result is the same up to the order of sums
 * Two calls that may run concurrently must not share a workspace.
 */
int ssq_attention_decode(const uint16_t* q, int64_t q_stride, int64_t requests, int fresh,
                         int q_heads, int kv_heads, int head_dim, float scale,
                         const uint16_t* k_pages, const uint16_t* v_pages, int64_t pages, int page_size,
                         const int32_t* table, int64_t table_stride, const int32_t* lens,
                         int64_t max_len, int64_t prefix, uint16_t* out, int64_t out_stride,
                         void* workspace, size_t workspace_bytes, hipStream_t stream);

/* ssq_attention_decode for binary32 q, caches and out. */
int ssq_attention_decode_f32(const float* q, int64_t q_stride, int64_t requests, int fresh,
                             int q_heads, int kv_heads, int head_dim, float scale,
                             const float* k_pages, const float* v_pages, int64_t pages, int page_size,
                             const int32_t* table, int64_t table_stride, const int32_t* lens,
                             int64_t max_len, int64_t prefix, float* out, int64_t out_stride,
                             void* workspace, size_t workspace_bytes, hipStream_t stream);

/* Bytes of workspace for ssq_attention_decode and its _f32 form with these sizes; 0 where
 * nothing would be split, or for invalid sizes. */
size_t ssq_attention_decode_workspace_size(int64_t requests, int fresh, int q_heads, int kv_heads,
                                           int head_dim, int64_t max_len, int64_t prefix);

#ifdef __cplusplus
}
#endif

#endif /* SSQ_ATTENTION_H */
