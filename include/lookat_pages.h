/*
 * lookat_pages.h -- a paged LOOKAT cache with values in 8 bits: writing it, attention over it, upkeep of its pages.
 *
 * The general rules, status codes and error text of lookat.h hold here too.
 *
 * A layer's cache is a POOL of pages, each with room for `page` tokens of all H key/value heads:
 *     codes      [pages, H, page, m]          uint8, the product-quantised keys (paper Sec. 3.4)
 *     values     [pages, H, page/8, d_k, 8]   8-bit values: coordinate d of a page's token t at [t / 8, d, t % 8], so that
 *                                             eight tokens of one coordinate are eight consecutive bytes (an operand of
 *                                             the matrix cores as it is loaded)
 *     exponents  [pages, H]                   int8: a stored q stands for q * 2^exponent, one exponent per page and head
 * A SEQUENCE is a row of `table` (page ids in order of position) with `lengths` tokens: its token at position t lies in
 * page table[t / page] at t % page.  Rows are W entries long, table_stride apart; a sequence's tokens behind W * page, and
 * those in pages whose id is outside [0, pages), are neither read nor written (attention passes over them).  A length
 * below zero counts as zero.  `refs` counts, for every page, the sequences that hold it; 0 is a free page.
 * A model keeps a pool for each layer and one set of books (table, lengths, refs) for all of them: lookat_pages_reserve copies shared pages in
 * the pool it is given and says which, for lookat_pages_copy on the others; lookat_pages_compact, which leaves the books that it reads as they
 * are, is called for each pool; fork and free touch the books alone.
 *
 * Exponents lie in [-40, 40]: values up to 1.4e14 (I8) or 4.9e14 (E4M3) are kept, and below 2^-41 (I8) or 2^-50 (E4M3) nothing but
 * zero.  Scales are powers of two on purpose: the division v / 2^e and the widening q * 2^e are exact, so a value is rounded
 * once, bit for bit the same everywhere; and when a page's exponent has to grow its tokens are rounded again to half as
 * many steps or fewer, so that all roundings of a token together stay below one step of the exponent it has in the end.
 *
 * Supported: d_k in {64, 128}, m in {2, 4, 8, 16} dividing d_k, page in {16, 32, 64, 128}, at most 2^30 pages of
 * at most 4096 heads, at most 65535 sequences, W * page at most 2^30, and per call fewer than 2^23 workgroups
 * (sequences * heads * num_splits of attention, pages of one sequence written), fewer than 2^24 16 KB pieces of pages to copy and at most
 * 65535 list entries of a fork or free; otherwise LOOKAT_ERR_UNSUPPORTED or LOOKAT_ERR_SHAPE.
 */
#ifndef LOOKAT_PAGES_H
#define LOOKAT_PAGES_H

#include "lookat.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    LOOKAT_VALUES_I8 = 1,   /* two's complement, -127..127 */
    LOOKAT_VALUES_E4M3 = 2, /* 8-bit floating point: 4 exponent bits, 3 mantissa bits, no infinities, largest 448 */
    /* Not types: they give the type the whole range of int (as in lookat_dtype). */
    LOOKAT_VALUES_RANGE_LOW_ = -0x7fffffff - 1,
    LOOKAT_VALUES_RANGE_HIGH_ = 0x7fffffff
} lookat_value_type;

typedef struct {
    int32_t pages, H, d_k, m, page;
    lookat_value_type value_type;
    uint8_t *codes;    /* device, 16-byte aligned */
    void *values;      /* device, 16-byte aligned */
    int8_t *exponents; /* device */
} lookat_page_pool;

/*
 * Writes the last counts[b] tokens of every sequence b into its pages: row n of codes / values [B,H,N,*] goes to position
 * lengths[b] - counts[b] + n, for n < min(counts[b], N) (counts NULL: N for every b).  Rows whose position is negative are
 * left out.  For a page with new tokens, per head,
 *     exponent = the least e in [-40, 40] with |v| <= 127 * 2^e (I8) or 448 * 2^e (E4M3) for all of the page's new values,
 *                but not below the exponent that it has if it already holds tokens of the sequence (positions before the first new one)
 *     stored   = v * 2^-exponent rounded to the nearest stored number, ties to even; larger ones to the largest, NaN to 0
 * and tokens that the page holds already are brought to the new exponent by the same rounding.  What the page has behind
 * the sequence's last token stays as it was.  Codes are copied.
 * The pages are written in place: no other sequence may hold them (lookat_pages_reserve sees to that), and no page may
 * be named twice among those written.
 *   codes         element (b,h,n,i) at codes[(b*H+h)*code_stride_bh + n*m + i]; base and stride multiples of m bytes
 *   values        fp16 or fp32, element (b,h,n,j) at values[(b*H+h)*value_stride_bh + n*d_k + j]; base 16-byte aligned,
 *                 stride a multiple of 8 (fp16) or 4 (fp32) elements
 *   table         [B, W] int32, rows table_stride >= W apart;  lengths, counts  [B] int32
 *   N             >= 0 (0: nothing is done)
 */
int lookat_pages_write(const lookat_page_pool *pool, int32_t B, int64_t N,
                       const uint8_t *codes, int64_t code_stride_bh,
                       const void *values, lookat_dtype value_dtype, int64_t value_stride_bh,
                       const int32_t *table, int32_t W, int64_t table_stride,
                       const int32_t *lengths, const int32_t *counts,
                       void *stream);

/*
 * Attention decode over the pages (paper Algorithm 1), one query per (b, query head), `group` consecutive query heads on
 * each key/value head as in lookat_attend_decode_gqa:
 *     s[b,hq,l]   = sum_i lut[b,hq,i, code(b, hq/group, l, i)]
 *     out[b,hq,:] = sum_l softmax_l(scale * s[b,hq,:]) * value(b, hq/group, l, :)       l < lengths[b]
 * A sequence without tokens gives zeros, and so does one whose tokens all have a score of -inf (a -inf in a table is a token
 * without weight).  A NaN score, or one of +inf, makes its query head's row NaN, however the sequence is cut; other rows are
 * not touched by it.  Scores (times scale and log2(e), so that 2.35e38 is their end), softmax statistics and sums are held
 * in fp32; a weight enters the product with the values as two fp16 terms (22 bits), the stored 8-bit numbers exactly.
 *   lut           [B, H*group, m, 256] fp32, 16-byte aligned, from lookat_build_lut
 *   max_length    the longest length the host knows of, or 0 for W * page: it sizes the launch alone; longer sequences are
 *                 right too.  Above 2048, sequences may be cut, which costs a second launch (3 to 4 us) in every call
 *   group         1, 2, 4 or 8, otherwise LOOKAT_ERR_UNSUPPORTED
 *   num_splits    0: the sequences are cut into ranges by their lengths, on the device, where they are long enough to gain from it and there
 *                 are at most 1024 of them (more are not cut); >= 1: that many equal ranges of max_length per (b, key/value head).
 *                 The result does not depend on it beyond fp32 rounding
 *   workspace     lookat_attend_pages_workspace_bytes(pool, B, group, W, max_length, num_splits) bytes, 16-byte aligned (NULL when 0);
 *                 calls in flight at once must not share one
 *   out           [B, H*group, d_k] fp32, 16-byte aligned
 */
size_t lookat_attend_pages_workspace_bytes(const lookat_page_pool *pool, int32_t B, int32_t group, int32_t W,
                                           int64_t max_length, int32_t num_splits);

int lookat_attend_pages(const lookat_page_pool *pool, int32_t B, int32_t group,
                        const float *lut,
                        const int32_t *table, int32_t W, int64_t table_stride,
                        const int32_t *lengths, int64_t max_length,
                        float scale, int32_t num_splits,
                        void *workspace, size_t workspace_bytes,
                        float *out,
                        void *stream);

/*
 * Attention of a chunk of new tokens over the pages: pieces of prompts, drafted tokens to be verified.  Row n of sequence b, n < min(counts[b], N)
 * (counts NULL: N for every b), stands at position p = lengths[b] - counts[b] + n, as in lookat_pages_write (which comes first: the rows' own
 * tokens are read from the pages), and sees the tokens l <= p.  With k^ the key that a token's codes stand for (its centroids side by side):
 *     s[b,hq,n,l]   = sum_j q[b,hq,n,j] * k^(b, hq/group, l)_j
 *     out[b,hq,n,:] = sum_{l <= p} softmax_l(scale * s[b,hq,n,:]) * value(b, hq/group, l, :)
 * A row that sees no token gives zeros, and so does one whose tokens all have a score of -inf; other rows of out are left as they were.  A NaN
 * score or one of +inf makes its row NaN; other rows are not touched by it.  A scale of NaN makes every row NaN that sees a token, a stored NaN (E4M3)
 * its coordinate in the rows that see its token.
 * Centroids enter the product as two fp16 terms, scaled by one power of two per key/value head: exactly to 2^-22 of themselves, or to 2^-39 of the
 * head's largest finite centroid entry where that is more (whether a token has that centroid or not: one of 1e30 leaves nothing of others of 1);
 * fp16 queries exactly, fp32 queries to 2^-22 of themselves or 2^-39 of the row's largest entry; weights, sums and values as in
 * lookat_attend_pages.  An infinite centroid entry makes the scores of the tokens that have it NaN; centroids that no token has may be NaN or infinite.
 *   q             [B, H*group, N, d_k] fp16 or fp32: element (b,hq,n,j) at q[b*q_stride_b + hq*q_stride_h + n*q_stride_n + j]; base 16-byte
 *                 aligned, strides multiples of 8 (fp16) or 4 (fp32) elements
 *   codebooks     [H, m, 256, d_k/m] fp32, 16-byte aligned
 *   max_length    as in lookat_attend_pages: it sizes the launch alone
 *   group         1 to 64;  N * group at most 2^24, H * group at most 65535
 *   num_splits    0: the library's choice; >= 1: the tokens that a tile of rows sees are cut into that many ranges, merged by another launch
 *   workspace     lookat_attend_pages_chunk_workspace_bytes(pool, B, N, group, W, max_length, num_splits) bytes, 16-byte aligned; calls in flight
 *                 at once must not share one
 *   out           [B, H*group, N, d_k] fp32, 16-byte aligned
 */
size_t lookat_attend_pages_chunk_workspace_bytes(const lookat_page_pool *pool, int32_t B, int32_t N, int32_t group, int32_t W,
                                                 int64_t max_length, int32_t num_splits);

int lookat_attend_pages_chunk(const lookat_page_pool *pool, int32_t B, int32_t N, int32_t group,
                              const void *q, lookat_dtype q_dtype, int64_t q_stride_b, int64_t q_stride_h, int64_t q_stride_n,
                              const float *codebooks,
                              const int32_t *table, int32_t W, int64_t table_stride,
                              const int32_t *lengths, const int32_t *counts, int64_t max_length,
                              float scale, int32_t num_splits,
                              void *workspace, size_t workspace_bytes,
                              float *out,
                              void *stream);

/*
 * Adds up the attention that every token is paid, from the tables of the newest queries (those that lookat_attend_pages takes), for a cache that
 * is held to a budget:
 *     weights[b,h,l] = decay * weights[b,h,l] + sum_g softmax_l(scale * s[b, h*group + g, :])        l < min(lengths[b], columns)
 * with s as in lookat_attend_pages.  The maximum and the sum of a softmax are taken over all of the sequence's tokens.  decay 0 takes no notice of what
 * weights held.  A token in a page outside the pool, and a query head whose tokens all have a score of -inf, add nothing; a NaN score or one
 * of +inf makes the weights of its key/value head NaN (that sequence's).  Weights behind a sequence's last token are left as they were.  Every weight
 * has one writer and its sum one order: results are reproducible bit for bit.
 * One query per query head and call: what the rows of a prompt pay is not summed by lookat_attend_pages_chunk, so after a prompt weights are what
 * the caller put there, until later queries add theirs (or the prompt's do, a call with their tables for each row that is to count).
 *   lut           [B, H*group, m, 256] fp32, 16-byte aligned;  group 1, 2, 4 or 8
 *   weights       element (b,h,l) at weights[(b*H+h)*weight_stride_bh + l], l < columns <= weight_stride_bh
 *   max_length    the longest length the host knows of, or 0 for W * page: it sizes the launch alone
 *   workspace     lookat_pages_weigh_workspace_bytes(pool, B, group, W, max_length) bytes, 16-byte aligned (NULL when 0); calls in flight at once
 *                 must not share one
 * The pool's values are not read.
 */
size_t lookat_pages_weigh_workspace_bytes(const lookat_page_pool *pool, int32_t B, int32_t group, int32_t W, int64_t max_length);

int lookat_pages_weigh(const lookat_page_pool *pool, int32_t B, int32_t group,
                       const float *lut,
                       const int32_t *table, int32_t W, int64_t table_stride,
                       const int32_t *lengths, int64_t max_length,
                       float scale, float decay,
                       float *weights, int32_t columns, int64_t weight_stride_bh,
                       void *workspace, size_t workspace_bytes, void *stream);

/*
 * Keeps k = min(lengths[b], keep[b]) tokens of every sequence b (at least 0, at most W_out * page), each key/value head its own: the last `recent`
 * tokens (k at most), the first `first` (what is left at most), and of the others the heaviest, among equal weights those of the lowest positions.  NaN
 * counts as less than any weight, both zeros as equal; tokens from `columns` on weigh 0.  The kept tokens enter the pages of row b of table_out
 * at positions 0..k-1, in their order, as if lookat_pages_write wrote the values that they stand for into an empty sequence: a page's exponent is
 * the least that its tokens allow, so a token is rounded only where its exponent grows, by half a step of the new one at most.  What these
 * pages have behind the last token stays as it was; table, lengths and the books are not changed.  So a user reserves k tokens for an empty slot, calls
 * this with its row, and frees the old slot: pages shared with other sequences are read, not written.  Both slots hold pages in between: a pool
 * that is brought down when it is full keeps ceil(k / page) pages back for each sequence of a call.  Where all weights are equal (zeros after a
 * prompt) the lowest positions are kept beside the last `recent`.
 * No page of table_out may be named twice or be one that is read.  A kept token in a page outside the pool leaves its place as it was, and so do
 * those whose place is in one.
 *   weights       as in lookat_pages_weigh, read;  keep [B] int32;  first, recent >= 0
 *   table_out     [B, W_out] int32, rows table_out_stride >= W_out apart
 *   weights_out   NULL, or element (b,h,j) at weights_out[(b*H+h)*weight_out_stride_bh + j], j < columns_out: the kept tokens' weights, in their
 *                 new places; must not overlap weights
 *   workspace     lookat_pages_evict_workspace_bytes(pool, B, W_out) bytes, 16-byte aligned: afterwards the kept positions, [B, H, W_out * page]
 *                 int32, of which the first k of each head are set; calls in flight at once must not share one
 */
size_t lookat_pages_evict_workspace_bytes(const lookat_page_pool *pool, int32_t B, int32_t W_out);

int lookat_pages_evict(const lookat_page_pool *pool, int32_t B,
                       const int32_t *table, int32_t W, int64_t table_stride, const int32_t *lengths,
                       const float *weights, int32_t columns, int64_t weight_stride_bh,
                       const int32_t *keep, int32_t first, int32_t recent,
                       const int32_t *table_out, int32_t W_out, int64_t table_out_stride,
                       float *weights_out, int32_t columns_out, int64_t weight_out_stride_bh,
                       void *workspace, size_t workspace_bytes, void *stream);

/*
 * Copies pages src[i] onto pages dst[i] (codes, values, exponents), i < n.  Pairs with an id outside [0, pages) or with
 * src = dst are passed over.  No page may be a destination twice, or both a source and a destination (its content would be
 * unspecified).
 *   src, dst   [n] int32, device;  n >= 0
 */
int lookat_pages_copy(const lookat_page_pool *pool, int32_t n, const int32_t *src, const int32_t *dst, void *stream);

/*
 * Lets sequence dst[i] begin as sequence src[i], i < n: its row, up to its length, and its length are copied and its pages counted
 * once more.  The pages are shared: lookat_pages_reserve copies one before it is written.  Only an empty slot
 * (length <= 0) is a destination; a pair is passed over when a slot is outside [0, S), its destination is not empty or is that of
 * an earlier pair, or its source is a destination of the call (it is empty).
 *   table   [S, W] int32, rows table_stride >= W apart;  lengths [S], refs [pages] int32;  src, dst [n] int32; all on the device
 */
int lookat_pages_fork(const lookat_page_pool *pool, int32_t S, int32_t *table, int32_t W, int64_t table_stride,
                      int32_t *lengths, int32_t *refs, int32_t n, const int32_t *src, const int32_t *dst, void *stream);

/*
 * Gives up the sequences slots[i], i < n: each of their pages is counted once less (at 0 it is free), the row's entries become -1 and the
 * length 0.  Slots outside [0, S) and repeated ones are passed over.
 */
int lookat_pages_free(const lookat_page_pool *pool, int32_t S, int32_t *table, int32_t W, int64_t table_stride,
                      int32_t *lengths, int32_t *refs, int32_t n, const int32_t *slots, void *stream);

/*
 * Makes room: sequence s grows from lengths[s] to new_lengths[s] tokens (not above lengths[s]: it stays as it is).  It needs
 * a page for every entry of its row that new tokens reach first, and one more if they begin inside a page that was counted more
 * than once when the call began: that page's content is copied to the new one, which takes its place in the row.
 * The needed entries, in row-major order of the table, get the free pages in ascending order, each counted once; the
 * lengths become the new ones.  If there are too few free pages, or a row is too short for a page it needs, NOTHING is changed and
 * missing[0] says by how many pages, else missing[0] = 0.
 * (Of several sequences that share a last page and all grow, all get a copy; the page itself becomes free.)
 *   new_lengths  [S] int32, must not overlap lengths;  missing  [1] int32.  Neither missing nor copies overlaps another array of the call
 *   copies       NULL, or [2, S] int32: copies[0,s] the page that was copied for sequence s and copies[1,s] the one it was copied to, -1
 *                where none was: what lookat_pages_copy takes to do the same in the pools of other layers that share these books
 *   workspace    lookat_pages_reserve_workspace_bytes(pool, S) bytes, 16-byte aligned
 */
size_t lookat_pages_reserve_workspace_bytes(const lookat_page_pool *pool, int32_t S);

int lookat_pages_reserve(const lookat_page_pool *pool, int32_t S, int32_t *table, int32_t W, int64_t table_stride,
                         int32_t *lengths, int32_t *refs, const int32_t *new_lengths, int32_t *missing, int32_t *copies,
                         void *workspace, size_t workspace_bytes, void *stream);

/*
 * Compacts the pool: with n pages in use, those at ids >= n move, in ascending order, to the free ids below n, content and all, so
 * that pages 0..n-1 are in use and the rest are free.  The books are written to new arrays (which must not overlap
 * the old ones): table_out [S, W] has the new ids and -1 behind each sequence's pages, refs_out [pages] the new counts, live[0] = n.  `lengths`
 * stays valid.  Page contents at ids >= n are left as they were, so until the pool is written again the old books are still good.
 *   workspace    lookat_pages_compact_workspace_bytes(pool) bytes, 16-byte aligned
 */
size_t lookat_pages_compact_workspace_bytes(const lookat_page_pool *pool);

int lookat_pages_compact(const lookat_page_pool *pool, int32_t S, const int32_t *table, int32_t W, int64_t table_stride,
                         const int32_t *lengths, const int32_t *refs,
                         int32_t *table_out, int64_t table_out_stride, int32_t *refs_out, int32_t *live,
                         void *workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* LOOKAT_PAGES_H */
