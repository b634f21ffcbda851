/*
 * paged_kv -- a paged 8-bit key/value cache and what reads it, on AMD MI355X (gfx950).
 *
 * The calls that stand around a Top-K selection (topk_ragged.h) when a model
 * with sparse attention is served:
 *   paged_kv_tables   a step's block tables, row tables and slots, from request lengths;
 *   paged_kv_store    new keys and values into the cache's pages, in 8 bits;
 *   paged_kv_score    the FP32 score rows that the selection reads, over paged keys;
 *   paged_kv_attend_selected   attention of each row over its selected tokens;
 *   paged_kv_attend   attention of each row over all tokens of its request.
 *
 * The cache.  A page holds `page` consecutive tokens of one request; entry
 * [p][h][i][d] of `k` and `v` is an 8-bit code (OCP e4m3 or int8), and
 * k_scale[p][h], v_scale[p][h] are the FP32 scales of a page's entries of one
 * head, not negative: value = code * scale.  Token t of request r lies in page
 * table[r][t / page], at t % page.  Entries past a request's length may hold
 * anything; entries within it are finite (the store writes no others).
 *
 * A step's rows.  A row is one new token.  Rows of a request are consecutive:
 * request r has rows row_starts[r] .. row_starts[r + 1]; row i sees the first
 * row_lengths[i] tokens of its request row_request[i] (its own among them).
 * A row whose request is outside the table, or whose length is not positive,
 * sees nothing; so does a row at the tokens of a page outside the cache, and
 * lengths end where the table's width does.
 *
 * All entry points return a status code at once, enqueue only on `stream` (a
 * hipStream_t, NULL = the default stream), allocate nothing and never
 * synchronise, so that calls can be captured in a HIP graph.  Pointers are
 * device memory owned by the caller.  Sizes that live on the device are never
 * read by the host: the launch depends on the arguments alone.
 */
#ifndef PAGED_KV_H
#define PAGED_KV_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Status codes. */
#define PAGED_KV_OK 0
#define PAGED_KV_EINVAL (-1)       /* bad scalar argument, null or misaligned pointer */
#define PAGED_KV_EUNSUPPORTED (-2) /* a size or type that no kernel takes, or no gfx950 */
#define PAGED_KV_ELAUNCH (-3)      /* a HIP call failed */
#define PAGED_KV_EWORKSPACE (-4)   /* workspace too small */

/* Types of cache entries and of activations. */
#define PAGED_KV_E4M3 0
#define PAGED_KV_INT8 1
#define PAGED_KV_BF16 0
#define PAGED_KV_F16 1

typedef struct paged_kv_cache {
    void *k;               /* 8-bit codes, 16-byte aligned */
    void *v;               /* NULL: keys alone (an indexer's cache) */
    float *k_scale;        /* [n_pages][scale_stride], the first n_heads of each used */
    float *v_scale;        /* NULL where v is */
    int64_t page_stride;   /* entries from one page to the next, >= n_heads * page * head_dim and
                              a multiple of head_dim; n_pages * page_stride / head_dim < 2^32 */
    int64_t scale_stride;  /* floats from one page's scales to the next, >= n_heads */
    int32_t n_pages;       /* >= 1 */
    int32_t page;          /* tokens to a page: 16, 32, 64, 128 or 256 */
    int32_t n_heads;       /* >= 1 */
    int32_t head_dim;      /* 64, 128 or 256 (64 or 128 for paged_kv_score) */
    int32_t code;          /* PAGED_KV_E4M3 or PAGED_KV_INT8 */
} paged_kv_cache;

/* A step's tables from request lengths.
 *   ring, ring_size   int32: the numbers of the free pages, a queue in a ring;
 *   pool_in, pool_out int32 [4]: place of the ring's first free page, count of
 *                     free pages; out also the count of refused requests, and 0;
 *   lens_in, lens_out int32 [n_requests]: tokens in the cache before and after;
 *   new_lens          int32 [n_requests]: tokens added; negative: taken off the
 *                     end (all of them where it exceeds the length);
 *   table             int32 [n_requests][table_stride], `table_width` used;
 *   page              tokens to a page (a power of two from 16 to 256);
 *   row_starts        int32 [n_requests + 1] out: first row of each request;
 *   row_request, row_lengths  int32 [n_rows] out; slots int64 [n_rows] out:
 *                     page * tokens-to-a-page + place, for paged_kv_store.
 * Pages that a request no longer needs go to the ring's end, in the requests'
 * order; then requests that need more take them from its front, in order.  A
 * request is refused, and keeps its length, when the pages asked for up to and
 * including its own exceed the free ones, or when it needs more than
 * table_width: its rows have length 0 and slot -1.  Table entries past a
 * request's pages are left as they are.  Rows past the last request's have
 * request -1, length 0 and slot -1; rows that do not fit n_rows are not
 * written (row_starts still counts them, up to 2^31 - 1).
 * pool_out may be pool_in.  lens_out may not be lens_in (EINVAL): the rows are
 * made from the lengths before the step and from those after it. */
int paged_kv_tables(int32_t *ring, int32_t ring_size, const int32_t *pool_in, int32_t *pool_out,
                    const int32_t *lens_in, const int32_t *new_lens, int32_t *lens_out,
                    int32_t n_requests, int32_t *table, int32_t table_stride, int32_t table_width,
                    int32_t page, int32_t n_rows, int32_t *row_starts, int32_t *row_request,
                    int32_t *row_lengths, int64_t *slots, void *stream);

/* New entries into the cache.
 *   k_new, v_new  BF16 or F16 (`act`) [n_rows][n_heads][head_dim]; *_row and
 *                 *_head are strides in elements (multiples of 8; 16-byte
 *                 aligned pointers); v_new is NULL where the cache has no values;
 *   slots         int64 [n_rows]: page * tokens-to-a-page + place.  Rows of a
 *                 slot outside the cache are left out.  Rows of one page follow
 *                 each other, at consecutive places (as paged_kv_tables lays them).
 * For each page written to and each head, a = the largest |x| of the finite new
 * entries: e4m3's scale is the least power of two s with 448 s >= a, int8's is
 * a times the FP32 number nearest to 1 / 127, both at least 2^-100.  Where the first new entry is not the page's
 * first, the entries before it are kept: the scale is then the larger of the
 * old and the new one, and codes under a smaller old scale are rounded anew.
 * New entries are x / scale, rounded to nearest even; NaN is stored as 0, and
 * infinities as the type's largest. */
int paged_kv_store(const paged_kv_cache *cache, int32_t act, const void *k_new, int64_t k_row,
                   int64_t k_head, const void *v_new, int64_t v_row, int64_t v_head,
                   const int64_t *slots, int32_t n_rows, void *stream);

/* Bytes of workspace for the two attention calls on the current device, for
 * any lengths; 0 for arguments that they refuse.  The workspace is 256-byte
 * aligned; its first PAGED_KV_WORKSPACE_ZEROED bytes are zeroed by the caller
 * before its first use (the kernels leave them zero), and calls that overlap do
 * not share one. */
#define PAGED_KV_WORKSPACE_ZEROED 8192
size_t paged_kv_attend_workspace(int32_t n_rows, int32_t n_requests, int32_t heads,
                                 int32_t kv_heads, int32_t head_dim);

/* out[i][h] = sum_t p_t v_t with p = softmax(scale * q[i][h] . k_t) over the
 * tokens t < row_lengths[i] of row i's request, head h reading cache head
 * h / (heads / n_heads).
 *   q       BF16 or F16 (`act`) [n_rows][heads][head_dim], strides q_row and
 *           q_head in elements (multiples of 8, 16-byte aligned pointer);
 *   out     [n_rows][heads][head_dim], of q's type, contiguous, 16-byte aligned;
 *   lse     FP32 [n_rows][heads], log sum exp of the scaled products, or NULL;
 *   table   int32 [n_requests][table_stride], table_width entries used;
 *   heads   a multiple of the cache's n_heads;
 *   scale   finite and not negative.
 * A row that sees no token, or that no request has (row_starts[0] may be past 0), gets
 * 0 and -inf.  Scores, sums and lse are FP32; weights are rounded to f16 before they
 * meet the values, whatever q's type: 11 bits down to 2^-20 of the row's largest
 * product of weight and value scale. */
int paged_kv_attend(const paged_kv_cache *cache, int32_t act, const void *q, int64_t q_row,
                    int64_t q_head, int32_t heads, const int32_t *table, int32_t table_stride,
                    int32_t table_width, const int32_t *row_starts, int32_t n_requests,
                    const int32_t *row_lengths, int32_t n_rows, float scale, void *out, float *lse,
                    void *workspace, size_t workspace_bytes, void *stream);

/* The same over the tokens idx[i][0 .. K) of row i (int32 [n_rows][K], any
 * order; a selection's out_idx).  Entries below 0 or at and past
 * row_lengths[i] are absent; an entry given twice counts twice. */
int paged_kv_attend_selected(const paged_kv_cache *cache, int32_t act, const void *q,
                             int64_t q_row, int64_t q_head, int32_t heads, const int32_t *idx,
                             int32_t K, const int32_t *table, int32_t table_stride,
                             int32_t table_width, const int32_t *row_request, int32_t n_requests,
                             const int32_t *row_lengths, int32_t n_rows, float scale, void *out,
                             float *lse, void *workspace, size_t workspace_bytes, void *stream);

/* scores[row_offsets[i] + j] = scale * sum_h w[i][h] * max(0, q[i][h] . k_j)
 * for j < row_lengths[i], over the keys of a cache with one head: the rows that
 * topk_ragged selects from.  Nothing past a row's length is written; at the
 * tokens of a page outside the cache the score is -inf.
 *   q    as above, `heads` from 1 to 128;  w  FP32 [n_rows][heads]; both finite
 *        (a product that is NaN may count as 0);
 *   row_offsets  int64 [n_rows], in elements. */
int paged_kv_score(const paged_kv_cache *cache, int32_t act, const void *q, int64_t q_row,
                   int64_t q_head, int32_t heads, const float *w, const int32_t *table,
                   int32_t table_stride, int32_t table_width, const int32_t *row_request,
                   int32_t n_requests, const int32_t *row_lengths, int32_t n_rows, float scale,
                   float *scores, const int64_t *row_offsets, void *stream);

/* Human-readable text for a status code. */
const char *paged_kv_status_str(int status);

#ifdef __cplusplus
}
#endif

#endif /* PAGED_KV_H */
