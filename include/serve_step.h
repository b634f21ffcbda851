/*
 * serve_step -- the calls of a serving step on either side of the paged cache
 * (paged_kv.h) and of the Top-K selection (topk_ragged.h), on AMD MI355X (gfx950).
 *
 *   serve_rotate    rotary positions onto queries and keys, before paged_kv_store,
 *                   paged_kv_attend and paged_kv_score;
 *   serve_weigh     what every token of the cache gets of a step's attention, added
 *                   to rows of FP32 weights that topk_ragged selects from;
 *   serve_keep      the tokens that such a selection keeps, as an ascending list;
 *   serve_compact   the kept tokens of a cache moved together, in the request's own
 *                   pages (paged_kv_tables takes back those that are free then);
 *   serve_adjust    penalties, biases and grammar masks on logits, as the FP32 rows
 *                   that topk_ragged selects the next token's candidates from.
 *
 * Status codes, the cache and what a table is are paged_kv.h's.  As there, all
 * entry points return a status code at once, enqueue only on `stream` (a
 * hipStream_t, NULL = the default stream), allocate nothing and never synchronise,
 * so that calls can be captured in a HIP graph.  Pointers are device memory owned
 * by the caller.  Sizes that live on the device are never read by the host.
 * Results repeat to the bit.
 */
#ifndef SERVE_STEP_H
#define SERVE_STEP_H

#include "paged_kv.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Types of activations: PAGED_KV_BF16, PAGED_KV_F16, and for serve_rotate and serve_adjust */
#define SERVE_F32 2

/* How positions turn a head: pair p of its `rot` elements from `start` on by
 * position * turns[p] / 2^64 of a full turn, times `magnitude`. */
typedef struct serve_rotary {
    const uint64_t *turns; /* device [rot / 2]: turns a position in units of 2^-64, modulo one turn */
    float magnitude;       /* finite */
    int32_t rot;           /* even, from 2 to 1024 */
    int32_t start;         /* >= 0 */
    int32_t interleaved;   /* 0: pair p is elements p and p + rot / 2 of the part; 1: 2 p and 2 p + 1 */
} serve_rotary;

/* Heads [rows][heads][dim] that a call reads and those that it writes; strides in elements. */
typedef struct serve_heads {
    const void *in;
    int64_t in_row, in_head;
    void *out; /* `in` with its strides, or memory that does not overlap it */
    int64_t out_row, out_head;
    int32_t heads; /* >= 1 */
} serve_heads;

/* (a, b) -> m (a cos t - b sin t, a sin t + b cos t) for each pair (a, b) of each
 * row's heads, t its angle, m the magnitude; `transposed` takes -t: the map's
 * transpose, which takes a gradient of the output to that of the input.  Other
 * elements are copied.  Angles are off by at most 2^-28 + 2^-32 of a turn (beside what
 * the rounding of `turns` comes to) at any position: position * turns is cut to 2^-32,
 * and its distance from the nearest quarter turn is rounded to FP32.  Cosines,
 * sines and products are FP32, rounded once to the type.
 *   act        PAGED_KV_BF16, PAGED_KV_F16 or SERVE_F32;
 *   positions  int32, or int64 where `wide` is not 0, [n_rows], of any sign;
 *   q, k       heads of one row and dim; k may be NULL;
 *   dim        >= start + rot, at most 65536.
 * An alignment of 16 bytes of pointers and strides, and rot / 2, start and dim in
 * whole pieces of 16 bytes, make it fastest; any other is taken too. */
int serve_rotate(int32_t act, const serve_rotary *rotary, const void *positions, int32_t wide,
                 int32_t n_rows, int32_t dim, const serve_heads *q, const serve_heads *k,
                 int32_t transposed, void *stream);

/* Bytes of workspace for serve_weigh on the current device, for any lengths; 0
 * for arguments that it refuses.  256-byte aligned; it needs no preparation; calls
 * that overlap do not share one.  Where it is 256 a call uses none, and it may be
 * NULL: n_rows up to n_requests, or to 256 / heads. */
size_t serve_weigh_workspace(int32_t n_rows, int32_t n_requests, int32_t heads, int32_t kv_heads);

/* weights[weight_offsets[r] + j] += sum_i sum_h exp(scale q[i][h] . k_j - lse[i][h])
 * over the rows i of request r that see token j (row_starts[r] <= i < row_starts[r + 1],
 * j < row_lengths[i]) and all heads h, head h reading cache head
 * h / (heads / n_heads): with paged_kv_attend's lse, what token j got of the rows'
 * attention.  Tokens that no row sees, and those of a page outside the cache, keep
 * their weight.  A row with an lse of -inf (one that sees nothing) adds nothing.
 * FP32 products, exponentials and sums.
 *   q, act, table, row_starts, row_lengths, scale  as in paged_kv_attend, scale below
 *                   2.35e38; the cache need not have values;
 *   table_width     what the launch is laid out for, as the host knows no lengths: a table far
 *                   wider than the longest request costs time;
 *   lse             FP32 [n_rows][heads];
 *   weight_offsets  int64 [n_requests], in elements; no two requests' weights overlap. */
int serve_weigh(const paged_kv_cache *cache, int32_t act, const void *q, int64_t q_row,
                int64_t q_head, int32_t heads, const float *lse, const int32_t *table,
                int32_t table_stride, int32_t table_width, const int32_t *row_starts,
                int32_t n_requests, const int32_t *row_lengths, int32_t n_rows, float scale,
                float *weights, const int64_t *weight_offsets, void *workspace,
                size_t workspace_bytes, void *stream);

/* The tokens of each request that stay: of its lens[r], the first `first`, the last
 * `last`, and base + idx[r][0 .. K) (int32 [n_requests][K], a selection's out_idx, in
 * any order; entries below 0, and those that are no token of the request, are passed over, and a
 * token given twice stays once).
 *   kept    int32 [n_requests][width] out: their numbers, ascending, then -1;
 *           width >= first + K + last;
 *   counts  int32 [n_requests] out; neither lens nor, as kept, idx itself;
 *   weights FP32 or NULL: the weight of the i-th kept token moves to
 *           weights[weight_offsets[r] + i], and 0 follows up to lens[r].
 * lens[r] up to 2^31 - 1; one that is not positive keeps nothing. */
int serve_keep(const int32_t *idx, int32_t K, int32_t base, const int32_t *lens, int32_t n_requests,
               int32_t first, int32_t last, int32_t *kept, int32_t width, int32_t *counts,
               float *weights, const int64_t *weight_offsets, void *stream);

/* Token i of request r becomes what its token kept[r][i] was, for i < counts[r], in the
 * pages that the request has.  kept rises (serve_keep's list), and a page belongs
 * to one request, which has it once.  A page none of whose tokens moves stays as it is.  Of any other,
 * each head gets the scale that paged_kv_store would give these values, and codes
 * code * old scale / new scale, rounded once to nearest even (int8; e4m3: by way of
 * FP32).  Codes past the last token, and pages past it, stay.  Tokens from a page
 * outside the cache become 0; to such a page nothing is written.
 *   kept    int32 [n_requests][width], counts int32 [n_requests];
 *   table   int32 [n_requests][table_stride], table_width entries used. */
int serve_compact(const paged_kv_cache *cache, const int32_t *table, int32_t table_stride,
                  int32_t table_width, const int32_t *kept, int32_t width, const int32_t *counts,
                  int32_t n_requests, void *stream);

/* What serve_adjust takes beside the logits.  Lists are ragged: row i's tokens are
 * tokens[token_starts[i]] .. tokens[token_starts[i + 1]), and likewise its biases;
 * ids outside [0, vocab) are passed over. */
typedef struct serve_lists {
    const int32_t *tokens;       /* the row's tokens so far, or NULL */
    const int64_t *token_starts; /* [n_rows + 1] */
    const int32_t *prompt_lens;  /* [n_rows]: how many of them, from the first on, are the prompt's; NULL: none */
    const float *repetition;     /* [n_rows], or NULL: 1 */
    const float *frequency;      /* [n_rows], or NULL: 0 */
    const float *presence;       /* [n_rows], or NULL: 0 */
    const int32_t *bias_ids;     /* or NULL; of an id given twice in a row the later entry counts */
    const float *bias;
    const int64_t *bias_starts;  /* [n_rows + 1] */
    const uint32_t *mask;        /* [n_masks][mask_stride]: token t is allowed where bit t % 32 of word t / 32 is set; or NULL */
    int64_t mask_stride;         /* words, >= (vocab + 31) / 32 */
    int32_t n_masks;
    const int32_t *row_mask;     /* [n_rows]: the row's mask; outside [0, n_masks): none.  NULL: mask i of row i */
} serve_lists;

/* out[i][t], FP32, from x = logits[i][t], in this order, each step rounded to FP32:
 *   of a token among the row's: x / repetition where x > 0, x * repetition elsewhere;
 *   of one n times among those behind the prompt's, n > 0: x - frequency * n, then - presence;
 *   of a biased token: x + bias;
 *   of a token that the mask does not allow: -inf, whatever x is.
 *   act         PAGED_KV_BF16, PAGED_KV_F16 or SERVE_F32;
 *   logits      [n_rows][vocab], x_row elements from row to row;
 *   out         FP32 [n_rows][vocab], out_row >= vocab elements from row to row; may be
 *               logits where these are FP32 and have its stride, or memory apart. */
int serve_adjust(int32_t act, const void *logits, int64_t x_row, float *out, int64_t out_row,
                 int32_t n_rows, int32_t vocab, const serve_lists *lists, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* SERVE_STEP_H */
