// The score rows that a Top-K selects from: s_ij = scale sum_h w_ih relu(q_ih . k_j).
//
// Few rows: bound by memory (D bytes of keys read and 4 written a token).  Many
// rows: by the matrix products and the two vector operations that each product
// needs behind them.  A wave keeps the keys of 64 tokens in registers as the
// columns of 32 x 32 x 16 products and passes the rows' queries by, from LDS;
// the 32 rows of a product are laid out so that all heads of a row lie in the
// accumulator of one lane, which adds them without crossing lanes.
#include "paged_common.h"

namespace paged {
namespace {

constexpr int kBlock = 256;
constexpr int kTokens = 256;  // of a workgroup: 64 to a wave

struct ScoreArgs {
    const uint8_t *k;
    const float *ks;
    int64_t page_stride, scale_stride;
    int n_pages, lp;
    const void *q;
    int64_t q_row, q_head;
    int heads;
    const float *w;
    const int *table;
    int table_stride, table_width;
    const int *row_request, *row_lengths;
    int n_requests, n_rows, window;
    float scale;
    float *scores;
    const int64_t *row_offsets;
};

// HP: heads of a row in one product, a power of two up to 16 (the rest of `heads`
// in further products); a product has 32 / HP rows, half of them to a half wave.
template <int D, int HP, class T, class C>
__global__ __launch_bounds__(kBlock) void score_kernel(ScoreArgs a) {
    constexpr int ROWS = 32 / HP, HALF = 16 / HP;  // of a product, and of a lane
    __shared__ alignas(16) uint8_t qs[32][2 * D + 16];
    __shared__ alignas(16) float ws[32];
    __shared__ int lens[ROWS];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = lane & 31, g = lane >> 5;
    const int P = 1 << a.lp;
    const int chunks = (a.heads + HP - 1) / HP;  // more than one only where HP is 16
    const int tok0 = blockIdx.x * kTokens + 64 * wave;
    const int row_end = min((int)(blockIdx.y + 1) * a.window, a.n_rows);
    const int64_t cap = (int64_t)a.table_width << a.lp;

    int row = blockIdx.y * a.window;
    while (row < row_end) {
        // the rows from here on that share their request
        const int request = a.row_request[row];
        int stop = row + 1;
        while (stop < row_end && a.row_request[stop] == request) ++stop;
        if (request < 0 || request >= a.n_requests) {
            row = stop;
            continue;
        }
        // keys of this wave's tokens
        typename Act<T>::frag k[2][D / 16];
        float ks[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int tok = tok0 + 32 * t + n;
            int pg = tok < cap ? a.table[(int64_t)request * a.table_stride + (tok >> a.lp)] : -1;
            if (pg >= a.n_pages) pg = -1;
            const uint8_t *p = a.k + max(pg, 0) * a.page_stride + (int64_t)(tok & (P - 1)) * D;
            ks[t] = pg < 0 ? 0.0f : a.ks[pg * a.scale_stride] * a.scale;
#pragma unroll
            for (int j = 0; j < D / 16; ++j) {
                const u32x2 x = *(const u32x2 *)(p + 16 * j + 8 * g);
                k[t][j] = eight<C, T>(x[0], x[1]);
            }
            if (pg < 0) ks[t] = -__builtin_inff();  // marks a page outside the cache
        }
        for (int r0 = row; r0 < stop; r0 += ROWS) {
            float sum[2][HALF];
            for (int t = 0; t < 2; ++t)
                for (int i = 0; i < HALF; ++i) sum[t][i] = 0.0f;
            for (int c = 0; c < chunks; ++c) {
                __syncthreads();
                for (int i = tid; i < 32 * (D / 8); i += kBlock) {
                    const int mm = i / (D / 8), d = i % (D / 8) * 8;
                    // product row mm: half (mm >> 2) & 1, place 4 (mm >> 3) + (mm & 3) of the half's 16
                    const int place = 4 * (mm >> 3) + (mm & 3), r = r0 + ((mm >> 2) & 1) * HALF + place / HP;
                    const int h = c * HP + place % HP;
                    u32x4 x = {0, 0, 0, 0};
                    if (r < stop && h < a.heads)
                        x = *(const u32x4 *)((const char *)a.q + 2 * (r * a.q_row + h * a.q_head + d));
                    *(u32x4 *)&qs[mm][2 * d] = x;
                }
                if (tid < 32) {
                    const int half = tid >> 4, place = tid & 15, r = r0 + half * HALF + place / HP, h = c * HP + place % HP;
                    ws[tid] = r < stop && h < a.heads ? a.w[(int64_t)r * a.heads + h] : 0.0f;
                }
                if (tid < ROWS)
                    lens[tid] = r0 + tid < stop ? (int)min((int64_t)max(a.row_lengths[r0 + tid], 0), cap) : 0;
                __syncthreads();
                f32x16 s[2];
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[t][i] = 0.0f;
#pragma unroll
                for (int j = 0; j < D / 16; ++j) {
                    const auto x = __builtin_bit_cast(typename Act<T>::frag, *(const u32x4 *)&qs[n][32 * j + 16 * g]);
#pragma unroll
                    for (int t = 0; t < 2; ++t) s[t] = Act<T>::mfma32(x, k[t][j], s[t]);
                }
#pragma unroll
                for (int i = 0; i < 16; ++i)
#pragma unroll
                    for (int t = 0; t < 2; ++t) sum[t][i / HP] += ws[16 * g + i] * fmaxf(s[t][i], 0.0f);
            }
#pragma unroll
            for (int i = 0; i < HALF; ++i) {
                const int rr = g * HALF + i;
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const int tok = tok0 + 32 * t + n;
                    if (tok < lens[rr])
                        a.scores[a.row_offsets[r0 + rr] + tok] =
                            ks[t] == -__builtin_inff() ? -__builtin_inff() : sum[t][i] * ks[t];
                }
            }
        }
        row = stop;
        __syncthreads();
    }
}

template <int D, class T, class C>
int launch_heads(const ScoreArgs &a, dim3 grid, void *stream) {
    const dim3 b(kBlock);
    if (a.heads == 1) return launch(score_kernel<D, 1, T, C>, grid, b, stream, a);
    if (a.heads == 2) return launch(score_kernel<D, 2, T, C>, grid, b, stream, a);
    if (a.heads <= 4) return launch(score_kernel<D, 4, T, C>, grid, b, stream, a);
    if (a.heads <= 8) return launch(score_kernel<D, 8, T, C>, grid, b, stream, a);
    return launch(score_kernel<D, 16, T, C>, grid, b, stream, a);
}

template <int D>
int launch_dim(const ScoreArgs &a, int act, int code, dim3 grid, void *stream) {
    if (code == PAGED_KV_E4M3)
        return act == PAGED_KV_BF16 ? launch_heads<D, bf16, E4M3>(a, grid, stream) : launch_heads<D, f16, E4M3>(a, grid, stream);
    return act == PAGED_KV_BF16 ? launch_heads<D, bf16, Int8>(a, grid, stream) : launch_heads<D, f16, Int8>(a, grid, stream);
}

}  // namespace
}  // namespace paged

extern "C" int paged_kv_score(const paged_kv_cache *cache, int32_t act, const void *q, int64_t q_row, int64_t q_head,
                              int32_t heads, const float *w, const int32_t *table, int32_t table_stride,
                              int32_t table_width, const int32_t *row_request, int32_t n_requests,
                              const int32_t *row_lengths, int32_t n_rows, float scale, float *scores,
                              const int64_t *row_offsets, void *stream) {
    using namespace paged;
    const int rc = check_cache(cache, false);
    if (rc != PAGED_KV_OK) return rc;
    if ((act != PAGED_KV_BF16 && act != PAGED_KV_F16) || n_rows < 0 || n_requests < 0 || heads < 1 ||
        table_width < 1 || table_stride < table_width)
        return PAGED_KV_EINVAL;
    if (n_rows == 0) return PAGED_KV_OK;
    if (!q || !w || !row_request || !row_lengths || !scores || !row_offsets || (n_requests > 0 && !table) ||
        !aligned16(q) || q_row % 8 || q_head % 8)
        return PAGED_KV_EINVAL;
    if (cache->head_dim == 256 || cache->n_heads != 1 || heads > 128) return PAGED_KV_EUNSUPPORTED;
    const int lp = log2_page(cache->page);
    if (((int64_t)table_width << lp) > 0x7FFFFFFF - kTokens) return PAGED_KV_EUNSUPPORTED;
    if (device_cus() == 0) return PAGED_KV_EUNSUPPORTED;
    ScoreArgs a = {(const uint8_t *)cache->k, cache->k_scale, cache->page_stride, cache->scale_stride, cache->n_pages,
                   lp, q, q_row, q_head, heads, w, table, table_stride, table_width, row_request, row_lengths,
                   n_requests, n_rows, 1, scale, scores, row_offsets};
    a.window = n_rows > n_requests ? 128 : 1;
    while ((n_rows + a.window - 1) / a.window > 65535) a.window *= 2;
    const dim3 grid((unsigned)((((int64_t)table_width << lp) + kTokens - 1) / kTokens),
                    (unsigned)((n_rows + a.window - 1) / a.window));
    return cache->head_dim == 64 ? launch_dim<64>(a, act, cache->code, grid, stream)
                                 : launch_dim<128>(a, act, cache->code, grid, stream);
}
