// The score rows that a Top-K selects from: s_ij = scale sum_h w_ih relu(q_ih . k_j).
//
// A wave keeps the keys of some tokens as the columns of 32 x 32 x 16 products
// and passes queries by, from LDS.  The 32 rows of a product are laid out so
// that all heads of a query row lie in the accumulator of one lane, which adds
// them without crossing lanes; the columns so that a lane's tokens follow each
// other, for wide stores; the dimensions so that a lane's codes come in
// 16-byte pieces.
//   many rows (score_block_kernel): bound by the matrix products and the two
//     vector operations behind each of their results (a maximum and a
//     multiply-add), and by the 4 bytes written for each;
//   single rows (score_row_kernel): bound by the keys' D bytes a token; every
//     wave streams tokens of its own, its next codes already on their way.
#include "paged_common.h"

namespace paged {
namespace {

constexpr int kBlock = 256;
constexpr int kTiles = 4;  // products of 32 query rows x heads in LDS at a time

// Tokens of a lane: what the registers hold beside the sums.
constexpr int tokens_of(int dim, int hp) { return dim == 64 && hp >= 4 ? 4 : 2; }

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
    int n_requests, n_rows, window, steps;
    float scale;
    float *scores;
    const int64_t *row_offsets;
};

typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef float f32x2_any __attribute__((ext_vector_type(2), aligned(4)));

// The part of a product's 32 rows that row mm is: half wave (mm >> 2) & 1 holds it
// at place 4 (mm >> 3) + (mm & 3) of its 16 accumulators.  HP heads to a query
// row (a power of two up to 16; more heads take further products).
template <int HP>
struct Rows {
    static constexpr int COUNT = 32 / HP, HALF = 16 / HP;  // query rows of a product, and of a half wave
    static __device__ int row(int mm) { return ((mm >> 2) & 1) * HALF + (4 * (mm >> 3) + (mm & 3)) / HP; }
    static __device__ int head(int mm) { return (4 * (mm >> 3) + (mm & 3)) % HP; }
};

// Keys: NT tokens of a lane, from token `tok` on (in one page), codes in 16-byte pieces g, g + 2, ..
template <int D, int NT>
struct Keys {
    u32x4 x[NT][D / 32];
    float scale;  // times the call's; -inf where the page is not in the cache
};

template <int D, int NT>
__device__ void load_keys(Keys<D, NT> &k, const ScoreArgs &a, int pg, int tok, int g) {
    const bool there = pg >= 0 && pg < a.n_pages;
    const uint8_t *p = a.k + (there ? pg : 0) * a.page_stride + (int64_t)(tok & ((1 << a.lp) - 1)) * D + 16 * g;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int j = 0; j < D / 32; ++j) k.x[t][j] = *(const u32x4 *)(p + t * D + 32 * j);
    k.scale = there ? a.ks[pg * a.scale_stride] : 0.0f;
    k.scale = there ? k.scale * a.scale : -__builtin_inff();
}

template <int D, class T>
__device__ typename Act<T>::frag query(const uint8_t *row, int step, int g) {
    return __builtin_bit_cast(typename Act<T>::frag, *(const u32x4 *)(row + 64 * (step >> 1) + 32 * g + 16 * (step & 1)));
}

template <int NT>
__device__ void put(float *to, const float (&x)[NT], float scale, int left) {
    float y[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) y[t] = scale == -__builtin_inff() ? scale : x[t] * scale;
    if (left >= NT) {
        if constexpr (NT == 4) *(f32x4_any *)to = f32x4_any{y[0], y[1], y[2], y[3]};
        else *(f32x2_any *)to = f32x2_any{y[0], y[1]};
    } else {
#pragma unroll
        for (int t = 0; t < NT; ++t)
            if (t < left) to[t] = y[t];
    }
}

// Windows of rows: workgroup = (4 waves x 32 NT tokens, `window` rows).
template <int D, int HP, class T, class C>
__global__ __launch_bounds__(kBlock, 2) void score_block_kernel(ScoreArgs a) {
    constexpr int NT = tokens_of(D, HP);
    typedef Rows<HP> R;
    constexpr int PIECES = 32 * kTiles * D / 8 / kBlock;  // 16-byte pieces of queries that a thread stages
    __shared__ alignas(16) uint8_t qs[32 * kTiles][2 * D + 16];
    __shared__ alignas(16) float ws[kTiles][2][16];  // by half wave
    __shared__ int64_t offs[kTiles][R::COUNT];
    __shared__ int lens[kTiles][R::COUNT];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = lane & 31, g = lane >> 5;
    const int chunks = (a.heads + HP - 1) / HP;  // more than one only where HP is 16
    const int wave_tok = (int)blockIdx.x * (kBlock / 64 * 32 * NT) + 32 * NT * wave, tok = wave_tok + NT * n;
    const int row_end = min((int)(blockIdx.y + 1) * a.window, a.n_rows);
    const int64_t cap = (int64_t)a.table_width << a.lp;

    int row = blockIdx.y * a.window;
    while (row < row_end) {
        // the rows from here on that share their request
        const int request = a.row_request[row];
        int stop = row;
        for (bool on = true; on && stop < row_end;) {
            const int i = stop + lane;
            const uint64_t other = __ballot(i >= row_end || a.row_request[i] != request);
            on = other == 0;
            stop += on ? 64 : __builtin_ctzll(other);
        }
        const int first = row;
        row = stop;
        if (request < 0 || request >= a.n_requests) continue;
        typename Act<T>::frag k[NT][D / 16];
        float scale;
        {
            Keys<D, NT> raw;
            load_keys<D, NT>(raw, a, tok < cap ? a.table[(int64_t)request * a.table_stride + (tok >> a.lp)] : -1, tok, g);
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int j = 0; j < D / 32; ++j) {
                    k[t][2 * j] = eight<C, T>(raw.x[t][j][0], raw.x[t][j][1]);
                    k[t][2 * j + 1] = eight<C, T>(raw.x[t][j][2], raw.x[t][j][3]);
                }
            scale = raw.scale;
        }
        const int products = (stop - first + R::COUNT - 1) / R::COUNT * chunks;  // product p: rows p / chunks, heads p % chunks
        u32x4 staged[PIECES];
        float staged_w = 0.0f;
        int64_t staged_off = 0;
        int staged_len = 0;
        const auto fetch = [&](int p0) {
#pragma unroll
            for (int e = 0; e < PIECES; ++e) {
                const int i = tid + e * kBlock, m = i / (D / 8), d = i % (D / 8) * 8, p = p0 + m / 32;
                const int r = first + p / chunks * R::COUNT + R::row(m % 32), h = p % chunks * HP + R::head(m % 32);
                staged[e] = u32x4{0, 0, 0, 0};
                if (r < stop && h < a.heads)
                    staged[e] = *(const u32x4 *)((const char *)a.q + 2 * (r * a.q_row + h * a.q_head + d));
            }
            if (tid < 32 * kTiles) {
                const int half = (tid >> 4) & 1, place = tid & 15, p = p0 + tid / 32;
                const int r = first + p / chunks * R::COUNT + half * R::HALF + place / HP, h = p % chunks * HP + place % HP;
                staged_w = r < stop && h < a.heads ? a.w[(int64_t)r * a.heads + h] : 0.0f;
            }
            if (tid < kTiles * R::COUNT) {
                const int r = first + (p0 + tid / R::COUNT) / chunks * R::COUNT + tid % R::COUNT;
                staged_len = r < stop ? (int)min((int64_t)max(a.row_lengths[r], 0), cap) : 0;
                staged_off = r < stop ? a.row_offsets[r] : 0;
            }
        };
        fetch(0);
        float sum[R::HALF][NT];
        for (int p0 = 0; p0 < products; p0 += kTiles) {
            __syncthreads();
#pragma unroll
            for (int e = 0; e < PIECES; ++e) {
                const int i = tid + e * kBlock;
                *(u32x4 *)&qs[i / (D / 8)][i % (D / 8) * 16] = staged[e];
            }
            if (tid < 32 * kTiles) ws[tid / 32][(tid >> 4) & 1][tid & 15] = staged_w;
            if (tid < kTiles * R::COUNT) {
                lens[tid / R::COUNT][tid % R::COUNT] = staged_len;
                offs[tid / R::COUNT][tid % R::COUNT] = staged_off;
            }
            __syncthreads();
            if (p0 + kTiles < products) fetch(p0 + kTiles);
            for (int m = 0; m < kTiles && p0 + m < products; ++m) {
                const int c = (p0 + m) % chunks;
                if (c == 0)
#pragma unroll
                    for (int i = 0; i < R::HALF; ++i)
#pragma unroll
                        for (int t = 0; t < NT; ++t) sum[i][t] = 0.0f;
                f32x16 s[NT];
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[t][i] = 0.0f;
#pragma unroll
                for (int j = 0; j < D / 16; ++j) {
                    const auto x = query<D, T>(qs[32 * m + n], j, g);
#pragma unroll
                    for (int t = 0; t < NT; ++t) s[t] = Act<T>::mfma32(x, k[t][j], s[t]);
                }
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float w = ws[m][g][i];
#pragma unroll
                    for (int t = 0; t < NT; ++t) sum[i / HP][t] = fmaf(w, fmaxf(s[t][i], 0.0f), sum[i / HP][t]);
                }
                if (c == chunks - 1)
#pragma unroll
                    for (int i = 0; i < R::HALF; ++i) {
                        const int r = g * R::HALF + i;
                        put<NT>(a.scores + offs[m][r] + tok, sum[i], scale, lens[m][r] - tok);
                    }
            }
        }
        __syncthreads();
    }
}

// Single rows: workgroup = (row, 4 waves x `steps` x 32 NT tokens).
template <int D, int HP, class T, class C>
__global__ __launch_bounds__(kBlock, 2) void score_row_kernel(ScoreArgs a) {
    constexpr int NT = tokens_of(D, HP);
    __shared__ alignas(16) uint8_t qs[128][2 * D + 16];
    __shared__ alignas(16) float ws[128];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = lane & 31, g = lane >> 5;
    const int row = blockIdx.y, request = a.row_request[row];
    if (request < 0 || request >= a.n_requests) return;
    const int len = (int)min((int64_t)max(a.row_lengths[row], 0), (int64_t)a.table_width << a.lp);
    const int64_t wg_tok = (int64_t)blockIdx.x * (kBlock / 64 * 32 * NT) * a.steps;
    if (wg_tok >= len) return;
    // wave w's steps are its workgroup's tiles w, w + 4, ..
    const int tok0 = (int)wg_tok + 32 * NT * wave;
    const int *pages = a.table + (int64_t)request * a.table_stride;
    const auto page_of = [&](int s) {
        const int tok = tok0 + s * (kBlock / 64 * 32 * NT) + NT * n;
        return s < a.steps && tok < len ? pages[tok >> a.lp] : -1;
    };
    int page = page_of(0);

    // the row's queries: product rows that no head has are 0, with weight 0
    const int chunks = (a.heads + HP - 1) / HP;
    for (int i = tid; i < chunks * HP * (D / 8); i += kBlock) {
        const int h = i / (D / 8), d = i % (D / 8) * 8;
        u32x4 x = {0, 0, 0, 0};
        if (h < a.heads) x = *(const u32x4 *)((const char *)a.q + 2 * (row * a.q_row + h * a.q_head + d));
        *(u32x4 *)&qs[h][2 * d] = x;
    }
    for (int h = tid; h < chunks * HP; h += kBlock) ws[h] = h < a.heads ? a.w[(int64_t)row * a.heads + h] : 0.0f;
    __syncthreads();

    Keys<D, NT> now, next;
    load_keys<D, NT>(now, a, page, tok0 + NT * n, g);
    page = page_of(1);
    float *out = a.scores + a.row_offsets[row];
    // half wave g's places i hold heads of this row where g = 0 alone: the other half repeats them
    const int mm = ((n >> 3) << 2) + (n & 3);  // place of product row n
    for (int s = 0; s < a.steps; ++s) {
        const int tile = tok0 + s * (kBlock / 64 * 32 * NT);
        if (tile >= len) break;
        const bool more = s + 1 < a.steps && tile + kBlock / 64 * 32 * NT < len;
        if (more) {
            load_keys<D, NT>(next, a, page, tile + kBlock / 64 * 32 * NT + NT * n, g);
            page = page_of(s + 2);
        }
        float sum[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) sum[t] = 0.0f;
        for (int c = 0; c < chunks; ++c) {
            f32x16 x[NT];
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i) x[t][i] = 0.0f;
#pragma unroll
            for (int j = 0; j < D / 16; ++j) {
                const auto q = query<D, T>(qs[c * HP + (mm & (HP - 1))], j, g);
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    const u32x4 raw = now.x[t][j >> 1];
                    const auto k = (j & 1) ? eight<C, T>(raw[2], raw[3]) : eight<C, T>(raw[0], raw[1]);
                    x[t] = Act<T>::mfma32(q, k, x[t]);
                }
            }
#pragma unroll
            for (int i = 0; i < HP; ++i) {
                const float w = ws[c * HP + i];
#pragma unroll
                for (int t = 0; t < NT; ++t) sum[t] = fmaf(w, fmaxf(x[t][i], 0.0f), sum[t]);
            }
        }
        if (g == 0) put<NT>(out + tile + NT * n, sum, now.scale, len - (tile + NT * n));
        if (more) now = next;
    }
}

template <int D, int HP, class T, class C>
int launch_rows(const ScoreArgs &a, dim3 grid, void *stream) {
    return a.window == 1 ? launch(score_row_kernel<D, HP, T, C>, grid, dim3(kBlock), stream, a)
                         : launch(score_block_kernel<D, HP, T, C>, grid, dim3(kBlock), stream, a);
}

template <int D, class T, class C>
int launch_heads(const ScoreArgs &a, dim3 grid, void *stream) {
    if (a.heads == 1) return launch_rows<D, 1, T, C>(a, grid, stream);
    if (a.heads == 2) return launch_rows<D, 2, T, C>(a, grid, stream);
    if (a.heads <= 4) return launch_rows<D, 4, T, C>(a, grid, stream);
    if (a.heads <= 8) return launch_rows<D, 8, T, C>(a, grid, stream);
    return launch_rows<D, 16, T, C>(a, grid, stream);
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
    if (((int64_t)table_width << lp) > 0x7FFFFFFF - 4096) return PAGED_KV_EUNSUPPORTED;
    if (device_cus() == 0) return PAGED_KV_EUNSUPPORTED;
    ScoreArgs a = {(const uint8_t *)cache->k, cache->k_scale, cache->page_stride, cache->scale_stride, cache->n_pages,
                   lp, q, q_row, q_head, heads, w, table, table_stride, table_width, row_request, row_lengths,
                   n_requests, n_rows, 1, 1, scale, scores, row_offsets};
    const int64_t cap = (int64_t)table_width << lp;
    int tokens = kBlock / 64 * 32 * tokens_of(cache->head_dim, heads > 2 ? 4 : 1);  // of a workgroup's step
    if (n_rows > n_requests || n_rows > 65535) {
        // rows share their keys: 128 of them to a workgroup
        a.window = 128;
        while (((int64_t)n_rows + a.window - 1) / a.window > 65535) a.window *= 2;
    } else {
        // a workgroup's steps: up to 4, as long as 1024 workgroups are left
        while (a.steps < 4 && cap / (2 * a.steps * tokens) * n_rows >= 1024) a.steps *= 2;
        tokens *= a.steps;
    }
    const dim3 grid((unsigned)((cap + tokens - 1) / tokens), (unsigned)((n_rows + a.window - 1) / a.window));
    return cache->head_dim == 64 ? launch_dim<64>(a, act, cache->code, grid, stream)
                                 : launch_dim<128>(a, act, cache->code, grid, stream);
}
