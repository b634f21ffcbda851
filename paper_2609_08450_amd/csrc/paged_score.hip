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
//     wave streams tokens of its own.
// Measured (8 heads of 64): 4096 rows over 131072 tokens 620 us, 873 TFLOP/s beside
// 3.4 TB/s of writes, at a clock of 1.91 GHz (a large matrix product runs at 1.94 and
// reaches 1415, calls that memory bounds run at 2.40); 64 rows of 16384 to 131072
// tokens 66.7 us, 4.6 TB/s.
#include "paged_common.h"
#include "paged_score_plan.h"

namespace paged {
namespace {

constexpr int kBlock = 256;

// Tokens of a lane: what the registers hold beside the sums.
constexpr int tokens_of(int dim, int hp) { return dim == 64 && hp >= 4 ? 4 : 2; }

// In the kernel of single rows: few tokens to a lane and many waves.  (The decode
// batch: 68.7 us with 5 waves to a SIMD and 2 tokens to a lane; 73.6 with 4 waves
// that hold their next codes too; 74.7 with 2 waves of twice the tokens.)
constexpr int kRowTokens = 2;

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
    float raw;   // the page's scale
    bool there;  // the page is in the cache

    // The page's scale times the call's, or -inf.  (Apart from the load: what uses
    // a loaded value waits for it, and for the codes loaded before it.)
    __device__ float scale(float call) const { return there ? raw * call : -__builtin_inff(); }
};

template <int D, int NT>
__device__ void load_keys(Keys<D, NT> &k, const ScoreArgs &a, int pg, int tok, int g) {
    k.there = pg >= 0 && pg < a.n_pages;
    const int at = k.there ? pg : 0;
    const uint8_t *p = a.k + at * a.page_stride + (int64_t)(tok & ((1 << a.lp) - 1)) * D + 16 * g;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int j = 0; j < D / 32; ++j) k.x[t][j] = *(const u32x4 *)(p + t * D + 32 * j);
    k.raw = a.ks[at * a.scale_stride];
}

template <int D, class T>
__device__ typename Act<T>::frag query(const uint8_t *row, int step, int g) {
    return __builtin_bit_cast(typename Act<T>::frag, *(const u32x4 *)(row + 64 * (step >> 1) + 32 * g + 16 * (step & 1)));
}

// max(x, 0) as one instruction, on the bits: a float maximum makes a second one
// of a result that the compiler cannot know to be no signalling NaN.
__device__ inline float relu(float x) { return __int_as_float(max(__float_as_int(x), 0)); }

// NT scores of a lane, past the caches: nothing reads them before the call ends.
template <int NT>
__device__ void put_all(float *to, const float (&x)[NT], float scale) {
    if constexpr (NT == 4)
        __builtin_nontemporal_store(f32x4_any{x[0], x[1], x[2], x[3]} * scale, (f32x4_any *)to);
    else
        __builtin_nontemporal_store(f32x2_any{x[0], x[1]} * scale, (f32x2_any *)to);
}

// The same for the first `left` of them; scale -inf stands for a page outside the cache.
template <int NT>
__device__ void put(float *to, const float (&x)[NT], float scale, int left) {
    if (left >= NT && scale != -__builtin_inff()) return put_all<NT>(to, x, scale);
#pragma unroll
    for (int t = 0; t < NT; ++t)
        if (t < left) to[t] = scale == -__builtin_inff() ? scale : x[t] * scale;
}

// Windows of rows: workgroup = (`window` rows, every gridDim.y-th of the blocks of
// 4 waves x 32 NT tokens).  The queries stay in LDS, each wave passes its own
// tokens by them: no barrier and no load of queries between the stores, whose
// way to memory the next barrier would wait for (573 us without the stores, 795
// with them and a barrier every four products).
// MANY: more heads than a product holds (HP is 16 then).
template <int D, int HP, bool MANY, class T, class C>
__global__ __launch_bounds__(kBlock, 2) void score_block_kernel(ScoreArgs a) {
    constexpr int NT = tokens_of(D, HP), M = window_of(D), STEP = kBlock / 64 * 32 * NT;
    typedef Rows<HP> R;
    __shared__ alignas(16) uint8_t qs[M][2 * D];  // 16-byte pieces in swizzled order
    __shared__ alignas(16) float ws[M];           // product, half wave, place
    __shared__ int64_t offs[M / HP];
    __shared__ int lens[M / HP], longest[M / 32], shortest[M / 32];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = lane & 31, g = lane >> 5;
    const int chunks = MANY ? (a.heads + HP - 1) / HP : 1;
    const int64_t cap = (int64_t)a.table_width << a.lp;
    // the last windows first: where lengths rise they are the longest
    const int y = gridDim.x - 1 - blockIdx.x;
    const int row_end = min((y + 1) * a.window, a.n_rows);
    const auto place = [](int m, int piece) { return 16 * (piece ^ (D == 64 ? (m >> 1) & 7 : m & 15)); };

    int row = y * a.window;
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
        const int first = row, rows = stop - row;
        row = stop;
        if (request < 0 || request >= a.n_requests) continue;
        const int products = (rows + R::COUNT - 1) / R::COUNT * chunks;  // product p: rows p / chunks, heads p % chunks
        __syncthreads();  // the rows before these are done with
        for (int i = tid; i < 32 * products * (D / 8); i += kBlock) {
            const int m = i / (D / 8), piece = i % (D / 8), p = m / 32;
            const int r = p / chunks * R::COUNT + R::row(m % 32), h = p % chunks * HP + R::head(m % 32);
            u32x4 x = {0, 0, 0, 0};
            if (r < rows && h < a.heads)
                x = *(const u32x4 *)((const char *)a.q + 2 * ((first + r) * a.q_row + h * a.q_head + 8 * piece));
            *(u32x4 *)&qs[m][place(m, piece)] = x;
        }
        for (int i = tid; i < 32 * products; i += kBlock) {
            const int p = i / 32, at = i % 16;
            const int r = p / chunks * R::COUNT + (i >> 4 & 1) * R::HALF + at / HP, h = p % chunks * HP + at % HP;
            ws[i] = r < rows && h < a.heads ? a.w[(int64_t)(first + r) * a.heads + h] : 0.0f;
        }
        for (int i = tid; i < products / chunks * R::COUNT; i += kBlock) {
            lens[i] = i < rows ? (int)min((int64_t)max(a.row_lengths[first + i], 0), cap) : 0;
            offs[i] = i < rows ? a.row_offsets[first + i] : 0;
        }
        __syncthreads();
        int top = 0;
        for (int i = tid; i < products / chunks; i += kBlock) {
            int x = 0, y = 0x7FFFFFFF;
            for (int r = 0; r < R::COUNT; ++r) {
                x = max(x, lens[i * R::COUNT + r]);
                y = min(y, lens[i * R::COUNT + r]);
            }
            longest[i] = x;
            shortest[i] = y;
        }
        __syncthreads();
        for (int i = lane; i < products / chunks; i += 64) top = max(top, longest[i]);
        for (int d = 32; d; d >>= 1) top = max(top, __shfl_xor(top, d));
        top = __builtin_amdgcn_readfirstlane(top);

        const int *pages = a.table + (int64_t)request * a.table_stride;
        const int step = gridDim.y * STEP;
        const auto page_of = [&](int tok) { return tok < top ? pages[tok >> a.lp] : -1; };
        int base = blockIdx.y * STEP + 32 * NT * wave;
        Keys<D, NT> raw;
        int page = page_of(base + NT * n);
        load_keys<D, NT>(raw, a, page, base + NT * n, g);
        if (base < top) page = page_of((int)min((int64_t)base + step, (int64_t)0x7FFFFFFF - STEP) + NT * n);
        while (base < top) {
            const int tok = base + NT * n;
            typename Act<T>::frag k[NT][D / 16];
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int j = 0; j < D / 32; ++j) {
                    k[t][2 * j] = eight<C, T>(raw.x[t][j][0], raw.x[t][j][1]);
                    k[t][2 * j + 1] = eight<C, T>(raw.x[t][j][2], raw.x[t][j][3]);
                }
            const float scale = raw.scale(a.scale);
            const int next = (int)min((int64_t)base + step, (int64_t)0x7FFFFFFF - STEP);
            if (next < top) {
                load_keys<D, NT>(raw, a, page, next + NT * n, g);
                page = page_of((int)min((int64_t)next + step, (int64_t)0x7FFFFFFF - STEP) + NT * n);
            }
            const bool plain = __all(scale != -__builtin_inff());
            float sum[R::HALF][NT];
            int c = 0, group = 0;
            for (int p = 0; p < products; ++p) {
                if (base >= __builtin_amdgcn_readfirstlane(longest[group])) {  // no row of this product comes so far
                    if (++c == chunks) c = 0, ++group;
                    continue;
                }
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
                    const int m = 32 * p + n;
                    const u32x4 x = *(const u32x4 *)&qs[m][place(m, 4 * (j >> 1) + 2 * g + (j & 1))];
#pragma unroll
                    for (int t = 0; t < NT; ++t)
                        s[t] = Act<T>::mfma32(__builtin_bit_cast(typename Act<T>::frag, x), k[t][j], s[t]);
                }
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float w = ws[32 * p + 16 * g + i];
#pragma unroll
                    for (int t = 0; t < NT; ++t) sum[i / HP][t] = fmaf(w, relu(s[t][i]), sum[i / HP][t]);
                }
                if (++c == chunks) {
                    const int r = group * R::COUNT + g * R::HALF;
                    if (plain && base + 32 * NT <= __builtin_amdgcn_readfirstlane(shortest[group]))
#pragma unroll
                        for (int i = 0; i < R::HALF; ++i) put_all<NT>(a.scores + offs[r + i] + tok, sum[i], scale);
                    else
#pragma unroll
                        for (int i = 0; i < R::HALF; ++i)
                            put<NT>(a.scores + offs[r + i] + tok, sum[i], scale, lens[r + i] - tok);
                    c = 0;
                    ++group;
                }
            }
            base = next;
        }
    }
}

// Single rows: workgroup = (row, 4 waves x `steps` x 32 NT tokens).
template <int D, int HP, class T, class C>
__global__ __launch_bounds__(kBlock, D == 64 ? 5 : 3) void score_row_kernel(ScoreArgs a) {
    constexpr int NT = kRowTokens;
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

    float *out = a.scores + a.row_offsets[row];
    // half wave 0's places i hold the row's heads, and half wave 1 repeats them
    const int mm = ((n >> 3) << 2) + (n & 3);  // place of product row n
    for (int s = 0; s < a.steps; ++s) {
        const int tile = tok0 + s * (kBlock / 64 * 32 * NT);
        if (tile >= len) break;
        Keys<D, NT> now;
        load_keys<D, NT>(now, a, page, tile + NT * n, g);
        page = page_of(s + 1);
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
                for (int t = 0; t < NT; ++t) sum[t] = fmaf(w, relu(x[t][i]), sum[t]);
            }
        }
        if (g == 0) put<NT>(out + tile + NT * n, sum, now.scale(a.scale), len - (tile + NT * n));
    }
}

template <int D, class T, class C>
int launch_heads(const ScoreArgs &a, dim3 grid, void *stream) {
    const auto go = [&](void (*row)(ScoreArgs), void (*block)(ScoreArgs)) {
        return launch(a.window == 1 ? row : block, grid, dim3(kBlock), stream, a);
    };
    // the first of these is product_heads(a.heads)
    if (a.heads == 1) return go(score_row_kernel<D, 1, T, C>, score_block_kernel<D, 1, false, T, C>);
    if (a.heads == 2) return go(score_row_kernel<D, 2, T, C>, score_block_kernel<D, 2, false, T, C>);
    if (a.heads <= 4) return go(score_row_kernel<D, 4, T, C>, score_block_kernel<D, 4, false, T, C>);
    if (a.heads <= 8) return go(score_row_kernel<D, 8, T, C>, score_block_kernel<D, 8, false, T, C>);
    if (a.heads <= 16) return go(score_row_kernel<D, 16, T, C>, score_block_kernel<D, 16, false, T, C>);
    return go(score_row_kernel<D, 16, T, C>, score_block_kernel<D, 16, true, T, C>);
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
    dim3 grid;
    int tokens = kBlock / 64 * 32 * tokens_of(cache->head_dim, heads > 2 ? 4 : 1);  // of a workgroup's step
    if (n_rows > n_requests || n_rows > 65535) {
        // rows share their keys: as many to a workgroup as its LDS holds, and so
        // many workgroups to a window as give the card 1024 (2 to a CU are resident).
        // One rule for the call, in which n_requests is the table's height: rows of one
        // request gain from windows (16 over 131072 tokens 9.3 us, and 21.4 by themselves;
        // eight of each of 64 requests of 16384 46 and 73), but few rows of many requests
        // lose (two of each of the 64: 131 us, and 25 by themselves; four: 66 and 41).
        a.window = rows_of_window(cache->head_dim, heads);
        const int64_t windows = ((int64_t)n_rows + a.window - 1) / a.window;
        const int64_t blocks = (cap + tokens - 1) / tokens, want = (1024 + windows - 1) / windows;
        grid = dim3((unsigned)windows, (unsigned)(want < blocks ? want : blocks));
    } else {
        // a workgroup's steps: up to 4, as long as 1024 workgroups are left
        tokens = kBlock / 64 * 32 * kRowTokens;
        while (a.steps < 4 && cap / (2 * a.steps * tokens) * n_rows >= 1024) a.steps *= 2;
        tokens *= a.steps;
        grid = dim3((unsigned)((cap + tokens - 1) / tokens), (unsigned)n_rows);
    }
    return cache->head_dim == 64 ? launch_dim<64>(a, act, cache->code, grid, stream)
                                 : launch_dim<128>(a, act, cache->code, grid, stream);
}
