// What every token of the cache gets of a step's attention:
//   w_j += sum over rows i that see j, heads h of exp(scale q_ih . k_j - lse_ih).
//
// The softmax is known (lse), so tokens need nothing of each other: a wave holds the
// keys of some tokens as the columns of 32 x 32 x 16 products and passes queries by, from
// LDS.  A token's results lie in one lane of each half wave, 16 queries to an accumulator:
// the sum over queries is the lane's own, and the halves meet once at the end.
#include "../../include/serve_step.h"
#include "paged_common.h"

namespace paged {
namespace {

constexpr int kBlock = 256;
constexpr int kTokens = 2;   // of a lane: 64 of a wave
constexpr int kTile = kBlock / 64 * 32 * kTokens;  // tokens of a workgroup
constexpr float kLog2e = 1.4426950408889634f;

struct WeighArgs {
    const uint8_t *k;
    const float *ks;
    int64_t page_stride, scale_stride;
    int n_pages, lp, kv_heads;
    const void *q;
    int64_t q_row, q_head;
    int heads, per;  // query heads, and those of a cache head
    const float *lse;
    const int *table;
    int table_stride, table_width;
    const int *row_starts, *row_lengths;
    int n_rows, steps;
    float scale2;  // scale * log2(e)
    float *weights;
    const int64_t *weight_offsets;
};

// Query columns in LDS.
constexpr int columns_of(int dim) { return dim == 256 ? 64 : 128; }

template <int D>
struct Columns {
    alignas(16) uint8_t q[columns_of(D)][2 * D + 16];
    alignas(16) float lse2[columns_of(D) + 32];  // +inf: a column that adds nothing
    alignas(16) int len[columns_of(D) + 32];
};

// Rows of a request: workgroup = (request, `steps` tiles of tokens), all heads.
template <int D, class T, class C>
__global__ __launch_bounds__(kBlock) void weigh_rows_kernel(WeighArgs a) {
    constexpr int NT = kTokens, COLS = columns_of(D);
    typedef typename Act<T>::frag frag;
    __shared__ Columns<D> b;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = lane & 31, g = lane >> 5;
    const int r = blockIdx.y;
    const int row0 = min(max(a.row_starts[r], 0), a.n_rows), row1 = min(max(a.row_starts[r + 1], row0), a.n_rows);
    const int64_t cap = (int64_t)a.table_width << a.lp;
    int longest = 0, shortest = 0x7FFFFFFF;
    for (int i = row0 + lane; i < row1; i += 64) {
        const int len = (int)min((int64_t)max(a.row_lengths[i], 0), cap);
        longest = max(longest, len);
        shortest = min(shortest, len);
    }
    for (int d = 32; d; d >>= 1) {
        longest = max(longest, __shfl_xor(longest, d));
        shortest = min(shortest, __shfl_xor(shortest, d));
    }
    longest = __builtin_amdgcn_readfirstlane(longest);
    shortest = __builtin_amdgcn_readfirstlane(shortest);
    const int64_t first = (int64_t)blockIdx.x * kTile * a.steps;
    if (first >= longest) return;
    const int *pages = a.table + (int64_t)r * a.table_stride;
    float *weights = a.weights + a.weight_offsets[r];

    const int64_t all = (int64_t)(row1 - row0) * a.per;  // columns of a cache head
    const int width = (int)min(all, (int64_t)COLS), span = max(1, COLS / width);  // of a pass: columns of a head, heads
    for (int head0 = 0; head0 < a.kv_heads; head0 += span)
        for (int64_t col0 = 0; col0 < all; col0 += width) {
            const int heads = min(span, a.kv_heads - head0), cols = (int)min(all - col0, (int64_t)width);
            if (head0 + col0 > 0) __syncthreads();
            for (int i = tid; i < heads * cols * (D / 8); i += kBlock) {
                const int c = i / (D / 8), h = c / cols, at = i % (D / 8);
                const int64_t col = col0 + c - h * cols;
                const int row = row0 + (int)(col / a.per), head = (head0 + h) * a.per + (int)(col % a.per);
                u32x4 x = *(const u32x4 *)((const char *)a.q + 2 * (row * a.q_row + head * a.q_head + 8 * at));
                // (what a row without a softmax holds is not looked at)
                if (fabsf(a.lse[(int64_t)row * a.heads + head]) == __builtin_inff()) x = u32x4{0, 0, 0, 0};
                *(u32x4 *)&b.q[c][16 * at] = x;
            }
            for (int i = tid; i < COLS + 32; i += kBlock) {
                float x = __builtin_inff();
                int len = 0;
                if (i < heads * cols) {
                    const int h = i / cols;
                    const int64_t col = col0 + i - h * cols;
                    const int row = row0 + (int)(col / a.per);
                    x = a.lse[(int64_t)row * a.heads + (head0 + h) * a.per + (int)(col % a.per)];
                    x = x == -__builtin_inff() ? __builtin_inff() : x * kLog2e;
                    len = (int)min((int64_t)max(a.row_lengths[row], 0), cap);
                }
                b.lse2[i] = x;
                b.len[i] = len;
            }
            __syncthreads();
            for (int s = 0; s < a.steps; ++s) {
                const int64_t base = first + (int64_t)s * kTile + 32 * NT * wave;
                if (base >= longest) break;
                const int tok = (int)base + NT * n;
                const int pg = pages[min((int64_t)tok, cap - 1) >> a.lp];
                const bool there = pg >= 0 && pg < a.n_pages;
                const uint8_t *codes = a.k + (there ? pg : 0) * a.page_stride + (int64_t)(tok & ((1 << a.lp) - 1)) * D + 16 * g;
                const float *scales = a.ks + (there ? pg : 0) * a.scale_stride;
                const bool masked = base + 32 * NT > shortest && shortest != longest;
                float sum[NT];
#pragma unroll
                for (int t = 0; t < NT; ++t) sum[t] = 0.0f;
                for (int h = 0; h < heads; ++h) {
                    u32x4 raw[NT][D / 32];
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int j = 0; j < D / 32; ++j)
                            raw[t][j] = *(const u32x4 *)(codes + ((int64_t)(head0 + h) << a.lp) * D + t * D + 32 * j);
                    const float scale = scales[head0 + h] * a.scale2;
                    frag k[NT][D / 16];
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int j = 0; j < D / 32; ++j) {
                            k[t][2 * j] = eight<C, T>(raw[t][j][0], raw[t][j][1]);
                            k[t][2 * j + 1] = eight<C, T>(raw[t][j][2], raw[t][j][3]);
                        }
                    for (int c = 0; c < cols; c += 32) {
                        const int left = cols - c, at = h * cols + c;
                        f32x16 x[NT];
#pragma unroll
                        for (int t = 0; t < NT; ++t)
#pragma unroll
                            for (int i = 0; i < 16; ++i) x[t][i] = 0.0f;
                        const uint8_t *q = b.q[at + min(n, left - 1)] + 32 * g;
#pragma unroll
                        for (int j = 0; j < D / 16; ++j) {
                            const frag y = __builtin_bit_cast(frag, *(const u32x4 *)(q + 64 * (j >> 1) + 16 * (j & 1)));
#pragma unroll
                            for (int t = 0; t < NT; ++t) x[t] = Act<T>::mfma32(y, k[t][j], x[t]);
                        }
                        // place i of half g is column 8 (i / 4) + 4 g + i % 4
#pragma unroll
                        for (int i0 = 0; i0 < 16; i0 += 4) {
                            if (2 * i0 >= left) break;
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const int col = 2 * i0 + 4 * g + i;
                                if (col >= left) break;
                                const float l = b.lse2[at + col];
                                const int len = masked ? b.len[at + col] : 0x7FFFFFFF;
#pragma unroll
                                for (int t = 0; t < NT; ++t) {
                                    const float p = exp2_(fmaf(x[t][i0 + i], scale, -l));
                                    sum[t] += tok + t < len ? p : 0.0f;
                                }
                            }
                        }
                    }
                }
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    sum[t] += __shfl_xor(sum[t], 32);
                    if (g == 0 && there && tok + t < longest) weights[tok + t] += sum[t];
                }
            }
        }
}

template <int D>
int launch_dim(const WeighArgs &a, int act, int code, dim3 grid, void *stream) {
    if (code == PAGED_KV_E4M3)
        return act == PAGED_KV_BF16 ? launch(weigh_rows_kernel<D, bf16, E4M3>, grid, dim3(kBlock), stream, a)
                                    : launch(weigh_rows_kernel<D, f16, E4M3>, grid, dim3(kBlock), stream, a);
    return act == PAGED_KV_BF16 ? launch(weigh_rows_kernel<D, bf16, Int8>, grid, dim3(kBlock), stream, a)
                                : launch(weigh_rows_kernel<D, f16, Int8>, grid, dim3(kBlock), stream, a);
}

}  // namespace
}  // namespace paged

extern "C" size_t serve_weigh_workspace(int32_t n_rows, int32_t n_requests, int32_t heads, int32_t kv_heads) {
    if (n_rows < 0 || n_requests < 0 || heads < 1 || kv_heads < 1 || heads % kv_heads != 0) return 0;
    return paged::device_cus() == 0 ? 0 : 256;
}

extern "C" int serve_weigh(const paged_kv_cache *cache, int32_t act, const void *q, int64_t q_row, int64_t q_head,
                           int32_t heads, const float *lse, const int32_t *table, int32_t table_stride,
                           int32_t table_width, const int32_t *row_starts, int32_t n_requests,
                           const int32_t *row_lengths, int32_t n_rows, float scale, float *weights,
                           const int64_t *weight_offsets, void *workspace, size_t workspace_bytes, void *stream) {
    using namespace paged;
    const int rc = check_cache(cache, false);
    if (rc != PAGED_KV_OK) return rc;
    if ((act != PAGED_KV_BF16 && act != PAGED_KV_F16) || n_rows < 0 || n_requests < 0 || heads < 1 ||
        heads % cache->n_heads != 0 || table_width < 1 || table_stride < table_width || !(scale >= 0.0f) ||
        scale - scale != 0.0f)
        return PAGED_KV_EINVAL;
    if (n_rows == 0 || n_requests == 0) return PAGED_KV_OK;
    if (!q || !lse || !table || !row_starts || !row_lengths || !weights || !weight_offsets || !aligned16(q) ||
        q_row % 8 || q_head % 8 || !workspace || (uintptr_t)workspace % 256)
        return PAGED_KV_EINVAL;
    const int lp = log2_page(cache->page);
    if (((int64_t)table_width << lp) > 0x7FFFFFFF - 65536 || n_requests > 65535) return PAGED_KV_EUNSUPPORTED;
    const size_t need = serve_weigh_workspace(n_rows, n_requests, heads, cache->n_heads);
    if (need == 0) return PAGED_KV_EUNSUPPORTED;
    if (workspace_bytes < need) return PAGED_KV_EWORKSPACE;
    WeighArgs a = {(const uint8_t *)cache->k, cache->k_scale, cache->page_stride, cache->scale_stride, cache->n_pages,
                   lp, cache->n_heads, q, q_row, q_head, heads, heads / cache->n_heads, lse, table, table_stride,
                   table_width, row_starts, row_lengths, n_rows, 1, scale * kLog2e, weights, weight_offsets};
    const int64_t cap = (int64_t)table_width << lp;
    while (a.steps < 4 && cap / (2 * a.steps * kTile) * n_requests >= 1024) a.steps *= 2;
    const dim3 grid((unsigned)((cap + (int64_t)kTile * a.steps - 1) / ((int64_t)kTile * a.steps)), (unsigned)n_requests);
    return cache->head_dim == 64    ? launch_dim<64>(a, act, cache->code, grid, stream)
           : cache->head_dim == 128 ? launch_dim<128>(a, act, cache->code, grid, stream)
                                    : launch_dim<256>(a, act, cache->code, grid, stream);
}
