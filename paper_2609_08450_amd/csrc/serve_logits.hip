// Penalties, biases and masks on logits.
//
// A workgroup takes a chunk of one row's vocabulary into registers.  How often the
// row's tokens fall into the chunk is counted in LDS, a word to a token (whole
// numbers: their order does not matter), then every element reads its word; the
// same words then hold, for each biased token, the last entry of the list that
// names it.  Every workgroup of a row reads the row's whole lists, out of the L2.
// Bound by memory: a logit read and an FP32 number written.
#include "../../include/serve_step.h"
#include "paged_common.h"

// every step of the definition is rounded: no product and sum become one operation
#pragma clang fp contract(off)

namespace paged {
namespace {

constexpr int kBlock = 512;
constexpr u32 kSeen = 0x80000000u;  // of a word: the token is among the row's; below: how often behind the prompt

struct AdjustArgs {
    const void *x;
    int64_t x_row;
    float *out;
    int64_t out_row;
    int n_rows, vocab;
    serve_lists l;
};

// V neighbouring logits as loaded, and as floats.
template <class T, int V>
struct Logits {
    typedef T type __attribute__((ext_vector_type(V)));
    static __device__ float at(const type &x, int i) { return (float)x[i]; }
};
template <class T>
struct Logits<T, 1> {
    typedef T type;
    static __device__ float at(const type &x, int) { return (float)x; }
};

// V: elements that lie together in x and in out, both aligned; E: of a thread.
template <class T, int V, int E>
__global__ __launch_bounds__(kBlock) void adjust_kernel(AdjustArgs a) {
    typedef Logits<T, V> L;
    typedef float out_t __attribute__((ext_vector_type(V)));
    constexpr int CHUNK = kBlock * E;
    __shared__ u32 words[CHUNK];
    const int tid = threadIdx.x, row = blockIdx.y;
    const int first = blockIdx.x * CHUNK, left = min(CHUNK, a.vocab - first);
    const T *x = (const T *)a.x + row * a.x_row + first;
    // piece i of the thread: elements V (i kBlock + tid) on
    typename L::type raw[E / V];
#pragma unroll
    for (int i = 0; i < E / V; ++i) {
        const int at = V * (i * kBlock + tid);
        if (at + V <= left) raw[i] = *(const typename L::type *)(x + at);
        else
            for (int j = 0; j < V; ++j) {
                const T one = at + j < left ? x[at + j] : (T)0.0f;
                if constexpr (V == 1) raw[i] = one;
                else raw[i][j] = one;
            }
    }
    int64_t begin = 0, end = 0, bias_begin = 0, bias_end = 0;
    if (a.l.tokens) {
        begin = a.l.token_starts[row];
        end = a.l.token_starts[row + 1];
    }
    if (a.l.bias_ids) {
        bias_begin = a.l.bias_starts[row];
        bias_end = a.l.bias_starts[row + 1];
    }
    const u32 *allowed = nullptr;
    if (a.l.mask) {
        const int m = a.l.row_mask ? a.l.row_mask[row] : row;
        if (m >= 0 && m < a.l.n_masks) allowed = a.l.mask + m * a.l.mask_stride;
    }
    const auto clear = [&] {
        for (int i = tid; i < CHUNK; i += kBlock) words[i] = 0;
        __syncthreads();
    };
    float y[E];
#pragma unroll
    for (int i = 0; i < E; ++i) y[i] = L::at(raw[i / V], i % V);

    if (end > begin) {
        const int64_t prompt = begin + (a.l.prompt_lens ? max(a.l.prompt_lens[row], 0) : 0);
        const float repetition = a.l.repetition ? a.l.repetition[row] : 1.0f;
        const float frequency = a.l.frequency ? a.l.frequency[row] : 0.0f;
        const float presence = a.l.presence ? a.l.presence[row] : 0.0f;
        clear();
        for (int64_t i = begin + tid; i < end; i += kBlock) {
            const u32 at = (u32)a.l.tokens[i] - (u32)first;
            if (at >= (u32)left) continue;
            atomicOr(&words[at], kSeen);
            if (i >= prompt) atomicAdd(&words[at], 1u);
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < E; ++i) {
            const u32 w = words[V * (i / V * kBlock + tid) + i % V];
            if (w == 0) continue;
            const u32 n = w & ~kSeen;
            float z = y[i];
            z = z > 0.0f ? __fdiv_rn(z, repetition) : z * repetition;
            if (n) {
                const float by = frequency * (float)n;
                z = (z - by) - presence;
            }
            y[i] = z;
        }
        __syncthreads();
    }
    if (bias_end > bias_begin) {
        clear();
        for (int64_t i = bias_begin + tid; i < bias_end; i += kBlock) {
            const u32 at = (u32)a.l.bias_ids[i] - (u32)first;
            if (at < (u32)left) atomicMax(&words[at], (u32)(i - bias_begin) + 1);
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < E; ++i) {
            const u32 w = words[V * (i / V * kBlock + tid) + i % V];
            if (w) y[i] += a.l.bias[bias_begin + (w - 1)];
        }
    }
    float *out = a.out + row * a.out_row + first;
#pragma unroll
    for (int i = 0; i < E / V; ++i) {
        const int at = V * (i * kBlock + tid);
        if (at >= left) continue;
        // (V divides 32, so that a piece lies in one word)
        const u32 bits = allowed ? allowed[(u32)(first + at) >> 5] >> ((first + at) & 31) : ~0u;
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (!(bits >> j & 1)) y[i * V + j] = -__builtin_inff();
        if (at + V <= left) {
            out_t z;
#pragma unroll
            for (int j = 0; j < V; ++j) z[j] = y[i * V + j];
            *(out_t *)(out + at) = z;
        } else
            for (int j = 0; at + j < left; ++j) out[at + j] = y[i * V + j];
    }
}

}  // namespace
}  // namespace paged

extern "C" int serve_adjust(int32_t act, const void *logits, int64_t x_row, float *out, int64_t out_row,
                            int32_t n_rows, int32_t vocab, const serve_lists *lists, void *stream) {
    using namespace paged;
    if (act < PAGED_KV_BF16 || act > SERVE_F32 || n_rows < 0 || vocab < 1 || !lists) return PAGED_KV_EINVAL;
    if (n_rows == 0) return PAGED_KV_OK;
    const int size = act == SERVE_F32 ? 4 : 2;
    if (!logits || !out || (uintptr_t)logits % size || (uintptr_t)out % 4) return PAGED_KV_EINVAL;
    if ((const void *)out == logits && (act != SERVE_F32 || x_row != out_row)) return PAGED_KV_EINVAL;
    const serve_lists &l = *lists;
    if (l.tokens && !l.token_starts) return PAGED_KV_EINVAL;
    if (l.bias_ids && (!l.bias || !l.bias_starts)) return PAGED_KV_EINVAL;
    if (l.mask && (l.n_masks < 0 || l.mask_stride < ((int64_t)vocab + 31) / 32 || (!l.row_mask && l.n_masks < n_rows)))
        return PAGED_KV_EINVAL;
    if (n_rows > 65535 || vocab > 0x7FFFFFFF - 65536) return PAGED_KV_EUNSUPPORTED;
    if (device_cus() == 0) return PAGED_KV_EUNSUPPORTED;
    const AdjustArgs a = {logits, x_row, out, out_row, n_rows, vocab, l};
    // pieces of four elements where every row of both sides is aligned to them
    const bool wide = (uintptr_t)logits % (4 * size) == 0 && (uintptr_t)out % 16 == 0 && x_row % 4 == 0 && out_row % 4 == 0;
    // chunks of 16384 tokens, so that lists are read seldom; of 4096 where that leaves CUs without work
    const bool large = (int64_t)n_rows * ((vocab + 16383) / 16384) >= 512;
    const int chunk = large ? 16384 : 4096;
    const dim3 grid((unsigned)((vocab + chunk - 1) / chunk), (unsigned)n_rows);
    const auto go = [&](auto t) {
        typedef decltype(t) T;
        if (large)
            return wide ? launch(adjust_kernel<T, 4, 32>, grid, dim3(kBlock), stream, a)
                        : launch(adjust_kernel<T, 1, 32>, grid, dim3(kBlock), stream, a);
        return wide ? launch(adjust_kernel<T, 4, 8>, grid, dim3(kBlock), stream, a)
                    : launch(adjust_kernel<T, 1, 8>, grid, dim3(kBlock), stream, a);
    };
    return act == PAGED_KV_BF16 ? go(bf16()) : act == PAGED_KV_F16 ? go(f16()) : go(0.0f);
}
