// Penalties, biases and masks on logits.
//
// A workgroup takes a chunk of one row's vocabulary into registers.  How often the
// row's tokens fall into the chunk is counted in LDS, a word to a token (whole
// numbers: their order does not matter); biased tokens get a bit there and an
// entry in one of some chains, by place.  Then every element reads its word, and goes through its
// chain if it has the bit (212 biases of a row of 5099: 5.4 us, and 24 with one list of them).
// Where a chunk has more biases than entries, a second pass adds them: the words then hold the greatest number
// of an entry that names the token.  Every workgroup of a row reads the row's whole lists, out of the L2.
// Bound by memory: a logit read and an FP32 number written (256 rows of 131072, lists of 8192 tokens and 100
// biases: 42.5 us, 4.85 TB/s; 4 rows of 32003: 4.6 us, of trips to memory).
#include "../../include/serve_step.h"
#include "paged_common.h"

// every step of the definition is rounded: no product and sum become one operation
#pragma clang fp contract(off)

namespace paged {
namespace {

constexpr int kBlock = 512;
constexpr u32 kSeen = 0x80000000u;    // of a word: the token is among the prompt's
constexpr u32 kBiased = 0x40000000u;  // it has a bias; below: how often it is behind the prompt
constexpr int kListed = 256;          // biases of a chunk that are listed in LDS (more would cost a workgroup of a CU)
constexpr u32 kChains = 128;
constexpr int kAhead = 8;             // tokens of a thread that are on their way at once

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

struct Bias {
    u32 at, entry;  // place in the chunk, and in the row's list
    float value;
    u32 next;       // of its chain; kListed: none
};

// V: elements that lie together in x and in out, both aligned; E: of a thread.
template <class T, int V, int E>
__global__ __launch_bounds__(kBlock) void adjust_kernel(AdjustArgs a) {
    typedef Logits<T, V> L;
    typedef float out_t __attribute__((ext_vector_type(V)));
    constexpr int CHUNK = kBlock * E;
    __shared__ alignas(16) u32 words[CHUNK];
    __shared__ Bias listed[kListed];
    __shared__ u32 biased, chains[kChains];
    const int tid = threadIdx.x;
    // the chunks of a row on one XCD (workgroups go round them), whose L2 then holds its lists
    const int chunks = gridDim.x, b = blockIdx.y * chunks + blockIdx.x, whole = a.n_rows & ~7;
    const bool round = b < whole * chunks;
    const int row = round ? b / (8 * chunks) * 8 + b % 8 : blockIdx.y, chunk = round ? b / 8 % chunks : blockIdx.x;
    const int first = chunk * CHUNK, left = min(CHUNK, a.vocab - first);
    const T *x = (const T *)a.x + row * a.x_row + first;
    // what the row's lists and mask are
    int64_t begin = 0, end = 0, prompt = 0, bias_begin = 0, bias_end = 0;
    float repetition = 1.0f, frequency = 0.0f, presence = 0.0f;
    if (a.l.tokens) {
        begin = a.l.token_starts[row];
        end = a.l.token_starts[row + 1];
        prompt = begin + (a.l.prompt_lens ? max(a.l.prompt_lens[row], 0) : 0);
        if (a.l.repetition) repetition = a.l.repetition[row];
        if (a.l.frequency) frequency = a.l.frequency[row];
        if (a.l.presence) presence = a.l.presence[row];
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
    // piece i of the thread: elements V (i kBlock + tid) on; V divides 32, so that a piece lies in one word of the mask
    typename L::type raw[E / V];
    u32 bits[E / V];
#pragma unroll
    for (int i = 0; i < E / V; ++i) {
        const int at = V * (i * kBlock + tid);
        bits[i] = allowed && at < left ? allowed[(u32)(first + at) >> 5] >> ((first + at) & 31) : ~0u;
        if (at + V <= left) raw[i] = *(const typename L::type *)(x + at);
        else
            for (int j = 0; j < V; ++j) {
                const T one = at + j < left ? x[at + j] : (T)0.0f;
                if constexpr (V == 1) raw[i] = one;
                else raw[i][j] = one;
            }
    }
    const bool lists = end > begin || bias_end > bias_begin;
    if (lists) {
        for (int i = 4 * tid; i < CHUNK; i += 4 * kBlock) *(u32x4 *)&words[i] = u32x4{0, 0, 0, 0};
        if (tid == 0) biased = 0;
        if (tid < (int)kChains) chains[tid] = kListed;
        __syncthreads();
        // (several tokens of a thread at once: one after the other each would cost a trip to memory)
        for (int64_t i0 = begin + tid; i0 < end; i0 += kAhead * kBlock) {
            int token[kAhead];
#pragma unroll
            for (int j = 0; j < kAhead; ++j) token[j] = a.l.tokens[min(i0 + j * kBlock, end - 1)];
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                const int64_t i = i0 + j * kBlock;
                const u32 at = (u32)token[j] - (u32)first;
                if (i >= end || at >= (u32)left) continue;
                if (i < prompt) atomicOr(&words[at], kSeen);
                else atomicAdd(&words[at], 1u);
            }
        }
        for (int64_t i = bias_begin + tid; i < bias_end; i += kBlock) {
            const u32 at = (u32)a.l.bias_ids[i] - (u32)first;
            if (at >= (u32)left) continue;
            atomicOr(&words[at], kBiased);
            const u32 place = atomicAdd(&biased, 1u);
            if (place < kListed)
                listed[place] = {at, (u32)(i - bias_begin), a.l.bias[i], atomicExch(&chains[at % kChains], place)};
        }
        __syncthreads();
    }
    const bool more = lists && biased > kListed;
    // the last entry of the list that names this place
    const auto bias_of = [&](u32 at) {
        int last = -1;
        float value = 0.0f;
        for (u32 i = chains[at % kChains]; i < kListed; i = listed[i].next)
            if (listed[i].at == at && (int)listed[i].entry > last) {
                last = (int)listed[i].entry;
                value = listed[i].value;
            }
        return value;
    };
    float *out = a.out + row * a.out_row + first;
#pragma unroll
    for (int i = 0; i < E / V; ++i) {
        const int at = V * (i * kBlock + tid);
        if (at >= left) continue;
        float y[V];
        u32 w[V];
#pragma unroll
        for (int j = 0; j < V; ++j) {
            y[j] = L::at(raw[i], j);
            w[j] = lists ? words[at + j] : 0;
        }
#pragma unroll
        for (int j = 0; j < V; ++j) {
            float z = y[j];
            if (w[j]) {
                if (w[j] & ~kBiased) z = z > 0.0f ? __fdiv_rn(z, repetition) : z * repetition;
                const u32 n = w[j] & ~(kSeen | kBiased);
                if (n) {
                    const float by = frequency * (float)n;
                    z = (z - by) - presence;
                }
                if (w[j] & kBiased && !more) z += bias_of((u32)(at + j));
            }
            y[j] = bits[i] >> j & 1 ? z : -__builtin_inff();
        }
        if (at + V <= left) {
            out_t z;
#pragma unroll
            for (int j = 0; j < V; ++j) z[j] = y[j];
            // past the caches where a call's rows are more than they hold (256 rows of 131072 with all lists: 43 us,
            // and 61 with stores that stay in them; without lists and with a Top-K behind it 64.3 and 65.9, but 27.4
            // and 25.4 for 64 rows, which the last-level cache holds)
            if constexpr (E == 16) __builtin_nontemporal_store(z, (out_t *)(out + at));
            else *(out_t *)(out + at) = z;
        } else
            for (int j = 0; at + j < left; ++j) out[at + j] = y[j];
    }
    if (!more) return;
    __syncthreads();
    for (int i = tid; i < CHUNK; i += kBlock) words[i] = 0;
    __syncthreads();
    for (int64_t i = bias_begin + tid; i < bias_end; i += kBlock) {
        const u32 at = (u32)a.l.bias_ids[i] - (u32)first;
        if (at < (u32)left) atomicMax(&words[at], (u32)(i - bias_begin) + 1);
    }
    __syncthreads();
    // (a thread's own elements: nobody else reads or writes them)
    for (int i = 0; i < E / V; ++i)
        for (int j = 0; j < V; ++j) {
            const int at = V * (i * kBlock + tid) + j;
            if (at >= left || words[at] == 0) continue;
            const int t = first + at;
            if (allowed && !(allowed[(u32)t >> 5] >> (t & 31) & 1)) continue;
            out[at] += a.l.bias[bias_begin + words[at] - 1];
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
    if (n_rows > 1 && out_row < vocab) return PAGED_KV_EINVAL;
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
    // chunks of 8192 tokens, so that lists are read seldom; of 2048 where that leaves CUs without work
    const bool large = (int64_t)n_rows * ((vocab + 8191) / 8192) >= 512;
    const int chunk = large ? 8192 : 2048;
    const dim3 grid((unsigned)((vocab + chunk - 1) / chunk), (unsigned)n_rows);
    const auto go = [&](auto t) {
        typedef decltype(t) T;
        if (large)
            return wide ? launch(adjust_kernel<T, 4, 16>, grid, dim3(kBlock), stream, a)
                        : launch(adjust_kernel<T, 1, 16>, grid, dim3(kBlock), stream, a);
        return wide ? launch(adjust_kernel<T, 4, 4>, grid, dim3(kBlock), stream, a)
                    : launch(adjust_kernel<T, 1, 4>, grid, dim3(kBlock), stream, a);
    };
    return act == PAGED_KV_BF16 ? go(bf16()) : act == PAGED_KV_F16 ? go(f16()) : go(0.0f);
}
