// What a cache keeps: the list of kept tokens, and the cache moved together.
//
// keep_kernel: a workgroup to a request marks its kept tokens as bits in LDS (a
// token that is named twice is one bit) and reads them off in order, by a prefix sum
// over words.  Weights move in place: the i-th kept token is not before place i, so
// rounds in rising order read nothing that an earlier one has written.
//
// compact_kernel: a workgroup to a request, head and side.  Its waves take the pages
// that follow each other, up to 8 KB of codes each in registers, all at once; after
// a barrier they write them.  What a round writes lies before everything that later
// rounds read, for the same reason, so the next round's loads are on their way
// meanwhile.  Bound by memory: the codes read, in rows of head_dim bytes, and written.
#include "../../include/serve_step.h"
#include "paged_codes.h"

namespace paged {
namespace {

constexpr int kKeep = 1024;
constexpr int kWords = 16384;  // words of LDS: 2^19 tokens at a time

struct KeepArgs {
    const int *idx;
    int K, base;
    const int *lens;
    int first, last;
    int *kept;
    int width;
    int *counts;
    float *weights;
    const int64_t *weight_offsets;
};

// Exclusive prefix of x over the workgroup; total in *sum.
__device__ int prefix(int x, int *waves, int *sum) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    int s = x;
    for (int d = 1; d < 64; d <<= 1) {
        const int y = __shfl_up(s, d);
        if (lane >= d) s += y;
    }
    __syncthreads();
    if (lane == 63) waves[w] = s;
    __syncthreads();
    int before = 0, all = 0;
    for (int i = 0; i < kKeep / 64; ++i) {
        if (i == w) before = all;
        all += waves[i];
    }
    *sum = all;
    return before + s - x;
}

// The bits of a word whose 32 numbers start at `at` that lie in [from, to).
__device__ u32 bits_of(int64_t at, int64_t from, int64_t to) {
    const int64_t a = max(from - at, (int64_t)0), b = min(to - at, (int64_t)32);
    if (a >= b) return 0;
    return (u32)(((1ull << b) - 1) & ~((1ull << a) - 1));
}

__global__ __launch_bounds__(kKeep) void keep_kernel(KeepArgs a) {
    __shared__ u32 words[kWords];
    __shared__ int waves[kKeep / 64];
    const int tid = threadIdx.x, r = blockIdx.x;
    const int len = max(a.lens[r], 0);
    const int *idx = a.idx + (int64_t)r * a.K;
    int *kept = a.kept + (int64_t)r * a.width;
    int count = 0;
    for (int64_t base = 0; base < len; base += 32 * (int64_t)kWords) {
        const int tokens = (int)min((int64_t)len - base, 32 * (int64_t)kWords), n = (tokens + 31) / 32;
        for (int i = tid; i < n; i += kKeep)
            words[i] = bits_of(base + 32 * i, 0, min(a.first, len)) |
                       bits_of(base + 32 * i, max((int64_t)len - a.last, (int64_t)0), len);
        __syncthreads();
        for (int i = tid; i < a.K; i += kKeep) {
            const int j = idx[i];
            const int64_t t = (int64_t)j + a.base - base;
            if (j >= 0 && t >= 0 && t < tokens) atomicOr(&words[t >> 5], 1u << (t & 31));
        }
        __syncthreads();
        // neighbouring words to a thread
        const int per = (n + kKeep - 1) / kKeep, from = min(tid * per, n), to = min(from + per, n);
        int mine = 0, all;
        for (int i = from; i < to; ++i) mine += __popc(words[i]);
        int at = count + prefix(mine, waves, &all);
        for (int i = from; i < to; ++i)
            for (u32 w = words[i]; w; w &= w - 1) kept[at++] = (int)(base + 32 * i + __builtin_ctz(w));
        count += all;
        __syncthreads();
    }
    for (int i = count + tid; i < a.width; i += kKeep) kept[i] = -1;
    if (tid == 0) a.counts[r] = count;
    if (!a.weights) return;
    float *w = a.weights + a.weight_offsets[r];
    for (int i0 = 0; i0 < count; i0 += 4 * kKeep) {
        float x[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int i = i0 + j * kKeep + tid;
            if (i < count) x[j] = w[kept[i]];
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int i = i0 + j * kKeep + tid;
            if (i < count) w[i] = x[j];
        }
        __syncthreads();
    }
    for (int64_t i = (int64_t)count + tid; i < len; i += kKeep) w[i] = 0.0f;
}

struct CompactArgs {
    uint8_t *codes[2];
    float *scale[2];
    int64_t scale_stride;
    u32 page_rows;  // rows of head_dim codes from one page to the next
    int n_pages, lp, n_heads, sides;
    const int *table;
    int table_stride, table_width;
    const int *kept;
    int width;
    const int *counts;
};

constexpr int kPart = 8192;  // bytes of codes that a wave holds
constexpr u32 kNone = 0xFFFFFFFFu;

typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef int16_t i16x2 __attribute__((ext_vector_type(2)));

// The largest magnitude among 16 codes.
template <class C>
__device__ float largest(u32x4 x);
template <>
__device__ inline float largest<E4M3>(u32x4 x) {
    // without their signs codes rise with their values
    u16x2 m = {0, 0};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, x[i] & 0x007F007Fu));
        m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, (x[i] >> 8) & 0x007F007Fu));
    }
    return value_of<E4M3>(min((u32)max(m[0], m[1]), 0x7Eu));
}
template <>
__device__ inline float largest<Int8>(u32x4 x) {
    // as the high bytes of 16 bits; what lies in the low ones does not reach the next code
    i16x2 hi = {0, 0}, lo = {0, 0};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const i16x2 a = __builtin_bit_cast(i16x2, x[i] & 0xFF00FF00u);
        const i16x2 b = __builtin_bit_cast(i16x2, (x[i] << 8) & 0xFF00FF00u);
        hi = __builtin_elementwise_max(__builtin_elementwise_max(hi, a), b);
        lo = __builtin_elementwise_min(__builtin_elementwise_min(lo, a), b);
    }
    return (float)(max(max((int)hi[0], (int)hi[1]), -min((int)lo[0], (int)lo[1])) >> 8);
}

// Codes of (code * old) / s, 16 at a time; ratio is old / s.
template <class C>
__device__ u32x4 anew(u32x4 x, float old, float s, float ratio);
template <>
__device__ inline u32x4 anew<E4M3>(u32x4 x, float old, float s, float) {
    // the product with a power of two is exact: one rounding to FP32, one to a code
    const float r = __uint_as_float((254u << 23) - __float_as_uint(s));
    u32x4 z;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            y[i] = __fmul_rn(value_of<E4M3>((x[j] >> (8 * i)) & 0xFFu), old);
            y[i] = __builtin_amdgcn_fmed3f(y[i] * r, -448.0f, 448.0f);
        }
        const int c = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
        z[j] = (u32)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], c, true);
    }
    return z;
}
template <>
__device__ inline u32x4 anew<Int8>(u32x4 x, float old, float s, float ratio) {
    // The product with the rounded ratio is within 128 * 2^-23 of the quotient, so it
    // rounds to the same unless it lies that near a half: then the wave divides, in 64
    // bits.  Added to 1.5 * 2^23 a product has its whole number in the lowest byte.
    constexpr float kWhole = 12582912.0f;
    u32x4 z;
    float off = 0.0f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        u32 y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float q = __builtin_amdgcn_fmed3f(value_of<Int8>((x[j] >> (8 * i)) & 0xFFu) * ratio, -127.0f, 127.0f);
            const float n = q + kWhole;
            y[i] = __float_as_uint(n);
            off = fmaxf(off, fabsf(q - (n - kWhole)));
        }
        const u32 lo = __builtin_amdgcn_perm(y[1], y[0], 0x0c0c0400u), hi = __builtin_amdgcn_perm(y[3], y[2], 0x04000c0cu);
        z[j] = lo | hi;
    }
    if (!(off < 0.4999f)) {
        u32 w[4] = {x[0], x[1], x[2], x[3]};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            u32 all = 0;
#pragma unroll 1
            for (int i = 0; i < 32; i += 8) {
                const double q = rint((double)(signed char)(w[j] >> i) * (double)old / (double)s);
                all |= ((u32)(int)fmin(fmax(q, -127.0), 127.0) & 0xFFu) << i;
            }
            z[j] = all;
        }
    }
    return z;
}

// The maxima of eight values over the wave: that of value i in the lanes l with l / 8 == i.
__device__ inline float eight_tops(const float (&t)[8]) {
    const int lane = threadIdx.x & 63;
    float u[4], v[2];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float keep = lane & 32 ? t[i + 4] : t[i], send = lane & 32 ? t[i] : t[i + 4];
        u[i] = fmaxf(keep, __shfl_xor(send, 32));
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const float keep = lane & 16 ? u[i + 2] : u[i], send = lane & 16 ? u[i] : u[i + 2];
        v[i] = fmaxf(keep, __shfl_xor(send, 16));
    }
    const float keep = lane & 8 ? v[1] : v[0], send = lane & 8 ? v[0] : v[1];
    float w = fmaxf(keep, __shfl_xor(send, 8));
#pragma unroll
    for (int d = 4; d; d >>= 1) w = fmaxf(w, __shfl_xor(w, d));
    return w;
}

template <class C, int D, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void compact_kernel(CompactArgs a) {
    constexpr int TOKENS = kPart / D;     // of a wave's part
    constexpr int SLOTS = (TOKENS + 63) / 64;
    constexpr int PIECES = kPart / 1024;  // of 16 bytes, of a lane
    __shared__ float tops[2][PIECES * WAVES];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int r = blockIdx.y, head = blockIdx.x / a.sides;
    uint8_t *codes = a.codes[blockIdx.x % a.sides];
    float *scales = a.scale[blockIdx.x % a.sides] + head;
    const int P = 1 << a.lp;
    const int64_t cap = (int64_t)a.table_width << a.lp;
    const int count = (int)min((int64_t)min(max(a.counts[r], 0), a.width), cap);
    const int *table = a.table + (int64_t)r * a.table_stride;
    const int *kept = a.kept + (int64_t)r * a.width;
    const auto page_of = [&](int i) {
        const int p = table[i];
        return p >= 0 && p < a.n_pages ? p : -1;
    };

    // the first page that changes: kept rises, so whole pages before a token that moves
    // stay if their last token does
    int stay = 0;
    {
        int lo = 0, hi = count;  // kept[i] == i for i < lo
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (kept[mid] == mid) lo = mid + 1;
            else hi = mid;
        }
        if (lo == count) return;
        stay = lo >> a.lp;
    }
    // a round: TOKENS of each wave, from a multiple of the page's on
    const int round = TOKENS * WAVES;
    int turn = 0;
    for (int64_t base = (int64_t)stay << a.lp; base < count; base += round, turn ^= 1) {
        const int64_t mine = base + (int64_t)wave * TOKENS;
        // this lane's tokens: the row of codes that each comes from, its scale
        u32 from[SLOTS];
        float old[SLOTS];
#pragma unroll
        for (int i = 0; i < SLOTS; ++i) {
            const int64_t t = mine + 64 * i + lane;
            from[i] = kNone;
            old[i] = 0.0f;
            if (lane < TOKENS && t < count) {
                const int k = kept[t];
                if (k < 0 || k >= cap) continue;
                const int p = page_of(k >> a.lp);
                if (p < 0) continue;
                from[i] = (u32)p * a.page_rows + (u32)(head << a.lp) + (u32)(k & (P - 1));
                old[i] = scales[p * a.scale_stride];
            }
        }
        u32x4 x[PIECES];
        float scale[PIECES];
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int t = (1024 * i + 16 * lane) / D;  // token of the part
            const u32 row = __shfl(from[SLOTS == 1 ? 0 : t >> 6], t & 63);
            scale[i] = __shfl(old[SLOTS == 1 ? 0 : t >> 6], t & 63);
            x[i] = u32x4{0, 0, 0, 0};
            if (row != kNone) x[i] = *(const u32x4 *)(codes + (int64_t)row * D + (16 * lane) % D);
        }
        // the largest magnitude of every 1024 bytes
        float top[PIECES];
#pragma unroll
        for (int i = 0; i < PIECES; ++i) top[i] = __fmul_rn(largest<C>(x[i]), scale[i]);
        const float mine_top = eight_tops(top);
        if (lane % 8 == 0) tops[turn][wave * PIECES + lane / 8] = mine_top;
        // all of this round is read, and its maxima are there
        __syncthreads();
        const int group = (D << a.lp) / 1024;  // entries of `tops` to a page
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int at = (wave * PIECES + i) / group * group;
            float m = 0.0f;
            for (int j = 0; j < group; ++j) m = fmaxf(m, tops[turn][at + j]);
            const float s = scale_of<C>(m);
            const int64_t t = mine + (1024 * i + 16 * lane) / D;
            const int page = t < count ? page_of((int)(t >> a.lp)) : -1;
            if (page < 0) continue;
            const float ratio = __fdiv_rn(scale[i], s);
            const u32x4 y = anew<C>(x[i], scale[i], s, ratio);
            const u32 row = (u32)page * a.page_rows + (u32)(head << a.lp) + (u32)(t & (P - 1));
            *(u32x4 *)(codes + (int64_t)row * D + (16 * lane) % D) = y;
            if ((t & (P - 1)) == 0 && (16 * lane) % D == 0) scales[page * a.scale_stride] = s;
        }
    }
}

template <class C, int D>
int launch_compact(const CompactArgs &a, int n_requests, void *stream) {
    const dim3 grid((unsigned)(a.n_heads * a.sides), (unsigned)n_requests);
    return launch(compact_kernel<C, D, 8>, grid, dim3(512), stream, a);
}

}  // namespace
}  // namespace paged

extern "C" int serve_keep(const int32_t *idx, int32_t K, int32_t base, const int32_t *lens, int32_t n_requests,
                          int32_t first, int32_t last, int32_t *kept, int32_t width, int32_t *counts,
                          float *weights, const int64_t *weight_offsets, void *stream) {
    using namespace paged;
    if (K < 0 || base < 0 || n_requests < 0 || first < 0 || last < 0 || width < (int64_t)first + K + last)
        return PAGED_KV_EINVAL;
    if (n_requests == 0) return PAGED_KV_OK;
    if ((K > 0 && !idx) || !lens || (width > 0 && !kept) || !counts || (weights && !weight_offsets) || lens == counts)
        return PAGED_KV_EINVAL;
    if (device_cus() == 0) return PAGED_KV_EUNSUPPORTED;
    const KeepArgs a = {idx, K, base, lens, first, last, kept, width, counts, weights, weight_offsets};
    return launch(keep_kernel, dim3((unsigned)n_requests), dim3(kKeep), stream, a);
}

extern "C" int serve_compact(const paged_kv_cache *cache, const int32_t *table, int32_t table_stride,
                             int32_t table_width, const int32_t *kept, int32_t width, const int32_t *counts,
                             int32_t n_requests, void *stream) {
    using namespace paged;
    const int rc = check_cache(cache, cache && cache->v);
    if (rc != PAGED_KV_OK) return rc;
    if (n_requests < 0 || table_width < 1 || table_stride < table_width || width < 0) return PAGED_KV_EINVAL;
    if (n_requests == 0 || width == 0) return PAGED_KV_OK;
    if (!table || !kept || !counts) return PAGED_KV_EINVAL;
    if (n_requests > 65535 || cache->n_heads > 1 << 20) return PAGED_KV_EUNSUPPORTED;
    const int lp = log2_page(cache->page);
    if (((int64_t)table_width << lp) > 0x7FFFFFFF) return PAGED_KV_EUNSUPPORTED;
    if (device_cus() == 0) return PAGED_KV_EUNSUPPORTED;
    const CompactArgs a = {{(uint8_t *)cache->k, (uint8_t *)cache->v}, {cache->k_scale, cache->v_scale},
                           cache->scale_stride, (u32)(cache->page_stride / cache->head_dim), cache->n_pages, lp,
                           cache->n_heads, cache->v ? 2 : 1, table, table_stride, table_width, kept, width, counts};
    const auto go = [&](auto c) {
        typedef decltype(c) C;
        return cache->head_dim == 64    ? launch_compact<C, 64>(a, n_requests, stream)
               : cache->head_dim == 128 ? launch_compact<C, 128>(a, n_requests, stream)
                                        : launch_compact<C, 256>(a, n_requests, stream);
    };
    return cache->code == PAGED_KV_E4M3 ? go(E4M3()) : go(Int8());
}
