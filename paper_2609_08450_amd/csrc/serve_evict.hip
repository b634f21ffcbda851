// What a cache keeps: the list of kept tokens, and the cache moved together.
//
// keep_kernel: a workgroup to a request marks its kept tokens as bits in LDS (a
// token that is named twice is one bit) and reads them off in order, by a prefix sum
// over words.  Weights move in place: the i-th kept token is not before place i, so
// rounds in rising order read nothing that an earlier one has written.  Bound by the chain of trips to memory
// and barriers: 5.8 us for 4 requests of up to 4096 tokens, 10 for 64 of up to 32768.
//
// compact_kernel: a workgroup to a request, head and side.  Its waves take the pages
// that follow each other, up to 8 KB of codes each in registers, all at once; after
// a barrier they write them.  What a round writes lies before everything that later
// rounds read, for the same reason, so the next round's loads are on their way
// meanwhile.  The codes read, in rows of head_dim bytes, and written bound it (64 requests of 2560 tokens, 2 heads
// of 128, e4m3: 31 us, 5.3 TB/s), with int8 beside vector work, 13 instructions a code (64 of 4096, 8 heads:
// 251 us, 4.2 TB/s; a 16-wave workgroup and few of them: trips to memory, 12 us).
#include "../../include/serve_step.h"
#include "paged_codes.h"

namespace paged {
namespace {

constexpr int kKeep = 1024;
constexpr int kWords = 16384;  // words of LDS: 2^19 tokens at a time
constexpr int kList = 4096;    // kept tokens that are written at a time

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
    __shared__ int list[kList];
    __shared__ int waves[kKeep / 64];
    const int tid = threadIdx.x, r = blockIdx.x;
    const int len = max(a.lens[r], 0);
    const int *idx = a.idx + (int64_t)r * a.K;
    int *kept = a.kept + (int64_t)r * a.width;
    float *weights = a.weights ? a.weights + a.weight_offsets[r] : nullptr;
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
        const int at = count + prefix(mine, waves, &all);
        // in order, by way of LDS
        for (int done = 0; done < all; done += kList) {
            int to_place = at - count - done;
            for (int i = from; i < to && to_place < kList; ++i)
                for (u32 w = words[i]; w; w &= w - 1, ++to_place)
                    if (to_place >= 0 && to_place < kList) list[to_place] = (int)(base + 32 * i + __builtin_ctz(w));
            __syncthreads();
            const int n = min(all - done, kList);
            float x[kList / kKeep];
#pragma unroll
            for (int j = 0; j < kList / kKeep; ++j) {
                const int i = j * kKeep + tid;
                if (i >= n) continue;
                kept[count + done + i] = list[i];
                if (weights) x[j] = weights[list[i]];
            }
            __syncthreads();
            if (weights)
#pragma unroll
                for (int j = 0; j < kList / kKeep; ++j) {
                    const int i = j * kKeep + tid;
                    if (i < n) weights[count + done + i] = x[j];
                }
        }
        count += all;
    }
    for (int i = count + tid; i < a.width; i += kKeep) kept[i] = -1;
    if (tid == 0) a.counts[r] = count;
    if (weights)
        for (int64_t i = (int64_t)count + tid; i < len; i += kKeep) weights[i] = 0.0f;
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
    // as the high bytes of 16 bits: what lies in the low ones decides between equal codes only
    i16x2 hi = {0, 0}, lo = {0, 0};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const u32 odd = x[i], even = odd << 8;  // (a bit cast of x[i] itself takes x[0])
        const i16x2 a = __builtin_bit_cast(i16x2, odd), b = __builtin_bit_cast(i16x2, even);
        hi = __builtin_elementwise_max(__builtin_elementwise_max(hi, a), b);
        lo = __builtin_elementwise_min(__builtin_elementwise_min(lo, a), b);
    }
    return (float)max(max((int)hi[0], (int)hi[1]) >> 8, -(min((int)lo[0], (int)lo[1]) >> 8));
}

// Codes of (code * old) / s, 16 at a time; no quotient is past the type's largest.  `ratio` is ratio_of(old, s).
template <class C>
__device__ float ratio_of(float old, float s);
template <class C>
__device__ u32x4 anew(u32x4 x, float old, float s, float ratio);
template <>
__device__ inline float ratio_of<E4M3>(float old, float s) {
    // s is a power of two, so that the factor is exact, and the product with it rounds as the
    // one with `old` does: once to FP32, once to a code.  (A factor this large is one of codes 0.)
    return fminf(old * __uint_as_float((254u << 23) - __float_as_uint(s)), 1e30f);
}
template <>
__device__ inline u32x4 anew<E4M3>(u32x4 x, float, float, float by) {
    u32x4 z;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)x[j], false);
        const f32x2 hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)x[j], true);
        const int c = __builtin_amdgcn_cvt_pk_fp8_f32(lo[0] * by, lo[1] * by, 0, false);
        z[j] = (u32)__builtin_amdgcn_cvt_pk_fp8_f32(hi[0] * by, hi[1] * by, c, true);
    }
    return z;
}
template <>
__device__ inline float ratio_of<Int8>(float old, float s) {
    return fminf(__fdiv_rn(old, s), 1e30f);  // (this large: codes are 0)
}
template <>
__device__ inline u32x4 anew<Int8>(u32x4 x, float old, float s, float ratio) {
    // The product with the rounded ratio is within 7.6e-6 of the quotient (2^-24 of 127), so it rounds to the
    // same unless it lies that near a half.  Added to 1.5 * 2^23 a product has its whole number in
    // the lowest byte.
    constexpr float kWhole = 12582912.0f;
    u32x4 z;
    float off = 0.0f;
    const auto packed = [](const u32 (&y)[4]) {
        return __builtin_amdgcn_perm(y[1], y[0], 0x0c0c0400u) | __builtin_amdgcn_perm(y[3], y[2], 0x04000c0cu);
    };
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        u32 y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float c = value_of<Int8>((x[j] >> (8 * i)) & 0xFFu), n = fmaf(c, ratio, kWhole);
            y[i] = __float_as_uint(n);
            off = fmaxf(off, fabsf(fmaf(c, ratio, kWhole - n)));
        }
        z[j] = packed(y);
    }
    if (!(off < 0.49999f)) {
        // code * old against h * s, h the half next to the product: its rounded product with s
        // taken from both, what is left of either is exact
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            u32 y[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float c = value_of<Int8>((x[j] >> (8 * i)) & 0xFFu);
                const float below = floorf(c * ratio), h = below + 0.5f, p = h * s;
                const float d = fmaf(c, old, -p) - fmaf(h, s, -p);
                const bool odd = (int)below & 1;
                y[i] = __float_as_uint(below + (d > 0.0f || (d == 0.0f && odd) ? 1.0f : 0.0f) + kWhole);
            }
            z[j] = packed(y);
        }
    }
    return z;
}

// The maxima of N values over the wave: that of value i in the lanes l with l / (64 / N) == i.
template <int N>
__device__ float tops_of(float (&t)[N]) {
    const int lane = threadIdx.x & 63;
    int d = 32;
#pragma unroll
    for (int n = N / 2; n; n /= 2, d /= 2)
#pragma unroll
        for (int i = 0; i < n; ++i) {
            const float keep = lane & d ? t[i + n] : t[i], send = lane & d ? t[i] : t[i + n];
            t[i] = fmaxf(keep, __shfl_xor(send, d));
        }
    for (; d; d /= 2) t[0] = fmaxf(t[0], __shfl_xor(t[0], d));
    return t[0];
}

// All waves are here, and what they wrote to LDS.  (Not __syncthreads(): that would wait for the
// loads that are on their way, too.)
__device__ inline void meet() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// WAVES of a workgroup hold PIECES of 1024 bytes of codes each, at least a page together.
template <class C, int D, int WAVES, int PIECES>
__global__ __launch_bounds__(64 * WAVES, 4) void compact_kernel(CompactArgs a) {
    constexpr int TOKENS = PIECES * 1024 / D;  // of a wave's part: each has a lane that knows where it lies
    static_assert(TOKENS <= 64, "a lane to a token");
    __shared__ float tops[2][PIECES * WAVES];
    __shared__ int first_moved;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int r = blockIdx.y, head = blockIdx.x / a.sides;
    uint8_t *codes = a.codes[blockIdx.x % a.sides];
    float *scales = a.scale[blockIdx.x % a.sides] + head;
    const int P = 1 << a.lp;
    const int64_t cap = (int64_t)a.table_width << a.lp;
    const int count = (int)min((int64_t)min(max(a.counts[r], 0), a.width), cap);
    const int *table = a.table + (int64_t)r * a.table_stride;
    const int *kept = a.kept + (int64_t)r * a.width;

    // the first page that changes: kept rises, so a page stays if its last token does
    const int pages = (count + P - 1) >> a.lp;
    int stay = pages;
    for (int p = tid; p < pages; p += 64 * WAVES) {
        const int last = min((int)min(((int64_t)p + 1) << a.lp, (int64_t)0x7FFFFFFF), count) - 1;
        if (kept[last] != last) {
            stay = p;
            break;
        }
    }
    if (tid == 0) first_moved = pages;
    __syncthreads();
    if (stay < pages) atomicMin(&first_moved, stay);
    __syncthreads();
    stay = first_moved;
    if (stay == pages) return;

    // A round: TOKENS of each wave.  Four of them are on their way at a time: the numbers of
    // kept tokens, pages, scales and codes each need those before.
    const int64_t begin = ((int64_t)stay << a.lp) + (int64_t)wave * TOKENS;
    constexpr int64_t ROUND = TOKENS * WAVES;
    const u32 head_row = (u32)(head << a.lp);
    int kk, pg = -1, pk = -1;  // kept token, and page with the token that it is of
    u32 from;
    float old, next_old;
    int to, next_to;  // lane i: the page that piece i goes to
    const auto numbers = [&](int64_t at) {
        kk = -1;
        if (lane < TOKENS && at + lane < count) kk = kept[at + lane];
    };
    const auto target = [&](int64_t at) {
        const int64_t t = at + lane * (1024 / D);
        next_to = -1;
        if (lane < PIECES && t < count) next_to = table[t >> a.lp];
    };
    const auto look_up = [&] {
        pk = kk;
        pg = -1;
        if (kk >= 0 && kk < cap) pg = table[kk >> a.lp];
    };
    const auto rows = [&] {
        from = kNone;
        next_old = 0.0f;
        if (pg >= 0 && pg < a.n_pages) {
            from = (u32)pg * a.page_rows + head_row + (u32)(pk & (P - 1));
            next_old = scales[pg * a.scale_stride];
        }
    };
    const auto fetch = [&](u32x4 (&x)[PIECES]) {
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const u32 row = __shfl(from, (1024 * i + 16 * lane) / D);  // (token of the part)
            x[i] = u32x4{0, 0, 0, 0};
            if (row != kNone) x[i] = *(const u32x4 *)(codes + (int64_t)row * D + (16 * lane) % D);
        }
    };
    u32x4 x[PIECES], next[PIECES];
    numbers(begin);
    look_up();
    numbers(begin + ROUND);
    rows();
    look_up();
    numbers(begin + 2 * ROUND);
    target(begin);
    fetch(next);
    int turn = 0;
    for (int64_t mine = begin; mine - (int64_t)wave * TOKENS < count; mine += ROUND, turn ^= 1) {
#pragma unroll
        for (int i = 0; i < PIECES; ++i) x[i] = next[i];
        old = next_old;
        to = next_to;
        rows();
        look_up();
        numbers(mine + 3 * ROUND);
        target(mine + ROUND);
        fetch(next);

        // the largest magnitude of every 1024 bytes
        const auto scale_at = [&](int i) { return __shfl(old, (1024 * i + 16 * lane) / D); };
        float top[PIECES];
#pragma unroll
        for (int i = 0; i < PIECES; ++i) top[i] = __fmul_rn(largest<C>(x[i]), scale_at(i));
        const float mine_top = tops_of(top);
        if (lane % (64 / PIECES) == 0) tops[turn][wave * PIECES + lane / (64 / PIECES)] = mine_top;
        // all of this round is read, and its maxima are there
        meet();
        const int group = (D << a.lp) / 1024;  // entries of `tops` to a page, a power of two
        float s = 0.0f, ratio = 0.0f;
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            if (i == 0 || group < PIECES) {  // (a larger page's are all the same)
                const int at = (wave * PIECES + i) & -group;
                float m = 0.0f;
                for (int j = 0; j < group; ++j) m = fmaxf(m, tops[turn][at + j]);
                s = scale_of<C>(m);
                ratio = ratio_of<C>(old, s);  // lane: of a token, as old
            }
            __builtin_amdgcn_sched_barrier(0);  // one after the other: registers
            // a piece lies in one page
            const int page = __builtin_amdgcn_readlane(to, i);
            const int64_t t = mine + 1024 * i / D;
            if (page < 0 || page >= a.n_pages) continue;
            // (codes under the scale that the page gets are what they are)
            const float was = scale_at(i), by = __shfl(ratio, (1024 * i + 16 * lane) / D);
            const u32x4 y = was == s ? x[i] : anew<C>(x[i], was, s, by);
            const u32 row = (u32)page * a.page_rows + head_row + (u32)(t & (P - 1));
            if (t + 16 * lane / D < count) __builtin_nontemporal_store(y, (u32x4 *)(codes + (int64_t)row * D + 16 * lane));
            if ((t & (P - 1)) == 0 && lane == 0) scales[page * a.scale_stride] = s;
        }
    }
}

template <class C, int D>
int launch_compact(const CompactArgs &a, int n_requests, void *stream) {
    const dim3 grid((unsigned)(a.n_heads * a.sides), (unsigned)n_requests);
    // 16 waves where workgroups are few, so that one has more on its way (with keep: four requests of 604
    // tokens 17.0 us, and 20.8 with 8 waves); 8 where there are more than the card holds at a time,
    // so that one computes while another waits (1024 of 4096 tokens 255 us, and 277 with 16)
    const bool small = (int64_t)grid.x * n_requests >= 512 && (D << a.lp) <= 32768;
    return small ? launch(compact_kernel<C, D, 8, 4>, grid, dim3(512), stream, a)
                 : launch(compact_kernel<C, D, 16, 4>, grid, dim3(1024), stream, a);
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
    if ((K > 0 && !idx) || !lens || (width > 0 && !kept) || !counts || (weights && !weight_offsets) || lens == counts ||
        (K > 0 && idx == kept))
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
