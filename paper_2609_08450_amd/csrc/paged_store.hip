// New keys and values into the cache's pages, in 8 bits.
//
// A run is the rows of one page (they follow each other, at consecutive places).
// One wave takes a run of one head and side at a time: its rows into registers,
// their largest magnitude, the page's scale, then the codes; no wave waits for
// another.  Bound by memory (3 bytes an element) and by vector work (24 instructions
// an element, 10 us of a SIMD's time in the first case below) where the rows are
// many, by the chain slots - rows - codes where they are few.  8192 rows of 8 heads
// of 128, K and V, int8: 15.7 us, 3.2 TB/s; 64 single rows: 7.6 us.
#include "paged_codes.h"

namespace paged {
namespace {

constexpr int kWindow = 64;  // rows whose slots a wave looks through for runs
constexpr int kHeld = 8;     // pieces of eight elements that a lane holds; longer runs are read twice

struct Side {
    uint8_t *codes;
    float *scale;
    const void *x;
    int64_t row, head;
};

struct StoreArgs {
    Side side[2];
    int sides;
    const int64_t *slots;
    int64_t n_slots;  // slots of the cache
    int64_t page_stride, scale_stride;
    int n_rows, lp, dim, splits;
};

// Codes of x / s, eight at a time, x finite or not.
template <class C>
__device__ u32x2 codes_of(const float (&x)[8], float s);
template <>
__device__ u32x2 codes_of<E4M3>(const float (&x)[8], float s) {
    // A scale of this call's is a power of two: products with 1 / s are exact.  A
    // page's earlier one may be any.
    const float r = __fdiv_rn(1.0f, s);
    const bool exact = (__builtin_amdgcn_readfirstlane(__float_as_uint(s)) & 0x7FFFFFu) == 0;
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        y[i] = fminf(fmaxf(exact ? x[i] * r : __fdiv_rn(x[i], s), -448.0f), 448.0f);
        y[i] = x[i] != x[i] ? 0.0f : y[i];
    }
    u32x2 z;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        int c = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * h], y[4 * h + 1], 0, false);
        z[h] = (u32)__builtin_amdgcn_cvt_pk_fp8_f32(y[4 * h + 2], y[4 * h + 3], c, true);
    }
    return z;
}
template <>
__device__ u32x2 codes_of<Int8>(const float (&x)[8], float s) {
    // The quotient rounded to FP32, then to a whole number.  A product with 1 / s is
    // within 3e-5 of the quotient, so it rounds to the same unless it lies within
    // 1e-4 of a half; then, and where an entry is not finite, all of the wave divide.
    // Added to 1.5 * 2^23 the product has its whole number in the lowest byte.
    constexpr float kWhole = 12582912.0f;
    const float r = __fdiv_rn(1.0f, s);
    u32 y[8];
    float off = 0.0f, odd = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float q = __builtin_amdgcn_fmed3f(x[i] * r, -127.0f, 127.0f), z = q + kWhole;
        y[i] = __float_as_uint(z);
        off = fmaxf(off, fabsf(q - (z - kWhole)));
        odd = fmaf(x[i], 0.0f, odd);  // 0, or NaN
    }
    if (__any(!(off < 0.4999f) || odd != 0.0f))
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float q = fminf(fmaxf(rintf(__fdiv_rn(x[i], s)), -127.0f), 127.0f);
            y[i] = __float_as_uint((x[i] != x[i] ? 0.0f : q) + kWhole);
        }
    u32x2 z;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const u32 lo = __builtin_amdgcn_perm(y[4 * h + 1], y[4 * h], 0x0c0c0400u);
        const u32 hi = __builtin_amdgcn_perm(y[4 * h + 3], y[4 * h + 2], 0x04000c0cu);
        z[h] = lo | hi;
    }
    return z;
}

template <class T>
__device__ void elements(u32x4 v, float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const u32 w = v[i >> 1];
        if constexpr (__is_same(T, bf16)) x[i] = __uint_as_float((i & 1) ? w & 0xFFFF0000u : w << 16);
        else x[i] = (float)__builtin_bit_cast(f16x2, w)[i & 1];
    }
}

// The largest magnitude, infinite where one is (NaN is passed over).
template <class T>
__device__ float largest(u32x4 v, float top) {
    float x[8];
    elements<T>(v, x);
#pragma unroll
    for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(x[i]));
    return top;
}
// The same of the finite ones alone.
template <class T>
__device__ float largest_finite(u32x4 v, float top) {
    float x[8];
    elements<T>(v, x);
#pragma unroll
    for (int i = 0; i < 8; ++i) top = fabsf(x[i]) < __builtin_inff() ? fmaxf(top, fabsf(x[i])) : top;
    return top;
}

template <class T, class C>
__global__ __launch_bounds__(64) void store_kernel(StoreArgs a) {
    const int lane = threadIdx.x;
    const int first = blockIdx.x * kWindow, head = blockIdx.y / a.sides;
    const Side o = a.side[blockIdx.y % a.sides];
    const int P = 1 << a.lp;
    const auto slot_at = [&](int i) { return i >= 0 && i < a.n_rows ? a.slots[i] : (int64_t)-1; };
    const auto page_at = [&](int64_t s) { return s >= 0 && s < a.n_slots ? s >> a.lp : (int64_t)-1; };

    // the rows of this window that begin a run, and those that go on with one
    const int64_t mine = slot_at(first + lane), outside = slot_at(first - 1);
    int64_t before = __shfl_up(mine, 1);
    if (lane == 0) before = outside;
    const bool in = page_at(mine) >= 0, on = in && page_at(before) == page_at(mine) && before + 1 == mine;
    uint64_t begins = __ballot(in && !on);
    const uint64_t goes_on = __ballot(on);
    for (int k = 0; begins; ++k) {
        const int at = __builtin_ctzll(begins);
        begins &= begins - 1;
        if (k % a.splits != (int)blockIdx.z) continue;
        const int row = first + at;
        const int64_t slot = __shfl(mine, at), page = slot >> a.lp;
        const int place = (int)(slot & (P - 1));
        // its length: to the window's end, and past it up to the page's
        int count = 1 + (at == 63 ? 0 : __builtin_ctzll(~(goes_on >> (at + 1))));
        if (at + count == 64)
            for (bool more = true; more && count < P - place;) {
                const int j = count + lane;
                const uint64_t m = __ballot(j < P - place && slot_at(row + j) == slot + j);
                more = m == ~0ull;
                count += more ? 64 : __builtin_ctzll(~m);
            }
        const int per = a.dim / 8, units = count * per;  // pieces of eight elements
        const bool held = units <= 64 * kHeld;
        float *where = o.scale + page * a.scale_stride + head;
        const float old = *where;
        uint8_t *codes = o.codes + page * a.page_stride + (int64_t)head * P * a.dim;
        const char *x = (const char *)o.x + 2 * (row * o.row + head * o.head);
        const auto piece = [&](int u) {
            const int j = u / per;
            return *(const u32x4 *)(x + 2 * (j * o.row + (u - j * per) * 8));
        };
        u32x4 v[kHeld];
        float top = 0.0f;
        if (held) {
#pragma unroll
            for (int i = 0; i < kHeld; ++i)
                if (64 * i < units) v[i] = piece(min(64 * i + lane, units - 1));
#pragma unroll
            for (int i = 0; i < kHeld; ++i)
                if (64 * i < units) top = largest<T>(v[i], top);
        } else {
            for (int u = lane; u < units; u += 64) top = largest<T>(piece(u), top);
        }
        if (__any(top == __builtin_inff())) {
            top = 0.0f;
            for (int u = lane; u < units; u += 64) top = largest_finite<T>(piece(u), top);
        }
        for (int d = 32; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
        const float fresh = scale_of<C>(top), s = place > 0 ? fmaxf(old, fresh) : fresh;
        if (place > 0 && s > old)
            // codes under a smaller scale: (code * old) / s, rounded anew
            for (int u = lane; u < place * per; u += 64) {
                const u32x2 w = ((const u32x2 *)codes)[u];
                float y[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) y[i] = __fmul_rn(value_of<C>((w[i >> 2] >> (8 * (i & 3))) & 0xFFu), old);
                ((u32x2 *)codes)[u] = codes_of<C>(y, s);
            }
        u32x2 *to = (u32x2 *)(codes + (int64_t)place * a.dim);
        float y[8];
        if (held) {
#pragma unroll
            for (int i = 0; i < kHeld; ++i)
                if (64 * i < units) {
                    elements<T>(v[i], y);
                    const u32x2 z = codes_of<C>(y, s);
                    if (64 * i + lane < units) to[64 * i + lane] = z;
                }
        } else {
            for (int u = lane; u < units; u += 64) {
                elements<T>(piece(u), y);
                to[u] = codes_of<C>(y, s);
            }
        }
        if (lane == 0) *where = s;
    }
}

}  // namespace
}  // namespace paged

extern "C" int paged_kv_store(const paged_kv_cache *cache, int32_t act, const void *k_new, int64_t k_row,
                              int64_t k_head, const void *v_new, int64_t v_row, int64_t v_head, const int64_t *slots,
                              int32_t n_rows, void *stream) {
    using namespace paged;
    const bool values = cache && cache->v;
    const int rc = check_cache(cache, values);
    if (rc != PAGED_KV_OK) return rc;
    if (n_rows < 0 || (act != PAGED_KV_BF16 && act != PAGED_KV_F16)) return PAGED_KV_EINVAL;
    if (values != (v_new != nullptr) && n_rows > 0) return PAGED_KV_EINVAL;
    if (n_rows == 0) return PAGED_KV_OK;
    if (!k_new || !slots || !aligned16(k_new) || !aligned16(v_new)) return PAGED_KV_EINVAL;
    if (k_row % 8 || k_head % 8 || (values && (v_row % 8 || v_head % 8))) return PAGED_KV_EINVAL;
    if (device_cus() == 0) return PAGED_KV_EUNSUPPORTED;
    StoreArgs a = {};
    a.side[0] = {(uint8_t *)cache->k, cache->k_scale, k_new, k_row, k_head};
    a.side[1] = {(uint8_t *)cache->v, cache->v_scale, v_new, v_row, v_head};
    a.sides = values ? 2 : 1;
    a.slots = slots;
    a.lp = log2_page(cache->page);
    a.n_slots = (int64_t)cache->n_pages << a.lp;
    a.page_stride = cache->page_stride;
    a.scale_stride = cache->scale_stride;
    a.n_rows = n_rows;
    a.dim = cache->head_dim;
    // a window holds from 1 run (a prompt's) to 64 (single tokens): it is shared by
    // as many waves as give the card about 16384, 8 at least
    const int windows = (n_rows + kWindow - 1) / kWindow;
    int splits = kWindow;
    while (splits > 8 && (int64_t)windows * cache->n_heads * a.sides * splits > 16384) splits >>= 1;
    a.splits = splits;
    if ((int64_t)cache->n_heads * a.sides > 65535) return PAGED_KV_EUNSUPPORTED;
    const dim3 grid((unsigned)windows, (unsigned)(cache->n_heads * a.sides), (unsigned)splits);
    if (cache->code == PAGED_KV_E4M3)
        return act == PAGED_KV_BF16 ? launch(store_kernel<bf16, E4M3>, grid, dim3(64), stream, a)
                                    : launch(store_kernel<f16, E4M3>, grid, dim3(64), stream, a);
    return act == PAGED_KV_BF16 ? launch(store_kernel<bf16, Int8>, grid, dim3(64), stream, a)
                                : launch(store_kernel<f16, Int8>, grid, dim3(64), stream, a);
}
