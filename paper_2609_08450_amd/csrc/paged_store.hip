// New keys and values into the cache's pages, in 8 bits.
//
// A run is the rows of one page (they follow each other, at consecutive
// places); one workgroup takes a run of one head at a time: the largest
// magnitude, the page's scale, then the codes, K and V alike.  Rows are read
// twice, the second time from the L2.  Bound by memory where the rows are
// many, by the chain load - maximum - store where they are few.
#include "paged_common.h"

namespace paged {
namespace {

constexpr int kBlock = 256;
constexpr int kWindow = 64;  // rows whose slots a workgroup looks through for runs

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

constexpr float kLeast = 7.888609052210118e-31f;  // 2^-100

template <class C>
__device__ float scale_of(float top);
template <>
__device__ float scale_of<E4M3>(float top) {
    // least power of two s with 448 s >= top; 448 = 1.75 * 2^8
    const u32 b = __float_as_uint(top);
    const int e = (int)(b >> 23) - 127 - 8 + ((b & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return __uint_as_float((u32)(max(e, -100) + 127) << 23);
}
template <>
__device__ float scale_of<Int8>(float top) { return fmaxf(__fmul_rn(top, 1.0f / 127.0f), kLeast); }

// Code of x / s, x finite or not.
template <class C>
__device__ u32 code_of(float x, float s);
template <>
__device__ u32 code_of<E4M3>(float x, float s) {
    float y = fminf(fmaxf(__fdiv_rn(x, s), -448.0f), 448.0f);
    y = x != x ? 0.0f : y;
    return (u32)__builtin_amdgcn_cvt_pk_fp8_f32(y, y, 0, false) & 0xFFu;
}
template <>
__device__ u32 code_of<Int8>(float x, float s) {
    float y = fminf(fmaxf(rintf(__fdiv_rn(x, s)), -127.0f), 127.0f);
    y = x != x ? 0.0f : y;
    return (u32)(int)y & 0xFFu;
}

template <class C>
__device__ float value_of(u32 code);
template <>
__device__ float value_of<E4M3>(u32 code) { return __builtin_amdgcn_cvt_f32_fp8((int)code, 0); }
template <>
__device__ float value_of<Int8>(u32 code) { return (float)(signed char)code; }

template <class T>
__device__ float element(u32x4 v, int i) {
    const u32 w = v[i >> 1];
    if constexpr (__is_same(T, bf16)) return __uint_as_float((i & 1) ? w & 0xFFFF0000u : w << 16);
    const f16x2 h = __builtin_bit_cast(f16x2, w);
    return (float)h[i & 1];
}

template <class T, class C>
__global__ __launch_bounds__(kBlock) void store_kernel(StoreArgs a) {
    __shared__ float tops[2][kBlock / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int first = blockIdx.x * kWindow, head = blockIdx.y;
    const int P = 1 << a.lp;
    const auto slot_at = [&](int i) { return i >= 0 && i < a.n_rows ? a.slots[i] : (int64_t)-1; };
    const auto page_at = [&](int64_t s) { return s >= 0 && s < a.n_slots ? s >> a.lp : (int64_t)-1; };

    // the rows of this window that begin a run
    const int64_t s0 = slot_at(first + lane), before = slot_at(first + lane - 1);
    const int64_t p0 = page_at(s0);
    uint64_t begins = __ballot(p0 >= 0 && !(page_at(before) == p0 && before + 1 == s0));
    for (int k = 0; begins; ++k) {
        const int at = __builtin_ctzll(begins);
        begins &= begins - 1;
        if (k % a.splits != (int)blockIdx.z) continue;
        const int row = first + at;
        const int64_t slot = a.slots[row], page = slot >> a.lp;
        const int place = (int)(slot & (P - 1));
        // its length: rows up to the page's end whose slots go on
        int count = 1;
        for (int base = 1; base < P - place; base += 64) {
            const int j = base + lane;
            const bool on = j < P - place && slot_at(row + j) == slot + j;
            const uint64_t m = __ballot(on);
            const int run = ~m ? __builtin_ctzll(~m) : 64;
            count += run;
            if (run < 64) break;
        }
        const int per = a.dim / 8, units = count * per;  // eight elements at a time

        float top[2] = {0.0f, 0.0f};
        for (int t = 0; t < a.sides; ++t) {
            const char *x = (const char *)a.side[t].x;
            for (int u = tid; u < units; u += kBlock) {
                const int j = u / per, d = (u - j * per) * 8;
                const u32x4 v = *(const u32x4 *)(x + 2 * ((row + j) * a.side[t].row + head * a.side[t].head + d));
                for (int i = 0; i < 8; ++i) {
                    const float y = fabsf(element<T>(v, i));
                    top[t] = y < __builtin_inff() ? fmaxf(top[t], y) : top[t];  // finite ones alone
                }
            }
            for (int d = 32; d; d >>= 1) top[t] = fmaxf(top[t], __shfl_xor(top[t], d));
            if (lane == 0) tops[t][wave] = top[t];
        }
        __syncthreads();
        for (int t = 0; t < a.sides; ++t) {
            const Side &o = a.side[t];
            float m = 0.0f;
            for (int i = 0; i < kBlock / 64; ++i) m = fmaxf(m, tops[t][i]);
            float *where = o.scale + page * a.scale_stride + head;
            const float fresh = scale_of<C>(m), old = *where;
            const float s = place > 0 ? fmaxf(old, fresh) : fresh;
            uint8_t *codes = o.codes + page * a.page_stride + (int64_t)head * P * a.dim;
            if (place > 0 && s > old) {
                // codes under a smaller scale: (code * old) / s, rounded anew
                for (int u = tid; u < place * a.dim / 4; u += kBlock) {
                    const u32 w = ((const u32 *)codes)[u];
                    u32 z = 0;
                    for (int i = 0; i < 4; ++i)
                        z |= code_of<C>(__fmul_rn(value_of<C>((w >> (8 * i)) & 0xFFu), old), s) << (8 * i);
                    ((u32 *)codes)[u] = z;
                }
            }
            const char *x = (const char *)o.x;
            for (int u = tid; u < units; u += kBlock) {
                const int j = u / per, d = (u - j * per) * 8;
                const u32x4 v = *(const u32x4 *)(x + 2 * ((row + j) * o.row + head * o.head + d));
                u32 z[2] = {0, 0};
                for (int i = 0; i < 8; ++i) z[i >> 2] |= code_of<C>(element<T>(v, i), s) << (8 * (i & 3));
                *(u32x2 *)(codes + (int64_t)(place + j) * a.dim + d) = u32x2{z[0], z[1]};
            }
            __syncthreads();  // everyone has read the old scale
            if (tid == 0) *where = s;
        }
        __syncthreads();
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
    // a window holds from 1 run (a prompt's) to 64 (single tokens): it is shared
    // by as many workgroups as give the card about 4096, 2 at least
    const int windows = (n_rows + kWindow - 1) / kWindow;
    int splits = kWindow;
    while (splits > 2 && (int64_t)windows * cache->n_heads * splits > 4096) splits >>= 1;
    a.splits = splits;
    if (cache->n_heads > 65535) return PAGED_KV_EUNSUPPORTED;
    const dim3 grid((unsigned)windows, (unsigned)cache->n_heads, (unsigned)splits);
    if (cache->code == PAGED_KV_E4M3)
        return act == PAGED_KV_BF16 ? launch(store_kernel<bf16, E4M3>, grid, dim3(kBlock), stream, a)
                                    : launch(store_kernel<f16, E4M3>, grid, dim3(kBlock), stream, a);
    return act == PAGED_KV_BF16 ? launch(store_kernel<bf16, Int8>, grid, dim3(kBlock), stream, a)
                                : launch(store_kernel<f16, Int8>, grid, dim3(kBlock), stream, a);
}
