// Attention of few query rows to a cache head: single tokens (one row to a
// request) and selected tokens (one row to a selection).
//
// Bound by memory: 2 D bytes a token and cache head, read once, straight into
// registers.  A wave takes 32 tokens at a time; the query heads of a cache head
// are the 16 columns of its matrix products:
//   S^T [token][col]  = K Q^T       K rows as they lie: lane (m, g) reads 16-byte pieces g, g + 4, .. of token m
//   O^T [dim][col]   += V^T P^T     lane (m, g) reads D/16 bytes at m D/16 of the tokens 4 g + i, i < 4
// The accumulator of S^T holds tokens 4 g + i of column m in lane (m, g), which
// is just the operand layout of P^T with the tokens in the order (i, g); V's
// bytes are brought to it by 4 x 4 byte transposes.  No value crosses lanes
// but the maximum, and that only when it moves by more than 2^8.
// P is rounded to f16 (11 bits, whatever q's type: V's codes are exact in it),
// weighted with V's scale over a reference of each column's own that follows the
// largest product of weight and scale seen so far: full bits down to 2^-20 of that
// product, whatever the scales of pages that weigh nothing.
// (Of the scale alone instead, a page with values 2^22 times as large took the others'
// bits and 2^30 times the others, where it weighed nothing: one long row took 59.2 us
// instead of 60.7 then, the selected prompt block 255 instead of 258.)
// Measured (heads of 128, e4m3): 64 rows of 16384 to 131072 tokens 402 us, 5.75
// TB/s; one row of 131071 tokens on 8 heads 58.3 us; 4096 rows of 2048 selected
// tokens 268 us, 8.0 TB/s of gathers beside vector work in half of the cycles.
#include "paged_attend.h"

namespace paged {
namespace {

constexpr int kBlock = 256;
constexpr int kUnit = 128;     // tokens: 32 to a wave
constexpr int kSliceRows = kStreamRows;
constexpr float kLeastRef = 0x1p-120f;  // of a reference: one over it is finite
constexpr float kMostWeight = 32768.0f; // of a weight in f16

// 32 tokens' codes of one lane.
template <int D>
struct Tile {
    u32x4 k[2][D / 64];
    u32 v[2][4][D / 64];
};

template <int D>
__device__ void load_v(u32 (&to)[D / 64], const uint8_t *p) {
    if constexpr (D == 64) {
        to[0] = *(const u32 *)p;
    } else if constexpr (D == 128) {
        const u32x2 x = *(const u32x2 *)p;
        to[0] = x[0]; to[1] = x[1];
    } else {
        const u32x4 x = *(const u32x4 *)p;
        to[0] = x[0]; to[1] = x[1]; to[2] = x[2]; to[3] = x[3];
    }
}

// One wave's running softmax and values for NT x 16 columns.
template <int D, int NT, class T, class C>
struct Wave {
    typename Act<T>::frag q[NT][D / 32];
    f32x4 o[NT][D / 16];
    float m[NT], l[NT];
    float ref[NT], inv[NT];  // values are held over `ref`, and inv = 1 / ref

    __device__ void clear() {
        for (int t = 0; t < NT; ++t) {
            m[t] = kLow;
            l[t] = 0.0f;
            ref[t] = kLeastRef;
            inv[t] = 1.0f / kLeastRef;
            for (int j = 0; j < D / 16; ++j) o[t][j] = f32x4{0, 0, 0, 0};
        }
    }

    // seen: bit 4 a + i says whether token 16 a + 4 g + i is there; kf, vf: scales
    // of those tokens, the keys' times scale * log2(e).
    __device__ void take(const Tile<D> &x, u32 seen, bool all, const float (&kf)[2][4], const float (&vf)[2][4]) {
        f32x4 s[NT][2];
#pragma unroll
        for (int a = 0; a < 2; ++a) {
#pragma unroll
            for (int t = 0; t < NT; ++t) s[t][a] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int j = 0; j < D / 64; ++j)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const auto kk = eight<C, T>(x.k[a][j][2 * h], x.k[a][j][2 * h + 1]);
#pragma unroll
                    for (int t = 0; t < NT; ++t) s[t][a] = Act<T>::mfma16(kk, q[t][2 * j + h], s[t][a]);
                }
        }
        u32x4 p[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            float top = kLow;
#pragma unroll
            for (int a = 0; a < 2; ++a)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    s[t][a][i] *= kf[a][i];
                    if (!all && !((seen >> (4 * a + i)) & 1)) s[t][a][i] = -__builtin_inff();
                    top = fmaxf(top, s[t][a][i]);
                }
            if (__any(top > m[t] + kSlack)) {
                top = fmaxf(top, __shfl_xor(top, 16));
                top = fmaxf(top, __shfl_xor(top, 32));
                top = fmaxf(top, m[t]);
                const float by = exp2_(m[t] - top), to = ref[t] * by;
                l[t] *= by;
                m[t] = top;
                // the values so far weigh less: so does what they are held over
                if (__any(to < kLeastRef)) {
                    const float left = fminf(to * (1.0f / kLeastRef), 1.0f);
#pragma unroll
                    for (int j = 0; j < D / 16; ++j) o[t][j] *= left;
                }
                ref[t] = fmaxf(to, kLeastRef);
                inv[t] = __builtin_amdgcn_rcpf(ref[t]);
            }
            float e[2][4], w[2][4], most = 0.0f;
            const auto weigh = [&] {
#pragma unroll
                for (int a = 0; a < 2; ++a)
#pragma unroll
                    for (int i = 0; i < 4; ++i) w[a][i] = e[a][i] * fminf(vf[a][i] * inv[t], 3e38f);  // (finite: 0 stays 0)
            };
#pragma unroll
            for (int a = 0; a < 2; ++a)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    e[a][i] = exp2_(s[t][a][i] - m[t]);
                    l[t] += e[a][i];
                }
            weigh();
#pragma unroll
            for (int a = 0; a < 2; ++a)
#pragma unroll
                for (int i = 0; i < 4; ++i) most = fmaxf(most, w[a][i]);
            if (__any(most > kMostWeight)) {  // it is 2^6 then
                float to = 0.0f;
#pragma unroll
                for (int a = 0; a < 2; ++a)
#pragma unroll
                    for (int i = 0; i < 4; ++i) to = fmaxf(to, e[a][i] * vf[a][i]);
                to = fmaxf(to, __shfl_xor(to, 16));
                to = fmaxf(to, __shfl_xor(to, 32));
                to = fmaxf(to * 0.015625f, ref[t]);
                const float by = ref[t] * __builtin_amdgcn_rcpf(to);
#pragma unroll
                for (int j = 0; j < D / 16; ++j) o[t][j] *= by;
                ref[t] = to;
                inv[t] = __builtin_amdgcn_rcpf(to);
                weigh();
            }
            p[t] = u32x4{pack_f16(w[0][0], w[0][1]), pack_f16(w[0][2], w[0][3]), pack_f16(w[1][0], w[1][1]),
                         pack_f16(w[1][2], w[1][3])};
        }
#pragma unroll
        for (int w = 0; w < D / 64; ++w) {
            u32 r[2][4], c[2][4];
#pragma unroll
            for (int a = 0; a < 2; ++a) {
#pragma unroll
                for (int i = 0; i < 4; ++i)  // what is not there is 0 whatever its bytes are
                    r[a][i] = all || ((seen >> (4 * a + i)) & 1) ? x.v[a][i][w] : 0u;
                transpose4(r[a][0], r[a][1], r[a][2], r[a][3], c[a]);
            }
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const auto vv = eight<C, f16>(c[0][b], c[1][b]);
#pragma unroll
                for (int t = 0; t < NT; ++t)
                    o[t][4 * w + b] = Act<f16>::mfma16(vv, __builtin_bit_cast(f16x8, p[t]), o[t][4 * w + b]);
            }
        }
    }
};

template <int D, int NT>
struct Shared {
    float red[16 * NT][D + 4];
    float top[4][16 * NT], sum[4][16 * NT];
    float tops[16 * NT], sums[16 * NT];
    Joined<kBlock> joined;
};

// The four waves' results into sh.red, sh.tops and sh.sums.
template <int D, int NT, class T, class C>
__device__ void join_waves(Wave<D, NT, T, C> &w, Shared<D, NT> &sh) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = lane & 15, g = lane >> 4;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        float l = w.l[t];
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
        if (g == 0) {
            sh.top[wave][16 * t + n] = w.m[t];
            sh.sum[wave][16 * t + n] = l;
        }
    }
    __syncthreads();
    float by[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int c = 16 * t + n;
        float m = sh.top[0][c];
        for (int i = 1; i < 4; ++i) m = fmaxf(m, sh.top[i][c]);
        by[t] = exp2_(w.m[t] - m) * w.ref[t];
        if (wave == 0 && g == 0) {
            float l = 0.0f;
            for (int i = 0; i < 4; ++i) l += sh.sum[i][c] * exp2_(sh.top[i][c] - m);
            sh.tops[c] = m;
            sh.sums[c] = l;
        }
    }
    for (int turn = 0; turn < 4; ++turn) {
        if (turn == wave) {
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < D / 16; j += 4) {
                        f32x4 *to = (f32x4 *)&sh.red[16 * t + n][(4 * g + i) * (D / 16) + j];
                        const f32x4 x = {w.o[t][j][i], w.o[t][j + 1][i], w.o[t][j + 2][i], w.o[t][j + 3][i]};
                        *to = (turn ? *to : f32x4{0, 0, 0, 0}) + x * by[t];
                    }
        }
        __syncthreads();
    }
}

template <int D, int NT, class T, class C>
__device__ void load_q(Wave<D, NT, T, C> &w, const AttendArgs &a, int row, int head0, int heads) {
    const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const bool on = 16 * t + n < heads;
        const char *p = (const char *)a.q + 2 * ((int64_t)row * a.q_row + (int64_t)(head0 + 16 * t + n) * a.q_head);
#pragma unroll
        for (int j = 0; j < D / 64; ++j)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                u32x4 x = {0, 0, 0, 0};
                if (on) x = *(const u32x4 *)(p + 2 * ((g + 4 * j) * 16 + h * 8));
                w.q[t][2 * j + h] = __builtin_bit_cast(typename Act<T>::frag, x);
            }
    }
}

// Where a row's units begin, for up to kSliceRows rows: every workgroup makes the
// plan for itself (a launch that makes it for all costs more: 6 us on a row of
// 131071 tokens).
struct Plan {
    int units[kSliceRows + 1];    // prefix sum
    int starts[kSliceRows + 1];   // row_starts, where they fit
    int waves[kBlock / 64];
};

__device__ void make_plan(const AttendArgs &a, Plan &plan) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t cap = (int64_t)a.table_width << a.lp;
    for (int i = tid; i < a.n_rows; i += kBlock) {
        const int len = (int)min((int64_t)max(a.row_lengths[a.row0 + i], 0), cap);
        plan.units[i] = max((len + kUnit - 1) / kUnit, 1);
    }
    if (a.n_requests <= kSliceRows)
        for (int i = tid; i <= a.n_requests; i += kBlock) plan.starts[i] = a.row_starts[i];
    __syncthreads();
    const int per = (a.n_rows + kBlock - 1) / kBlock, from = min(tid * per, a.n_rows), to = min(from + per, a.n_rows);
    int mine = 0;
    for (int i = from; i < to; ++i) mine += plan.units[i];
    int sum = mine;
    for (int d = 1; d < 64; d <<= 1) {
        const int y = __shfl_up(sum, d);
        if (lane >= d) sum += y;
    }
    if (lane == 63) plan.waves[wave] = sum;
    __syncthreads();
    int at = sum - mine;
    for (int i = 0; i < wave; ++i) at += plan.waves[i];
    for (int i = from; i < to; ++i) {
        const int u = plan.units[i];
        plan.units[i] = at;
        at += u;
    }
    if (tid == kBlock - 1) plan.units[a.n_rows] = at;
    __syncthreads();
}

// Largest i in [0, n) with f(i) <= x, f rising, or 0.
template <class F>
__device__ int last_not_above(int n, int64_t x, F f) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (f(mid) <= x) lo = mid; else hi = mid;
    }
    return lo;
}

// All tokens of single rows.
template <int D, int NT, class T, class C>
__global__ __launch_bounds__(kBlock, D * NT <= 128 ? 2 : 1) void stream_kernel(AttendArgs a) {
    __shared__ Plan plan;
    __shared__ Shared<D, NT> sh;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, m = lane & 15, g = lane >> 4;
    const int P = 1 << a.lp;
    make_plan(a, plan);
    const int vheads = a.kv_heads * a.parts;
    const int64_t total = (int64_t)plan.units[a.n_rows] * vheads;
    // Two workgroups to a CU where each gets 32 units; fewer, down to one to a CU,
    // where the joining of their parts costs more (one row of 131071 tokens on 8
    // heads: 67 us with 256 shares of 32 units, 76 with 512 of 16); but for small
    // calls as many as get two units each (a short batch: 15.7 us, and 21.2 with eight).
    const int64_t shares = min((int64_t)gridDim.x, max((total + 31) / 32, min((total + 1) / 2, (int64_t)gridDim.x / 2)));
    const int share = blockIdx.x;
    if (share >= shares) return;

    const int64_t begin = share_start(share, total, shares);
    int64_t left = share_start(share + 1, total, shares) - begin;
    int ri = last_not_above(a.n_rows, begin, [&](int i) { return (int64_t)plan.units[i] * vheads; });
    int head, unit;
    {
        const int units = plan.units[ri + 1] - plan.units[ri];
        const int64_t in = begin - (int64_t)plan.units[ri] * vheads;
        head = (int)(in / units);
        unit = (int)(in - (int64_t)head * units);
    }
    Wave<D, NT, T, C> w;
    while (left > 0) {
        const int row = a.row0 + ri;
        const int units = plan.units[ri + 1] - plan.units[ri];
        const int end = (int)min((int64_t)units, unit + left);
        const int kvh = head / a.parts, part = head - kvh * a.parts;
        const int head0 = kvh * a.per + part * 16 * NT, heads = min(a.per - part * 16 * NT, 16 * NT);
        w.clear();
        load_q(w, a, row, head0, heads);

        struct { int request, len; } gr;
        {
            const bool fits = a.n_requests <= kSliceRows;
            const int *starts = fits ? plan.starts : a.row_starts;
            gr.request = a.n_requests > 0 ? last_not_above(a.n_requests, row, [&](int i) { return (int64_t)starts[i]; }) : 0;
            const bool known = a.n_requests > 0 && row >= starts[gr.request] && row < starts[gr.request + 1];
            gr.len = known ? (int)min((int64_t)max(a.row_lengths[row], 0), (int64_t)a.table_width << a.lp) : 0;
        }
        const int *pages = a.table + (int64_t)gr.request * a.table_stride;
        const int64_t head_rows = (int64_t)kvh * P * D;
        // tiles of this wave: 32 tokens at kUnit * u + 32 * wave
        const int from = unit, stop = end;
        int known = -1;  // block of 32 units whose pages the lanes hold: lane 2 i + a has unit i's half a
        int page = -1;
        float ks = 0.0f, vs = 0.0f;
        const auto load = [&](Tile<D> &x, int u, int &lim0, int &lim1, float &k0, float &k1, float &v0, float &v1) {
            const int blk = (u - from) >> 5;
            if (blk != known) {
                known = blk;
                const int tok = kUnit * (from + 32 * blk + (lane >> 1)) + 32 * wave + 16 * (lane & 1);
                page = -1;
                ks = vs = 0.0f;
                if (tok < gr.len) {
                    const int pg = pages[tok >> a.lp];
                    if (pg >= 0 && pg < a.n_pages) {
                        page = pg;
                        ks = a.ks[pg * a.scale_stride + kvh] * a.scale2;
                        vs = a.vs[pg * a.scale_stride + kvh];
                    }
                }
            }
            const int i = 2 * ((u - from) & 31);
            const int pg[2] = {__builtin_amdgcn_readlane(page, i), __builtin_amdgcn_readlane(page, i + 1)};
            k0 = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(ks), i));
            k1 = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(ks), i + 1));
            v0 = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(vs), i));
            v1 = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(vs), i + 1));
            const int tok = kUnit * u + 32 * wave;
            lim0 = pg[0] < 0 ? 0 : gr.len - tok;
            lim1 = pg[1] < 0 ? 0 : gr.len - tok - 16;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int64_t at = max(pg[h], 0) * a.page_stride + head_rows + ((tok + 16 * h) & (P - 1)) * D;
                const uint8_t *kp = a.k + at, *vp = a.v + at;
#pragma unroll
                for (int j = 0; j < D / 64; ++j) x.k[h][j] = *(const u32x4 *)(kp + (u32)(m * D + g * 16 + 64 * j));
#pragma unroll
                for (int i2 = 0; i2 < 4; ++i2) load_v<D>(x.v[h][i2], vp + (u32)((4 * g + i2) * D + m * (D / 16)));
            }
        };
        const auto take = [&](const Tile<D> &x, int lim0, int lim1, float k0, float k1, float v0, float v1) {
            const float kf[2][4] = {{k0, k0, k0, k0}, {k1, k1, k1, k1}};
            const float vf[2][4] = {{v0, v0, v0, v0}, {v1, v1, v1, v1}};
            const bool all = lim0 >= 16 && lim1 >= 16;
            u32 seen = 0xFF;
            if (!all)
                seen = ((1u << min(max(lim0 - 4 * g, 0), 4)) - 1) | (((1u << min(max(lim1 - 4 * g, 0), 4)) - 1) << 4);
            if (all) w.take(x, 0xFF, true, kf, vf);
            else if (lim0 > 0 || lim1 > 0) w.take(x, seen, false, kf, vf);
        };
        if (from < stop) {
            Tile<D> x, y;
            int xa, xb, ya, yb;
            float xk0, xk1, xv0, xv1, yk0, yk1, yv0, yv1;
            load(x, from, xa, xb, xk0, xk1, xv0, xv1);
            for (int u = from; u < stop; u += 2) {
                if (u + 1 < stop) load(y, u + 1, ya, yb, yk0, yk1, yv0, yv1);
                take(x, xa, xb, xk0, xk1, xv0, xv1);
                if (u + 1 >= stop) break;
                if (u + 2 < stop) load(x, u + 2, xa, xb, xk0, xk1, xv0, xv1);
                take(y, ya, yb, yk0, yk1, yv0, yv1);
            }
        }
        join_waves(w, sh);
        // who else has a part of this row and head
        const int64_t at = (int64_t)plan.units[ri] * vheads + (int64_t)head * units;
        const int s0 = share_of(at, total, shares), s1 = share_of(at + units - 1, total, shares);
        const int first_slot = 2 * s0 + (at == share_start(s0, total, shares) ? 0 : 1);
        finish<D, 16 * NT, kBlock, T>(
            a, sh.red, sh.tops, sh.sums, sh.joined, heads, s0 == s1, share == s0 ? first_slot : 2 * share, s0,
            s1 - s0 + 1, first_slot, [&](int c) { return (int64_t)row * a.heads + head0 + c; });
        left -= end - unit;
        unit = 0;
        if (++head == vheads) {
            head = 0;
            ++ri;
        }
    }
}

// The selected tokens of single rows: workgroup = (row, head, split).  A wave takes
// 64 of them at a time, looks them up with a lane to a token, and passes rows and
// scales to the lanes that read them through LDS of its own.  Each step of a
// look-up (token, page, scales and codes) is on its way while the 64 before are
// worked on, and no wave waits for another before the end.
template <int D, int NT, class T, class C>
__global__ __launch_bounds__(kBlock, D * NT <= 128 ? 2 : 1) void selected_kernel(AttendArgs a) {
    __shared__ Shared<D, NT> sh;
    // of two times 64 tokens: head row in the cache, or all ones, and the scales
    __shared__ alignas(16) u32 rows[kBlock / 64][2][64];
    __shared__ alignas(16) float kf[kBlock / 64][2][64], vf[kBlock / 64][2][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, m = lane & 15, g = lane >> 4;
    const int P = 1 << a.lp, vheads = a.kv_heads * a.parts;
    // neighbouring rows on one XCD (workgroups go round them), whose L2 then serves
    // the tokens that such rows share
    const int eighth = gridDim.x / 8, b = blockIdx.x;
    const int w0 = b < 8 * eighth ? (b % 8) * eighth + b / 8 : b;
    const int item = w0 / a.splits, split = w0 - item * a.splits;
    const int row = item / vheads, head = item - row * vheads;
    const int kvh = head / a.parts, part = head - kvh * a.parts;
    const int head0 = kvh * a.per + part * 16 * NT, heads = min(a.per - part * 16 * NT, 16 * NT);
    const int units = (a.K + kSelectedUnit - 1) / kSelectedUnit;
    const int from = (int)((int64_t)units * split / a.splits) * kSelectedUnit;
    const int stop = (int)min((int64_t)units * (split + 1) / a.splits * kSelectedUnit, (int64_t)a.K);
    const int *list = a.idx + (int64_t)row * a.K;
    const int first = from + 64 * wave;  // of this wave's tokens, then every kSelectedUnit on
    const auto token = [&](int q) {
        const int64_t i = (int64_t)first + (int64_t)q * kSelectedUnit + lane;
        return i < stop ? list[i] : -1;
    };
    int t0 = token(0), t1 = token(1), t2 = token(2);
    const int request = a.row_request[row];
    const bool known = request >= 0 && request < a.n_requests;
    const int len = known ? (int)min((int64_t)max(a.row_lengths[row], 0), (int64_t)a.table_width << a.lp) : 0;
    const int *pages = a.table + (int64_t)(known ? request : 0) * a.table_stride;
    const u32 page_rows = (u32)(a.page_stride / D);
    const auto page_of = [&](int t) { return t >= 0 && t < len ? pages[t >> a.lp] : -1; };
    const auto row_of = [&](int t, int pg) {
        return (u32)pg < (u32)a.n_pages ? (u32)pg * page_rows + (u32)(kvh * P + (t & (P - 1))) : ~0u;
    };

    Wave<D, NT, T, C> w;
    w.clear();
    load_q(w, a, row, head0, heads);
    const auto load = [&](Tile<D> &x, int at, int i) {
        const u32 *r = rows[wave][at] + i;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const u32 kr = r[16 * h + m];
            const uint8_t *kp = a.k + (uint64_t)(kr == ~0u ? 0u : kr) * D;
#pragma unroll
            for (int j = 0; j < D / 64; ++j) x.k[h][j] = *(const u32x4 *)(kp + g * 16 + 64 * j);
            const u32x4 vr = *(const u32x4 *)&r[16 * h + 4 * g];
#pragma unroll
            for (int e = 0; e < 4; ++e)
                load_v<D>(x.v[h][e], a.v + (uint64_t)(vr[e] == ~0u ? 0u : vr[e]) * D + m * (D / 16));
        }
    };
    const auto take = [&](const Tile<D> &x, int at, int i) {
        u32 seen = 0;
        float k2[2][4], v2[2][4];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int j = i + 16 * h + 4 * g;
            const u32x4 r = *(const u32x4 *)&rows[wave][at][j];
            const f32x4 ks = *(const f32x4 *)&kf[wave][at][j], vs = *(const f32x4 *)&vf[wave][at][j];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                seen |= (r[e] != ~0u ? 1u : 0u) << (4 * h + e);
                k2[h][e] = ks[e];
                v2[h][e] = vs[e];
            }
        }
        if (__all(seen == 0xFF)) w.take(x, 0xFF, true, k2, v2);
        else if (__any(seen != 0)) w.take(x, seen, false, k2, v2);
    };
    const auto put_scales = [&](int at, bool there, float ks, float vs) {
        kf[wave][at][lane] = there ? ks * a.scale2 : 0.0f;
        vf[wave][at][lane] = there ? vs : 0.0f;
        __builtin_amdgcn_wave_barrier();
    };
    if (first < stop) {
        const int times = (stop - first + kSelectedUnit - 1) / kSelectedUnit;
        Tile<D> x, y;
        int p1 = page_of(t1);
        {
            const int p0 = page_of(t0);
            const u32 r = row_of(t0, p0);
            const int64_t s = (int64_t)(r == ~0u ? 0 : p0) * a.scale_stride + kvh;
            const float ks = a.ks[s], vs = a.vs[s];
            rows[wave][0][lane] = r;
            __builtin_amdgcn_wave_barrier();
            load(x, 0, 0);
            put_scales(0, r != ~0u, ks, vs);
        }
        for (int q = 0; q < times; ++q) {
            const int at = q & 1;
            load(y, at, 32);
            take(x, at, 0);
            const u32 r = row_of(t1, p1);
            const int64_t s = (int64_t)(r == ~0u ? 0 : p1) * a.scale_stride + kvh;
            const float ks = a.ks[s], vs = a.vs[s];
            rows[wave][at ^ 1][lane] = r;
            __builtin_amdgcn_wave_barrier();
            t1 = t2;
            p1 = page_of(t1);
            t2 = token(q + 3);
            if (q + 1 < times) load(x, at ^ 1, 0);
            take(y, at, 32);
            put_scales(at ^ 1, r != ~0u, ks, vs);
        }
    }
    join_waves(w, sh);
    // splits of an item have neighbouring workgroups: shares item * splits + split
    const int s0 = item * a.splits;
    finish<D, 16 * NT, kBlock, T>(a, sh.red, sh.tops, sh.sums, sh.joined, heads, a.splits == 1, 2 * (s0 + split), s0,
                                  a.splits, 2 * s0, [&](int c) { return (int64_t)row * a.heads + head0 + c; });
}

template <int D, class T, class C>
int launch_of(const AttendArgs &a, bool selected, int tiles, int grid, void *stream) {
    const dim3 g((unsigned)grid), b(kBlock);
    if constexpr (D < 256)  // (heads of 256 leave no registers for two)
        if (tiles == 2)
            return selected ? launch(selected_kernel<D, 2, T, C>, g, b, stream, a)
                            : launch(stream_kernel<D, 2, T, C>, g, b, stream, a);
    return selected ? launch(selected_kernel<D, 1, T, C>, g, b, stream, a)
                    : launch(stream_kernel<D, 1, T, C>, g, b, stream, a);
}

template <int D>
int launch_dim(const AttendArgs &a, int act, int code, bool selected, int tiles, int grid, void *stream) {
    if (code == PAGED_KV_E4M3)
        return act == PAGED_KV_BF16 ? launch_of<D, bf16, E4M3>(a, selected, tiles, grid, stream)
                                    : launch_of<D, f16, E4M3>(a, selected, tiles, grid, stream);
    return act == PAGED_KV_BF16 ? launch_of<D, bf16, Int8>(a, selected, tiles, grid, stream)
                                : launch_of<D, f16, Int8>(a, selected, tiles, grid, stream);
}

}  // namespace

int launch_stream(const AttendArgs &a, int head_dim, int act, int code, bool selected, int tiles, int grid,
                  void *stream) {
    if (head_dim == 64) return launch_dim<64>(a, act, code, selected, tiles, grid, stream);
    if (head_dim == 128) return launch_dim<128>(a, act, code, selected, tiles, grid, stream);
    return launch_dim<256>(a, act, code, selected, tiles, grid, stream);
}

}  // namespace paged
