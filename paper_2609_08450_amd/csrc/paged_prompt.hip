// Attention of many query rows to a cache head: prompts and chunks of them.
//
// Bound by the matrix products (4 D operations a pair of row and token) and by
// the vector work of the softmax beside them.  A workgroup holds COLS columns
// (rows x query heads of one cache head), 32 to a wave, their Q in registers;
// tiles of 64 tokens go through LDS once for all waves, already as 16-bit
// floats, while the next tile's codes are on their way from memory:
//   S^T [token][col]  = K Q^T        O^T [dim][col] += V^T P^T
// as 32 x 32 x 16 products.  The accumulator of S^T is the operand of P^T when
// V's tokens are laid out in its order, so P never leaves its registers; V is
// transposed on its way into LDS, by bytes.  4096 rows of three prompts of up to
// 13000 tokens, 32 heads of 128 on 8: 473 us with plan and joining, 850 TFLOP/s
// (a library's bf16 product reaches 1415).  Matrix cores are busy in 39 % of a
// SIMD's cycles and vector instructions issue in 48 %: its two waves overlap the two
// only in part.
#include "paged_attend.h"

namespace paged {
namespace {

constexpr int kTile = 64;
constexpr float kNoScale = -200.0f;  // log2 of a scale of 0, near enough: below every scale that a value survives
constexpr float kFaint = -60.0f;     // weights this far (powers of 2) below the maximum's have values of 0 in f16

// Chunk of 16 bytes of V's row d that holds chunk c: reads of 32 rows and writes
// of every fourth row both spread over the banks.
__device__ inline int swizzled(int d, int c) { return c ^ (((d >> 1) & 7) ^ ((d >> 4) & 1)); }

template <int D, int WAVES>
struct Buffers {
    alignas(16) uint8_t k[kTile][2 * D + 16];
    alignas(16) uint8_t v[D][2 * kTile];
    alignas(16) float kf[4], lv[4];  // of each 16 tokens: the keys' scale, the values' as a power of 2
    u32 valid;           // bit of each 16 tokens: its page is in the cache
};

template <int D, int WAVES, class T, class C>
__global__ __launch_bounds__(64 * WAVES) void prompt_kernel(AttendArgs a) {
    constexpr int THREADS = 64 * WAVES, COLS = 32 * WAVES, PART = COLS * (D + 2);
    constexpr int KI = kTile * D / 16, KN = (KI + THREADS - 1) / THREADS;  // 16-byte pieces of K, and of a thread
    constexpr int VI = (kTile / 4) * (D / 4), VN = (VI + THREADS - 1) / THREADS;  // 4 x 4 pieces of V
    __shared__ Buffers<D, WAVES> buf[2];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = lane & 31, g = lane >> 5;
    const int P = 1 << a.lp;
    const int64_t total = a.total[0], shares = a.total[1];

    // rows that no request has: before the first one's, and past the last one's
    const int lead = min(max(a.row_starts[0], 0), a.n_rows), past = max(a.row_starts[a.n_requests], lead);
    for (int64_t j = blockIdx.x; j < (int64_t)lead + max(a.n_rows - past, 0); j += gridDim.x) {
        const int64_t i = j < lead ? j : past + (j - lead);
        for (int e = tid; e < a.heads * D / 2; e += THREADS) ((u32 *)a.out)[i * a.heads * D / 2 + e] = 0;
        if (a.lse)
            for (int e = tid; e < a.heads; e += THREADS) a.lse[i * a.heads + e] = -__builtin_inff();
    }
    if ((int)blockIdx.x >= shares) return;

    // neighbouring shares, which read the same keys and values, on one XCD (workgroups
    // go round them), where every workgroup has one (501 us instead of 510 for 4096 rows
    // of three prompts)
    const int eighth = gridDim.x / 8, b8 = blockIdx.x;
    const int share = shares == gridDim.x && b8 < 8 * eighth ? (b8 % 8) * eighth + b8 / 8 : b8;
    const int64_t begin = share_start(share, total, shares);
    int64_t left = share_start(share + 1, total, shares) - begin;
    const int4 st = a.starts[share];
    int gi = st.x, head = st.y, unit = st.z, r = st.w;
    const int vheads = a.kv_heads * a.parts;
    const int per_row = min(a.per, COLS);  // columns of a row
    while (left > 0) {
        const Group gr = a.groups[gi];
        const int units = a.group_units[gi + 1] - a.group_units[gi];
        const int end = (int)min((int64_t)units, unit + left);
        const int kvh = head / a.parts, part = head - kvh * a.parts;
        const int *pages = a.table + (int64_t)gr.request * a.table_stride;

        // this lane's column
        const int col = 32 * wave + n, crow = col / per_row, chead = part * COLS + (col - crow * per_row);
        const bool on = crow < gr.rows && chead < a.per;
        const int64_t out_at = on ? (int64_t)(gr.row0 + crow) * a.heads + kvh * a.per + chead : -1;
        const int len = on ? min(a.row_lengths[gr.row0 + crow], gr.len) : 0;
        typename Act<T>::frag q[D / 16];
        {
            const char *p = (const char *)a.q + 2 * ((int64_t)(gr.row0 + crow) * a.q_row +
                                                     (int64_t)(kvh * a.per + chead) * a.q_head);
#pragma unroll
            for (int k = 0; k < D / 16; ++k) {
                u32x4 x = {0, 0, 0, 0};
                if (on) x = *(const u32x4 *)(p + 2 * (16 * k + 8 * g));
                q[k] = __builtin_bit_cast(typename Act<T>::frag, x);
            }
        }
        int shortest = on ? len : 0x7FFFFFFF, longest = len;
        for (int d = 16; d; d >>= 1) {
            shortest = min(shortest, __shfl_xor(shortest, d));
            longest = max(longest, __shfl_xor(longest, d));
        }
        shortest = __builtin_amdgcn_readfirstlane(shortest);
        longest = __builtin_amdgcn_readfirstlane(longest);

        f32x16 o[D / 32];
        for (int t = 0; t < D / 32; ++t)
            for (int i = 0; i < 16; ++i) o[t][i] = 0.0f;
        // The sum is held over 2^m, values over 2^ref.  `ref` follows the largest product of
        // weight and scale that the column has seen: f16 weights keep their bits down to
        // 2^-20 of that one, whatever the scales of pages that weigh nothing or that its
        // row does not see.
        float m = kLow, l = 0.0f, ref = kLow;

        // Codes on their way: pages a tile ahead of codes, codes a tile ahead of use.
        // Nothing that is loaded is used where it is loaded, not even in a
        // comparison: that would wait for all of it there.  A wave's tokens of one
        // load lie in 16 aligned ones, so in one page: pages are scalars, but loaded as
        // vectors (`zero` is no constant to the compiler), since LDS's pieces could not
        // be waited for one by one beside a scalar load.
        int zero = 0;
        asm("" : "+v"(zero));
        int kpage[KN], vpage[VN], spage = 0;
        u32x4 kc[KN];
        u32 vc[VN][4];
        float sc = 0.0f;
        const int last_tok = max(gr.len - 1, 0), wave_s = __builtin_amdgcn_readfirstlane(wave);
        const auto page_at = [&](int tok) { return pages[(min(tok, last_tok) >> a.lp) + zero]; };
        const auto in_cache = [&](int pg) { return (u32)pg < (u32)a.n_pages; };
        const auto k_tok = [&](int e) { return (64 * wave_s + e * THREADS) % KI / (D / 16); };      // first of the wave's
        const auto v_tok = [&](int e) { return (64 * wave_s + e * THREADS) % VI / (D / 4) * 4; };
        const auto look_up = [&](int u) {
#pragma unroll
            for (int e = 0; e < KN; ++e) kpage[e] = page_at(kTile * u + k_tok(e));
#pragma unroll
            for (int e = 0; e < VN; ++e) vpage[e] = page_at(kTile * u + v_tok(e));
            if (wave_s == 0) spage = page_at(kTile * u + 16 * (lane & 3));
        };
        int vleft[VN];  // tokens from the wave's first of vc on that are there
        bool sthere = false;
        const auto fetch = [&](int u) {
#pragma unroll
            for (int e = 0; e < KN; ++e) {
                const int tok = kTile * u + k_tok(e), pg = __builtin_amdgcn_readfirstlane(kpage[e]);
                const uint8_t *p = a.k + (in_cache(pg) ? pg : 0) * a.page_stride +
                                   ((int64_t)kvh * P + (tok & (P - 1))) * D;
                kc[e] = *(const u32x4 *)(p + (u32)(16 * lane));
            }
#pragma unroll
            for (int e = 0; e < VN; ++e) {
                const int tok = kTile * u + v_tok(e), pg = __builtin_amdgcn_readfirstlane(vpage[e]);
                const bool there = in_cache(pg);
                const uint8_t *p = a.v + (there ? pg : 0) * a.page_stride +
                                   ((int64_t)kvh * P + (tok & (P - 1))) * D;
                const u32 at = lane / (D / 4) * 4 * D + lane % (D / 4) * 4;
#pragma unroll
                for (int j = 0; j < 4; ++j) vc[e][j] = *(const u32 *)(p + (at + j * D));
                vleft[e] = there ? gr.len - tok : 0;
            }
            if (wave_s == 0) {
                sthere = in_cache(spage) && kTile * u + 16 * (lane & 3) < gr.len;
                sc = (lane < 4 ? a.ks : a.vs)[(sthere ? spage : 0) * a.scale_stride + kvh];
            }
        };
        const auto lay_out = [&](Buffers<D, WAVES> &b) {
#pragma unroll
            for (int e = 0; e < KN; ++e) {
                const int i = tid + e * THREADS;
                if (KI % THREADS != 0 && i >= KI) break;
                u32x4 *to = (u32x4 *)&b.k[i / (D / 16)][i % (D / 16) * 32];
                const u32x2 x0 = Four<C, T>::of(kc[e][0]), x1 = Four<C, T>::of(kc[e][1]);
                const u32x2 x2 = Four<C, T>::of(kc[e][2]), x3 = Four<C, T>::of(kc[e][3]);
                to[0] = u32x4{x0[0], x0[1], x1[0], x1[1]};
                to[1] = u32x4{x2[0], x2[1], x3[0], x3[1]};
            }
#pragma unroll
            for (int e = 0; e < VN; ++e) {
                const int i = tid + e * THREADS;
                if (VI % THREADS != 0 && i >= VI) break;
                const int quad = i / (D / 4), d = i % (D / 4) * 4;
                // tokens 16 s + 8 half + 4 g + j of 32 lie at 16 s + 8 g + 4 half + j
                const int chunk = (quad >> 2) * 2 + (quad & 1), half = (quad >> 1) & 1;
                if (vleft[e] < 64 / (D / 4) * 4) {  // bytes of tokens that are not there are 0 whatever they hold
                    const int n = vleft[e] - lane / (D / 4) * 4;
#pragma unroll
                    for (int j = 0; j < 4; ++j) vc[e][j] = j < n ? vc[e][j] : 0u;
                }
                u32 x[4];
                transpose4(vc[e][0], vc[e][1], vc[e][2], vc[e][3], x);
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    *(u32x2 *)&b.v[d + j][16 * swizzled(d + j, chunk) + 8 * half] = Four<C, f16>::of(x[j]);
            }
            if (wave_s == 0) {
                const float s = sthere ? sc : 0.0f;
                if (lane < 4) b.kf[lane] = s * a.scale2;
                else if (lane < 8) b.lv[lane - 4] = s > 0.0f ? __log2f(s) : kNoScale;
                const u32 valid = (u32)__ballot(lane < 4 && sthere);
                if (lane == 0) b.valid = valid;
            }
        };

        if (unit < end) {
            look_up(unit);
            fetch(unit);
            if (unit + 1 < end) look_up(unit + 1);
            lay_out(buf[0]);
            __syncthreads();
            for (int u = unit; u < end; ++u) {
                const Buffers<D, WAVES> &b = buf[(u - unit) & 1];
                if (u + 1 < end) {
                    fetch(u + 1);
                    look_up(u + 2);
                }
                const int tok0 = kTile * u;
                if (tok0 < longest) {
                    const u32 valid = __builtin_amdgcn_readfirstlane(b.valid);
                    const bool all = valid == 15u && tok0 + kTile <= shortest;
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        // All of LDS's pieces are asked for ahead of the products, and V's ahead of
                        // the softmax: one after the other each would cost LDS's latency.
                        f32x16 s;
#pragma unroll
                        for (int i = 0; i < 16; ++i) s[i] = 0.0f;
                        constexpr int AHEAD = D / 16 < 8 ? D / 16 : 8;
#pragma unroll
                        for (int k0 = 0; k0 < D / 16; k0 += AHEAD) {
                            typename Act<T>::frag kk[AHEAD];
#pragma unroll
                            for (int k = 0; k < AHEAD; ++k)
                                kk[k] = __builtin_bit_cast(typename Act<T>::frag,
                                                           *(const u32x4 *)&b.k[32 * t + n][32 * (k0 + k) + 16 * g]);
                            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                            for (int k = 0; k < AHEAD; ++k) s = Act<T>::mfma32(kk[k], q[k0 + k], s);
                        }
                        // (half of V's where a head of 256 leaves no registers for more)
                        constexpr int EARLY = D == 256 ? 1 : 2;
                        f16x8 vv[EARLY][D / 32];
                        const auto v_piece = [&](int h, int d) {
                            const int vd = 32 * d + n;
                            return __builtin_bit_cast(f16x8,
                                                      *(const u32x4 *)&b.v[vd][16 * swizzled(vd, 4 * t + 2 * h + g)]);
                        };
#pragma unroll
                        for (int h = 0; h < EARLY; ++h)
#pragma unroll
                            for (int d = 0; d < D / 32; ++d) vv[h][d] = v_piece(h, d);
                        const f32x2 kf = *(const f32x2 *)&b.kf[2 * t], lv = *(const f32x2 *)&b.lv[2 * t];
                        __builtin_amdgcn_sched_barrier(0);
                        // A weight with its value's scale is 2^(s kf + lv - ref): one multiply-add and one
                        // exponential; scales are not negative, so the maximum is taken before them.
                        u32 gone = 0;
                        if (!all)
#pragma unroll
                            for (int i = 0; i < 16; ++i) {
                                const int tok = tok0 + 32 * t + 8 * (i >> 2) + 4 * g + (i & 3);
                                if (tok >= len || !((valid >> (2 * t + (i >> 3))) & 1)) gone |= 1u << i;
                            }
                        float x[2];  // of 16 tokens each, in powers of 2
                        const auto highest = [&](auto masked) {
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                x[h] = -__builtin_inff();
#pragma unroll
                                for (int i = 8 * h; i < 8 * h + 8; ++i)
                                    x[h] = fmaxf(x[h], decltype(masked)::value && ((gone >> i) & 1) ? -__builtin_inff() : s[i]);
                                x[h] *= kf[h];  // (NaN of -inf and 0, which the maxima pass over)
                            }
                        };
                        if (all) highest(std::false_type{});
                        else highest(std::true_type{});
                        float top = fmaxf(fmaxf(kLow, x[0]), x[1]);
                        float heavy = fmaxf(x[0] + lv[0], x[1] + lv[1]);
                        if (__any(top > m + kSlack || heavy > ref + 15.0f)) {  // weights stay below 2^15 in f16
                            top = fmaxf(fmaxf(top, __shfl_xor(top, 32)), m);
                            l *= exp2_(m - top);
                            m = top;
                            heavy = fmaxf(heavy, __shfl_xor(heavy, 32));
                            if (__any(heavy > ref + 15.0f)) {
                                const float to = fmaxf(heavy - 6.0f, ref), by = exp2_(ref - to);
#pragma unroll
                                for (int d = 0; d < D / 32; ++d) o[d] *= by;
                                ref = to;
                            }
                        }
                        u32x4 p[2];
                        const auto weigh = [&](auto masked) {
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                const float f = kf[h], c = fmaxf(lv[h] - ref, kFaint - m);
                                float e[8], sum = 0.0f;
#pragma unroll
                                for (int i = 0; i < 8; ++i) {
                                    e[i] = exp2_(fmaf(s[8 * h + i], f, c));
                                    if (decltype(masked)::value && ((gone >> (8 * h + i)) & 1)) e[i] = 0.0f;
                                    sum += e[i];
                                }
                                p[h] = u32x4{pack_f16(e[0], e[1]), pack_f16(e[2], e[3]), pack_f16(e[4], e[5]),
                                             pack_f16(e[6], e[7])};
                                l = fmaf(sum, exp2_(-m - c), l);  // (the scale off again)
                            }
                        };
                        if (all) weigh(std::false_type{});
                        else weigh(std::true_type{});
#pragma unroll
                        for (int h = 0; h < 2; ++h)
#pragma unroll
                            for (int d = 0; d < D / 32; ++d)
                                o[d] = Act<f16>::mfma32(h < EARLY ? vv[h % EARLY][d] : v_piece(h, d),
                                                        __builtin_bit_cast(f16x8, p[h]), o[d]);
                    }
                }
                if (u + 1 < end) lay_out(buf[(u + 1 - unit) & 1]);
                __syncthreads();
            }
        }
        l += __shfl_xor(l, 32);

        // who else has a part of this group
        const int gb0 = a.group_base[r], gb1 = a.group_base[r + 1];
        const int64_t ru = a.group_units[gb1] - a.group_units[gb0];
        const int64_t at = (int64_t)a.group_units[gb0] * vheads + head * ru + (a.group_units[gi] - a.group_units[gb0]);
        const int s0 = share_of(at, total, shares), s1 = share_of(at + units - 1, total, shares), parts = s1 - s0 + 1;
        const float half = exp2_(0.5f * (ref - m));  // twice: this power may lie below FP32's normal numbers where the values do not
#pragma unroll
        for (int d = 0; d < D / 32; ++d) o[d] *= half;
        if (parts == 1) {
            const float by = l != 0.0f ? half / l : 0.0f;
            if (out_at >= 0) {
#pragma unroll
                for (int d = 0; d < D / 32; ++d)
#pragma unroll
                    for (int b = 0; b < 4; ++b)
                        *(u32x2 *)((uint16_t *)a.out + out_at * D + 32 * d + 8 * b + 4 * g) =
                            u32x2{pack2<T>(o[d][4 * b] * by, o[d][4 * b + 1] * by),
                                  pack2<T>(o[d][4 * b + 2] * by, o[d][4 * b + 3] * by)};
                if (a.lse && g == 0)
                    a.lse[out_at] = l != 0.0f ? (m + __log2f(l)) * 0.6931471805599453f : -__builtin_inff();
            }
        } else {
            const int first_slot = 2 * s0 + (at == share_start(s0, total, shares) ? 0 : 1);
            float *mine = a.left + (int64_t)(share == s0 ? first_slot : 2 * share) * PART;
            if (g == 0) *(f32x2 *)(mine + 2 * col) = f32x2{m, l};
#pragma unroll
            for (int d = 0; d < D / 32; ++d)
#pragma unroll
                for (int b = 0; b < 4; ++b)
                    *(f32x4 *)(mine + 2 * COLS + col * D + 32 * d + 8 * b + 4 * g) =
                        f32x4{o[d][4 * b], o[d][4 * b + 1], o[d][4 * b + 2], o[d][4 * b + 3]} * half;
        }
        left -= end - unit;
        unit = 0;
        if (left > 0) {
            ++gi;
            if (gi == gb1) {
                if (++head < vheads) gi = gb0;
                else head = 0;
            }
            if (head == 0 && gi == gb1) r = a.groups[gi].request;
        }
    }
}

// Groups that lie in several shares, after prompt_kernel: workgroup = (the share
// that such a group begins in, 16 of its columns).  (By the last workgroup to
// arrive instead, four rows over 65000 tokens took 93 us, and one row of 128 heads
// over 60000 took 392.)
template <int D, int WAVES, class T>
__global__ __launch_bounds__(256) void join_kernel(AttendArgs a) {
    constexpr int COLS = 32 * WAVES, PART = COLS * (D + 2);
    __shared__ Joined<256> joined;
    const int64_t total = a.total[0], shares = a.total[1];
    const int w = blockIdx.x, first = 16 * blockIdx.y;
    if (w + 1 >= shares) return;
    const int4 st = a.starts[w + 1];
    if (st.z == 0) return;  // share w + 1 begins with a group
    const int vheads = a.kv_heads * a.parts, head = st.y;
    const int gb0 = a.group_base[st.w], gb1 = a.group_base[st.w + 1];
    const int64_t ru = a.group_units[gb1] - a.group_units[gb0];
    const int units = a.group_units[st.x + 1] - a.group_units[st.x];
    const int64_t at = (int64_t)a.group_units[gb0] * vheads + head * ru + (a.group_units[st.x] - a.group_units[gb0]);
    const int s0 = share_of(at, total, shares), s1 = share_of(at + units - 1, total, shares);
    if (s0 != w) return;  // it began earlier
    const Group gr = a.groups[st.x];
    const int per_row = min(a.per, COLS), cols = min(gr.rows * per_row, COLS);
    if (first >= cols) return;
    const int kvh = head / a.parts, part = head - kvh * a.parts;
    const int first_slot = 2 * s0 + (at == share_start(s0, total, shares) ? 0 : 1);
    join_parts<D, COLS, 256, false>(
        joined, s1 - s0 + 1, first, min(first + 16, cols),
        [&](int p) { return a.left + (int64_t)(p == 0 ? first_slot : 2 * (s0 + p)) * PART; },
        [&](int c, int d, f32x4 x, float m, float l) {
            const int row = c / per_row, h = part * COLS + (c - row * per_row);
            if (h < a.per)
                write_out<D, T>(a, (int64_t)(gr.row0 + row) * a.heads + kvh * a.per + h, d, x, m, l);
        });
}

template <int D, int WAVES>
int launch_dim(const AttendArgs &a, int act, int code, int grid, void *stream) {
    const dim3 g((unsigned)grid), b(64 * WAVES);
    const auto go = [&](void (*kernel)(AttendArgs)) { return launch(kernel, g, b, stream, a); };
    const int rc = code == PAGED_KV_E4M3 ? go(act == PAGED_KV_BF16 ? prompt_kernel<D, WAVES, bf16, E4M3>
                                                                   : prompt_kernel<D, WAVES, f16, E4M3>)
                                         : go(act == PAGED_KV_BF16 ? prompt_kernel<D, WAVES, bf16, Int8>
                                                                   : prompt_kernel<D, WAVES, f16, Int8>);
    if (rc != PAGED_KV_OK || grid < 2) return rc;
    const dim3 joins((unsigned)(grid - 1), 2 * WAVES);
    return act == PAGED_KV_BF16 ? launch(join_kernel<D, WAVES, bf16>, joins, dim3(256), stream, a)
                                : launch(join_kernel<D, WAVES, f16>, joins, dim3(256), stream, a);
}

}  // namespace

int launch_prompt(const AttendArgs &a, int head_dim, int act, int code, int grid, void *stream) {
    if (head_dim == 64) return launch_dim<64, 8>(a, act, code, grid, stream);
    if (head_dim == 128) return launch_dim<128, 8>(a, act, code, grid, stream);
    return launch_dim<256, 4>(a, act, code, grid, stream);
}

}  // namespace paged
