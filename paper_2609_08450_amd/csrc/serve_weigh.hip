// What every token of the cache gets of a step's attention:
//   w_j += sum over rows i that see j, heads h of exp(scale q_ih . k_j - lse_ih).
//
// The softmax is known (lse), so tokens need nothing of each other: a wave holds the
// keys of some tokens as the columns of 32 x 32 x 16 products and passes queries by, from
// LDS.  A token's results lie in one lane of each half wave, 16 queries to an accumulator:
// the sum over queries is the lane's own, and the halves meet once at the end.
//
// Keys and queries are exact in the products (codes convert exactly to bf16 and f16), whose sums, the
// exponentials and all sums of them are FP32.
//
// weigh_rows_kernel, few rows: bound by memory, the codes read once (64 single rows of 16384 to 131072
// tokens, 2 heads of 128: 252 us, 4.71 TB/s; the same loads without the products 239 us, or 232 in one
// line).  Codes fetched ahead (265 us), pages and old weights ahead (267 to 281), one token to a lane (256)
// and equal shares for resident workgroups (305) were slower: waves of other workgroups cover the trips.
//
// weigh_block_kernel, many rows: bound by matrix and vector work, 2 instructions a result and an exponential
// at a quarter of their rate (4096 rows of three prompts, 32 heads of 128: 223 us with the plan's 8 and the
// join's 9, 905 TFLOP/s; 16 heads of 256: 225 us).  Matrix cores are busy in 43 % of the cycles and vector instructions
// issue in 57 %, which is all of them: the two follow one another more than they overlap.  Tiles of keys
// through LDS and an order left to the compiler took 265 us and more.
#include <cfloat>

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
    int64_t limit;   // rows x heads of the requests that the kernel of few rows takes
    u32 page_rows;   // rows of head_dim codes from one page to the next
    float scale2, stretch;  // scale * log2(e), and what its rounding leaves of it: (1 + stretch) scale2
    float *weights;
    const int64_t *weight_offsets;
};

// log2 of a softmax's sum as an FP32 number that exponents are taken from, and what its rounding
// and that of the call's scale leave, as a factor: near p's that count, q . k is about lse, so a
// scale off by `stretch` of itself is off by stretch * lse there.
struct Softmax {
    float lse2, fine;  // inf, 0: nothing is added
};
__device__ inline Softmax softmax_of(float lse, float stretch) {
    if (fabsf(lse) == __builtin_inff()) return {__builtin_inff(), 0.0f};
    constexpr float lo = 1.9259629911266175e-8f;  // log2(e) - kLog2e
    const float hi = lse * kLog2e;
    const float rest = fmaf(lse, kLog2e, -hi) + lse * lo;
    // (a factor of 0 or inf, of an lse past 1e9, would make NaN of the inf or the 0 that it belongs to)
    return {hi, exp2_(fminf(fmaxf(fmaf(hi, stretch, -rest), -126.0f), 126.0f))};
}

// Query columns in LDS.
constexpr int columns_of(int dim) { return dim == 256 ? 64 : 128; }

template <int D>
struct Columns {
    alignas(16) uint8_t q[columns_of(D)][2 * D + 16];
    alignas(16) float lse2[columns_of(D) + 32], fine[columns_of(D) + 32];
    alignas(16) int len[columns_of(D) + 32];
};

// Rows of a request: workgroup = (request, `steps` tiles of tokens), all heads.  SPLIT waves have the same
// tokens (then steps is 1), and share out the heads, or a head's columns.
template <int D, class T, class C, int SPLIT>
__global__ __launch_bounds__(kBlock) void weigh_rows_kernel(WeighArgs a) {
    constexpr int NT = kTokens, COLS = columns_of(D), TILE = kTile / SPLIT;
    typedef typename Act<T>::frag frag;
    __shared__ Columns<D> b;
    __shared__ float shared[SPLIT > 1 ? SPLIT : 1][32 * NT];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = lane & 31, g = lane >> 5;
    const int r = blockIdx.y;
    const int row0 = min(max(a.row_starts[r], 0), a.n_rows), row1 = min(max(a.row_starts[r + 1], row0), a.n_rows);
    if ((int64_t)(row1 - row0) * a.heads > a.limit) return;
    const int64_t cap = (int64_t)a.table_width << a.lp;
    int longest = 0;
    for (int i = row0 + lane; i < row1; i += 64) {
        const int len = (int)min((int64_t)max(a.row_lengths[i], 0), cap);
        longest = max(longest, len);
    }
    for (int d = 32; d; d >>= 1) longest = max(longest, __shfl_xor(longest, d));
    longest = __builtin_amdgcn_readfirstlane(longest);
    const int64_t first = (int64_t)blockIdx.x * TILE * a.steps;
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
                Softmax x = {__builtin_inff(), 0.0f};
                int len = 0;
                if (i < heads * cols) {
                    const int h = i / cols;
                    const int64_t col = col0 + i - h * cols;
                    const int row = row0 + (int)(col / a.per);
                    x = softmax_of(a.lse[(int64_t)row * a.heads + (head0 + h) * a.per + (int)(col % a.per)], a.stretch);
                    // (a column without a softmax sees nothing: a key that is NaN would make its product NaN, 0 or not)
                    if (x.lse2 != __builtin_inff()) len = (int)min((int64_t)max(a.row_lengths[row], 0), cap);
                }
                b.lse2[i] = x.lse2;
                b.fine[i] = x.fine;
                b.len[i] = len;
            }
            __syncthreads();
            for (int s = 0; s < a.steps; ++s) {
                const int64_t base = first + (int64_t)s * TILE + 32 * NT * (SPLIT > 1 ? wave / SPLIT : wave);
                if (base >= longest) break;
                const int tok = (int)base + NT * n;
                const int pg = pages[min((int64_t)tok, cap - 1) >> a.lp];
                const bool there = pg >= 0 && pg < a.n_pages;
                const uint8_t *codes = a.k + (there ? pg : 0) * a.page_stride + (int64_t)(tok & ((1 << a.lp) - 1)) * D + 16 * g;
                const float *scales = a.ks + (there ? pg : 0) * a.scale_stride;
                float sum[NT];
#pragma unroll
                for (int t = 0; t < NT; ++t) sum[t] = 0.0f;
                for (int h = 0; h < heads; ++h) {
                    int c = 0;  // the wave's first columns: every SPLIT-th 32 of all heads'
                    if constexpr (SPLIT > 1) {
                        c = 32 * ((wave - h * ((cols + 31) / 32)) & (SPLIT - 1));
                        if (c >= cols) continue;
                    }
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
                    for (; c < cols; c += 32 * SPLIT) {
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
                                const float l = b.lse2[at + col], f = b.fine[at + col];
                                const int len = b.len[at + col];
#pragma unroll
                                for (int t = 0; t < NT; ++t) {
                                    const float p = exp2_(fmaf(x[t][i0 + i], scale, -l)) * f;
                                    sum[t] += tok + t < len ? p : 0.0f;
                                }
                            }
                        }
                    }
                }
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    sum[t] += __shfl_xor(sum[t], 32);
                    if constexpr (SPLIT > 1) {
                        if (g == 0) shared[wave][NT * n + t] = sum[t];
                    } else if (g == 0 && there && tok + t < longest) weights[tok + t] += sum[t];
                }
                if constexpr (SPLIT > 1) {
                    // (the next pass' columns wait for all waves, so nobody writes this while it is read)
                    static_assert(SPLIT == kBlock / 64, "all waves have the same tokens");
                    __syncthreads();
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        float all = shared[0][NT * n + t];
#pragma unroll
                        for (int i = 1; i < SPLIT; ++i) all += shared[i][NT * n + t];
                        if (tid < 32 && there && tok + t < longest) weights[tok + t] += all;
                    }
                }
            }
        }
}

// Many rows.  A window is the queries of some rows to one cache head, up to 256 columns
// (128 of heads of 256), which stay in LDS while tokens pass by: every wave has its own, in
// registers, and no wave waits for another.  A step is 256 tokens of a request; its sums over one
// window are a part, and a launch of its own joins the parts of a step in order.
//
// The steps that windows see, window by window, are laid out in one line and cut into equal shares,
// one to a resident workgroup: each loads queries twice or three times, however many there are.
// Where the parts would be more than the workspace holds, several windows make a piece
// that adds up in one part, and units of a piece and 8 steps are dealt to workgroups as these come free.

constexpr int kPlan = 512;
constexpr int kRange = 8;      // steps of a unit
constexpr int kParts = 49152;  // parts of a call: 50 MB

// Columns of a window.
constexpr int window_of(int dim) { return dim == 256 ? 128 : 256; }

struct Request {
    int64_t base;     // what is dealt out before its own: steps that windows see, or units
    int longest;      // of its rows
    int window_base;  // its windows of a head, before all heads
    int part_base;    // parts before its own: of each of its pieces, all steps
    int step_base;    // steps that lie in parts before its own
    int row0, row1;
};

struct Plan {
    Request *requests;  // [n + 1]
    int *counter;       // units taken
    int *size;          // windows of a piece
    int *window_max, *window_min;  // [max_windows] lengths of a window's rows
    int *window_steps;  // [max_windows] steps that the windows before it see, of its request
    float *parts;       // [kParts][kTile]
};

struct BlockArgs {
    WeighArgs a;
    int n, rows, parts;  // requests; rows of a window; windows of a row, where a head's queries are more than a window
    int max_windows;
    u32 per_inverse;  // 65536 / per, rounded up: a column's row without a division
    int skip_heads;   // from one column of a thread to its next: heads (of the row it comes to),
    int64_t skip, wrap;  // bytes of q, and bytes more where the head is past the row's last
    Plan p;
};

__device__ inline int steps_of(int len) { return (int)(((int64_t)len + kTile - 1) / kTile); }
__device__ inline int bounded(const WeighArgs &a, int r) { return min(max(a.row_starts[r], 0), a.n_rows); }

// Exclusive prefix of x over the workgroup; total in *sum.
__device__ int64_t prefix(int64_t x, int64_t *waves, int64_t *sum) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    int64_t s = x;
    for (int d = 1; d < 64; d <<= 1) {
        const int64_t y = __shfl_up(s, d);
        if (lane >= d) s += y;
    }
    __syncthreads();
    if (lane == 63) waves[w] = s;
    __syncthreads();
    int64_t before = 0, all = 0;
    for (int i = 0; i < kPlan / 64; ++i) {
        if (i == w) before = all;
        all += waves[i];
    }
    *sum = all;
    return before + s - x;
}

// Last i in [0, n) with base(i) <= x (base rises, base(0) <= x), the wave's lanes looking at 64 at once.
template <class F>
__device__ int last_base(int n, int64_t x, F base) {
    const int lane = threadIdx.x & 63;
    int lo = 0;
    while (n > 1) {
        const int step = (n + 63) / 64;
        const uint64_t m = __ballot(lane * step < n && base(lo + min(lane * step, n - 1)) <= x);
        const int at = (63 - __builtin_clzll(m)) * step;
        lo += at;
        n = min(step, n - at);
    }
    return __builtin_amdgcn_readfirstlane(lo);
}

__global__ __launch_bounds__(kPlan) void plan_kernel(BlockArgs b) {
    __shared__ int64_t waves[kPlan / 64];
    __shared__ int first[kPlan + 1], most_of[kPlan];  // of a round: windows before a request's, its longest row
    __shared__ unsigned long long seen_by[kPlan];     // steps that its windows see, then those of the requests before
    __shared__ int window_max[kPlan];                 // of a round's first windows
    const WeighArgs &a = b.a;
    const Plan &p = b.p;
    const int tid = threadIdx.x;
    const int64_t cap = (int64_t)a.table_width << a.lp;
    int64_t windows = 0, work = 0, all = 0;
    Request only = {};  // a request of the only round
    for (int r0 = 0; r0 < b.n; r0 += kPlan) {
        const int r = r0 + tid, here = min(kPlan, b.n - r0);
        int row0 = 0, row1 = 0;
        if (r < b.n) {
            row0 = bounded(a, r);
            row1 = max(bounded(a, r + 1), row0);
        }
        // (the kernel of few rows has taken the others)
        const int64_t mine = (int64_t)(row1 - row0) * a.heads <= a.limit ? 0
                             : b.parts > 1 ? (int64_t)(row1 - row0) * b.parts
                                           : (row1 - row0 + b.rows - 1) / b.rows;
        const int from = (int)min(windows + prefix(mine, waves, &all), (int64_t)b.max_windows);
        first[tid] = from;
        most_of[tid] = 0;
        seen_by[tid] = 0;
        windows = min(windows + all, (int64_t)b.max_windows);
        if (tid == 0) first[here] = (int)windows;  // (thread `here`, if there is one, writes the same)
        __syncthreads();
        // the lengths of a window's rows: 8 lanes to a window, 8 lengths of a lane at once
        constexpr int LANES = 8, AHEAD = 8;
        for (int w0 = first[0] + tid / LANES; w0 < (int)windows; w0 += kPlan / LANES) {
            int lo = 0, hi = here;
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (first[mid] <= w0) lo = mid; else hi = mid;
            }
            const int i = w0 - first[lo], start = bounded(a, r0 + lo), stop = bounded(a, r0 + lo + 1);
            const int at = start + (b.parts > 1 ? i / b.parts : i * b.rows);
            const int end = min(at + (b.parts > 1 ? 1 : b.rows), stop);
            int most = 0, least = 0x7FFFFFFF;
            for (int row0 = at + tid % LANES; row0 < end; row0 += LANES * AHEAD) {
                int len[AHEAD];
#pragma unroll
                for (int j = 0; j < AHEAD; ++j) len[j] = a.row_lengths[min(row0 + LANES * j, end - 1)];
#pragma unroll
                for (int j = 0; j < AHEAD; ++j) {
                    const int x = (int)min((int64_t)max(len[j], 0), cap);
                    most = max(most, x);
                    least = min(least, x);
                }
            }
            for (int d = LANES / 2; d; d >>= 1) {
                most = max(most, __shfl_xor(most, d));
                least = min(least, __shfl_xor(least, d));
            }
            if (tid % LANES == 0) {
                if (w0 - first[0] < kPlan) window_max[w0 - first[0]] = most;
                p.window_max[w0] = most;
                p.window_min[w0] = least;
                atomicMax(&most_of[lo], most);
                atomicAdd(&seen_by[lo], (unsigned long long)steps_of(most));
            }
        }
        __syncthreads();
        const int count = first[min(tid + 1, here)] - from;
        prefix(r < b.n ? (int64_t)steps_of(most_of[tid]) * count * a.kv_heads : 0, waves, &all);
        work += all;
        // (the second round puts in the bases: until then what it needs for them)
        only = {(int64_t)seen_by[tid], most_of[tid], from, count, 0, row0, row1};
        if (r < b.n && b.n > kPlan) p.requests[r] = only;
        __syncthreads();
        const unsigned long long before = prefix((int64_t)seen_by[tid], waves, &all);
        __syncthreads();
        seen_by[tid] = before;
        __syncthreads();
        // the steps that windows before a window see: a line over all requests of the round, less what is before its own
        int64_t line = 0;
        for (int w0 = first[0]; w0 < (int)windows; w0 += kPlan) {
            const int w = w0 + tid;
            int64_t steps = 0;
            if (w < (int)windows) steps = steps_of(w0 == first[0] ? window_max[tid] : p.window_max[w]);
            const int64_t at = line + prefix(steps, waves, &all);
            line += all;
            if (w < (int)windows) {
                int lo = 0, hi = here;
                while (hi - lo > 1) {
                    const int mid = (lo + hi) >> 1;
                    if (first[mid] <= w) lo = mid; else hi = mid;
                }
                p.window_steps[w] = (int)min(at - (int64_t)seen_by[lo], (int64_t)0x7FFFFFFF);
            }
        }
        __syncthreads();
    }
    // all parts fit: pieces of one window; else of so many that half of them would
    const int64_t size = work <= kParts ? 1 : (2 * work + kParts - 1) / kParts;
    int64_t dealt = 0, parts = 0, joined = 0;
    for (int r0 = 0; r0 < b.n; r0 += kPlan) {
        const int r = r0 + tid;
        Request q = {};
        int64_t mine = 0, in_parts = 0, steps = 0;
        if (r < b.n) {
            q = b.n > kPlan ? p.requests[r] : only;
            const int64_t pieces = ((int64_t)q.part_base * a.kv_heads + size - 1) / size;
            steps = steps_of(q.longest);
            mine = size == 1 ? q.base * a.kv_heads : pieces * ((steps + kRange - 1) / kRange);
            if (pieces > 1) in_parts = pieces * steps;
            else steps = 0;
        }
        q.base = dealt + prefix(mine, waves, &all);
        dealt += all;
        q.part_base = (int)(parts + prefix(in_parts, waves, &all));
        parts += all;
        q.step_base = (int)(joined + prefix(steps, waves, &all));
        joined += all;
        if (r < b.n) p.requests[r] = q;
    }
    if (tid == 0) {
        p.requests[b.n] = {dealt, 0, (int)windows, (int)parts, (int)joined, 0, 0};
        *p.size = (int)min(size, (int64_t)0x7FFFFFFF);
        *p.counter = 0;
    }
}

template <int D>
struct Window {
    alignas(16) float lse2[window_of(D)], fine[window_of(D)];  // first: their offsets fit the instructions that load them
    alignas(16) int len[window_of(D)];
    alignas(16) uint8_t q[window_of(D)][2 * D + 16];
};

// The softmaxes of 32 columns: place i of half g is column 8 (i / 4) + 4 g + i % 4.
struct Softmaxes {
    f32x4 l[4], f[4];
    template <int D>
    __device__ void load(const Window<D> &o, int col0) {
        const int g = (threadIdx.x & 63) >> 5;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            l[i] = *(const f32x4 *)&o.lse2[col0 + 8 * i + 4 * g];
            f[i] = *(const f32x4 *)&o.fine[col0 + 8 * i + 4 * g];
        }
    }
    __device__ void add(const f32x16 &y, float scale, float &sum) const {
#pragma unroll
        for (int i = 0; i < 16; ++i) sum = fmaf(exp2_(fmaf(y[i], scale, -l[i / 4][i % 4])), f[i / 4][i % 4], sum);
    }
};

__device__ inline f32x16 zero16() {
    f32x16 y;
#pragma unroll
    for (int i = 0; i < 16; ++i) y[i] = 0.0f;
    return y;
}

// The products of 32 columns with the wave's 64 tokens, in two phases of eight groups: phase 0 makes
// those with its second 32 tokens beside the exponentials of the first, phase 1 those of the next 32
// columns with the first ones beside the exponentials of the second.  The order is written down, since the
// compiler would put the products first and the vector work behind them: a group holds one matrix
// instruction, and as much vector work as takes its time, on results that no instruction in flight still
// writes.  Result i of a phase is scaled in group at(i), raised in the next and added in the one after, which for
// the last ones is in the phase that follows.  A softmax is loaded as soon as its place is free.
template <int D, class T>
struct Pass {
    typedef typename Act<T>::frag frag;
    static constexpr int N = D / 16;  // matrix instructions of a product
    const Window<D> &o;
    const frag (&k)[kTokens][N];
    const uint8_t *q;
    const float *soft;
    float scale, sum[2], t[16], e[16];
    frag x[N];
    f32x16 y[2];
    f32x4 l[4], f[4];

    static constexpr int at(int i) { return i < 3 ? 1 : i >= 13 ? 7 : (i + 1) / 2; }

    __device__ Pass(const Window<D> &o, const frag (&k)[kTokens][N], float scale) : o(o), k(k), scale(scale) {
        const int lane = threadIdx.x & 63;
        q = o.q[lane & 31] + 32 * (lane >> 5);
        soft = o.lse2 + 4 * (lane >> 5);
#pragma unroll
        for (int j = 0; j < N; ++j) x[j] = query(0, j);
        y[0] = zero16();
#pragma unroll
        for (int j = 0; j < N; ++j) y[0] = Act<T>::mfma32(x[j], k[0][j], y[0]);
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            l[v] = lse2(0, v);
            f[v] = fine(0, v);
        }
        sum[0] = sum[1] = 0.0f;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            t[i] = -__builtin_inff();
            e[i] = 0.0f;
        }
        __builtin_amdgcn_sched_barrier(0);
    }
    __device__ frag query(int col0, int j) const {
        return __builtin_bit_cast(frag, *(const u32x4 *)(q + col0 * (2 * D + 16) + 64 * (j >> 1) + 16 * (j & 1)));
    }
    // place i of half g is column 8 (i / 4) + 4 g + i % 4
    __device__ f32x4 lse2(int col0, int v) const { return *(const f32x4 *)(soft + col0 + 8 * v); }
    __device__ f32x4 fine(int col0, int v) const { return *(const f32x4 *)(soft + window_of(D) + col0 + 8 * v); }

    // The vector work of a phase's group.
    __device__ void work(int phase, int g) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            if (at(i) + 2 == g) sum[phase] = fmaf(e[i], f[i / 4][i % 4], sum[phase]);
            if (at(i) - 6 == g) sum[phase ^ 1] = fmaf(e[i], f[i / 4][i % 4], sum[phase ^ 1]);
        }
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (at(i) + 1 == g || at(i) - 7 == g) e[i] = exp2_(t[i]);
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (at(i) == g) t[i] = fmaf(y[phase][i], scale, -l[i / 4][i % 4]);
    }
    // 32 columns from col0 on; `next` follow, if MORE.
    template <bool MORE>
    __device__ void columns(int col0, int next) {
#pragma unroll
        for (int g = 0; g < 8; ++g) {
            if (g % (8 / (N < 8 ? N : 8)) == 0) {
                constexpr int EACH = N > 8 ? N / 8 : 1;
#pragma unroll
                for (int h = 0; h < EACH; ++h) {
                    const int j = g / (8 / (N < 8 ? N : 8)) * EACH + h;
                    y[1] = Act<T>::mfma32(x[j], k[1][j], j == 0 ? zero16() : y[1]);
                    if (MORE) x[j] = query(next, j);
                }
            }
            work(0, g);
            // what the columns before have left their places to
            if (g == 0) l[3] = lse2(col0, 3);
            if (g == 1) f[2] = fine(col0, 2);
            if (g == 2) f[3] = fine(col0, 3);
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int g = 0; g < 8; ++g) {
            if (MORE && g % (8 / (N < 8 ? N : 8)) == 0) {
                constexpr int EACH = N > 8 ? N / 8 : 1;
#pragma unroll
                for (int h = 0; h < EACH; ++h) {
                    const int j = g / (8 / (N < 8 ? N : 8)) * EACH + h;
                    y[0] = Act<T>::mfma32(x[j], k[0][j], j == 0 ? zero16() : y[0]);
                }
            }
            work(1, g);
            if (MORE) {
                if (g == 3) l[0] = lse2(next, 0);
                if (g == 5) {
                    f[0] = fine(next, 0);
                    l[1] = lse2(next, 1);
                }
                if (g == 7) {
                    f[1] = fine(next, 1);
                    l[2] = lse2(next, 2);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    // What the last phase has left.
    __device__ void finish() {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            if (at(i) == 7) e[i] = exp2_(t[i]);
            if (at(i) >= 6) sum[1] = fmaf(e[i], f[i / 4][i % 4], sum[1]);
        }
    }
};

// A window of `cols` columns (a multiple of 32), every row of which sees all of the wave's tokens.
template <int D, class T>
__device__ inline void pass(const Window<D> &o, int cols, const typename Act<T>::frag (&k)[kTokens][D / 16], float scale,
                            float (&sum)[kTokens]) {
    static_assert(kTokens == 2, "two products for 32 columns");
    if constexpr (D == 256) {
        // (the keys take half of the registers: nothing runs ahead)
        const int lane = threadIdx.x & 63;
#pragma unroll 1
        for (int c0 = 0; c0 < cols; c0 += 32) {
            f32x16 y[kTokens] = {zero16(), zero16()};
            const uint8_t *q = o.q[c0 + (lane & 31)] + 32 * (lane >> 5);
#pragma unroll
            for (int j = 0; j < D / 16; ++j) {
                const auto x = __builtin_bit_cast(typename Act<T>::frag, *(const u32x4 *)(q + 64 * (j >> 1) + 16 * (j & 1)));
#pragma unroll
                for (int t = 0; t < kTokens; ++t) y[t] = Act<T>::mfma32(x, k[t][j], y[t]);
            }
            Softmaxes c;
            c.load(o, c0);
#pragma unroll
            for (int t = 0; t < kTokens; ++t) c.add(y[t], scale, sum[t]);
        }
    } else {
        Pass<D, T> p(o, k, scale);
#pragma unroll 1
        for (int c0 = 0; c0 < cols - 32; c0 += 32) p.template columns<true>(c0, c0 + 32);
        p.template columns<false>(cols - 32, 0);
        p.finish();
#pragma unroll
        for (int t = 0; t < kTokens; ++t) sum[t] += p.sum[t];
    }
}

// Any window, rows that see a part of the tokens among them.
template <int D, class T>
__device__ inline void pass_masked(const Window<D> &o, int cols, const typename Act<T>::frag (&k)[kTokens][D / 16],
                                   float scale, float (&sum)[kTokens], int tok) {
    const int lane = threadIdx.x & 63, g = lane >> 5;
#pragma unroll 1
    for (int c0 = 0; c0 < cols; c0 += 32) {
        const uint8_t *q = o.q[c0 + (lane & 31)] + 32 * g;
        f32x16 y[kTokens];
#pragma unroll
        for (int t = 0; t < kTokens; ++t) y[t] = zero16();
#pragma unroll
        for (int j = 0; j < D / 16; ++j) {
            const auto x = __builtin_bit_cast(typename Act<T>::frag, *(const u32x4 *)(q + 64 * (j >> 1) + 16 * (j & 1)));
#pragma unroll
            for (int t = 0; t < kTokens; ++t) y[t] = Act<T>::mfma32(x, k[t][j], y[t]);
        }
        Softmaxes c;
        c.load(o, c0);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int len = o.len[c0 + 8 * (i / 4) + 4 * g + i % 4];
#pragma unroll
            for (int t = 0; t < kTokens; ++t) {
                const float p = exp2_(fmaf(y[t][i], scale, -c.l[i / 4][i % 4])) * c.f[i / 4][i % 4];
                sum[t] += tok + t < len ? p : 0.0f;
            }
        }
    }
}

template <int D, class T, class C>
__global__ __launch_bounds__(kBlock, 2) void weigh_block_kernel(BlockArgs b) {
    constexpr int NT = kTokens, PER = D / 8;  // 16-byte pieces of a column
    typedef typename Act<T>::frag frag;
    __shared__ Window<D> o;
    __shared__ int taken, empty[kBlock / 64];
    const WeighArgs &a = b.a;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 31, g = lane >> 5;
    const int64_t cap = (int64_t)a.table_width << a.lp;
    const int size = *b.p.size, window_heads = (a.per + b.parts - 1) / b.parts;
    const int64_t total = b.p.requests[b.n].base;

    // In equal shares, neighbouring ones, which read the same keys, on one XCD (workgroups go round them).
    const int eighth = gridDim.x / 8, i8 = blockIdx.x;
    const int share = i8 < 8 * eighth ? (i8 % 8) * eighth + i8 / 8 : i8;
    // (then units are no more than kParts: 32 bits hold all of this)
    int64_t next = size == 1 ? (u32)total * (u32)share / gridDim.x : 0;
    const int64_t stop = size == 1 ? (u32)total * (u32)(share + 1) / gridDim.x : 0;
    int ahead = 0;
    if (size > 1 && tid == 0) ahead = atomicAdd(b.p.counter, 1);
    for (;;) {
        // the request, its windows [from, to), counted head by head, and steps [s0, s1)
        if (size > 1) {
            __syncthreads();
            if (tid == 0) taken = ahead;
            __syncthreads();
            next = __builtin_amdgcn_readfirstlane(taken);
            if (next >= total) return;
            if (tid == 0) ahead = atomicAdd(b.p.counter, 1);
        } else if (next >= stop) {
            return;
        }
        const int r = last_base(b.n, next, [&](int i) { return b.p.requests[i].base; });
        const Request q = b.p.requests[r];
        const int windows = b.p.requests[r + 1].window_base - q.window_base, steps = steps_of(q.longest);
        int64_t from, to;
        int s0, s1, piece;
        if (size == 1) {
            const u32 of_head = (u32)(b.p.requests[r + 1].base - q.base) / (u32)a.kv_heads;  // steps that its windows see
            const int head = (int)((u32)(next - q.base) / of_head), line = (int)((u32)(next - q.base) - head * of_head);
            const int *before = b.p.window_steps + q.window_base;
            const int w = last_base(windows, line, [&](int i) { return (int64_t)before[i]; });
            s0 = line - before[w];
            s1 = (int)min((int64_t)steps_of(b.p.window_max[q.window_base + w]), s0 + (stop - next));
            from = (int64_t)head * windows + w;
            to = from + 1;
            piece = (int)from;
            next += s1 - s0;
        } else {
            const int ranges = (steps + kRange - 1) / kRange, i = (int)(next - q.base);
            piece = i / ranges;
            s0 = (i - piece * ranges) * kRange;
            s1 = min(s0 + kRange, steps);
            from = (int64_t)piece * size;
            to = min(from + size, (int64_t)windows * a.kv_heads);
        }
        const int64_t all = (int64_t)windows * a.kv_heads;
        const int *pages = a.table + (int64_t)r * a.table_stride;
        const auto token = [&](int s) { return s * kTile + 32 * NT * wave + NT * n; };  // this lane's first one
        const auto page_of = [&](int s) { return pages[min((int64_t)token(min(s, s1 - 1)), cap - 1) >> a.lp]; };
        const auto in_cache = [&](int pg) { return pg >= 0 && pg < a.n_pages; };
        const int page = page_of(s0);
        int head = (int)(from / windows), w = (int)(from - (int64_t)head * windows) - 1;
        for (int64_t at = from; at < to; ++at) {
            if (++w == windows) {
                w = 0;
                ++head;
            }
            const int most = b.p.window_max[q.window_base + w], least = b.p.window_min[q.window_base + w];
            const int width = b.parts > 1 ? min(window_heads, a.per - w % b.parts * window_heads)
                                          : min(b.rows, q.row1 - q.row0 - w * b.rows) * a.per;
            const int cols = (width + 31) & ~31, row0 = q.row0 + (b.parts > 1 ? w / b.parts : w * b.rows);
            const int head0 = head * a.per + (b.parts > 1 ? w % b.parts * window_heads : 0);
            const bool sees = most > s0 * kTile && width > 0;
            const int end = sees ? min(s1, steps_of(most)) : s0;
            if (sees) {
                // Queries are asked for before the wait for the window before.  This thread's: piece
                // `part` of columns first, first + STRIDE, ..  (Their addresses go on by constants: a
                // product of 64 bits each would cost as much as eight exponentials.)
                constexpr int STRIDE = kBlock / PER, ROUNDS = window_of(D) / STRIDE, BATCH = 8;
                const int first = tid / PER, part = tid % PER;
                const auto row_of = [&](int col) { return b.parts > 1 ? 0 : (int)((u32)col * b.per_inverse >> 16); };
                const int row1 = row_of(first);
                int in_row = first - row1 * a.per, col = first;
                const char *from_q = (const char *)a.q + 2 * ((row0 + row1) * a.q_row + (head0 + in_row) * a.q_head + 8 * part);
                u32x4 x[BATCH];
                const auto ask = [&] {
#pragma unroll
                    for (int i = 0; i < BATCH; ++i) {
                        x[i] = *(const u32x4 *)(col < width ? from_q : (const char *)a.q);
                        col += STRIDE;
                        in_row += b.skip_heads;
                        from_q += b.skip;
                        if (in_row >= a.per && b.parts == 1) {
                            in_row -= a.per;
                            from_q += b.wrap;
                        }
                    }
                };
                ask();
                Softmax mine = {__builtin_inff(), 0.0f};
                int len = 0;
                if (tid < width) {
                    const int row = row_of(tid), h = head0 + tid - row * a.per;
                    mine = softmax_of(a.lse[(int64_t)(row0 + row) * a.heads + h], a.stretch);
                    len = (int)min((int64_t)max(a.row_lengths[row0 + row], 0), cap);
                }
                // A column without a softmax sees nothing: a key that is NaN would make its product NaN, 0 or not.
                // (The columns past the window's are not masked for it: such a key makes the others' sum NaN, too.)
                const bool none = tid < width && mine.lse2 == __builtin_inff(), any = __any(none);
                if (none) len = 0;
                __syncthreads();  // the window before is done with
                if (lane == 0) empty[wave] = any;
                if (tid < window_of(D)) {
                    o.lse2[tid] = mine.lse2;
                    o.fine[tid] = mine.fine;
                    o.len[tid] = len;
                }
                __syncthreads();
#pragma unroll 1
                for (int i0 = 0; i0 < ROUNDS; i0 += BATCH) {
                    if (i0 > 0) ask();
#pragma unroll
                    for (int i = 0; i < BATCH; ++i) {
                        const int c = first + (i0 + i) * STRIDE;
                        // (columns past the window's; and what a row without a softmax holds is not looked at)
                        *(u32x4 *)&o.q[c][16 * part] = o.fine[c] == 0.0f ? u32x4{0, 0, 0, 0} : x[i];
                    }
                    if ((i0 + BATCH) * STRIDE >= cols) break;
                }
            }
            u32x4 raw[NT][D / 32];
            float raw_scale;
            const auto fetch = [&](int s, int pg) {
                const u32 page = in_cache(pg) ? pg : 0;
                const u32 row = page * a.page_rows + (u32)(head << a.lp) + (u32)(token(s) & ((1 << a.lp) - 1));
                const uint8_t *p = a.k + (uint64_t)row * D + 16 * g;
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int j = 0; j < D / 32; ++j) raw[t][j] = *(const u32x4 *)(p + t * D + 32 * j);
                raw_scale = a.ks[page * a.scale_stride + head];
            };
            int next_page = page, seen_by_all = least;
            if (sees) {
                fetch(s0, page);
                next_page = page_of(s0 + 1);
                __syncthreads();
                for (int i = 0; i < kBlock / 64; ++i) seen_by_all = empty[i] ? 0 : seen_by_all;
                seen_by_all = __builtin_amdgcn_readfirstlane(seen_by_all);
            }
#pragma unroll 1
            for (int s = s0; s < end; ++s) {
                const int base = s * kTile + 32 * NT * wave, tok = base + NT * n;
                float sum[NT] = {0.0f, 0.0f};
                frag k[NT][D / 16];
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int j = 0; j < D / 32; ++j) {
                        k[t][2 * j] = eight<C, T>(raw[t][j][0], raw[t][j][1]);
                        k[t][2 * j + 1] = eight<C, T>(raw[t][j][2], raw[t][j][3]);
                    }
                const float scale = raw_scale * a.scale2;
                // the next step's codes are on their way beside the products (but for heads of 256,
                // whose keys take half of the registers); after the last step the last ones again
                if (D < 256) {
                    fetch(min(s + 1, end - 1), next_page);
                    next_page = page_of(s + 2);
                }
                if (base + 32 * NT <= seen_by_all) pass<D, T>(o, cols, k, scale, sum);
                else if (base < most) pass_masked<D, T>(o, cols, k, scale, sum, tok);
                if (D == 256) {
                    fetch(min(s + 1, end - 1), next_page);
                    next_page = page_of(s + 2);
                }
#pragma unroll
                for (int t = 0; t < NT; ++t) sum[t] += __shfl_xor(sum[t], 32);
                if (g == 0) {
                    if (all > size) {
                        f32x2 *to = (f32x2 *)(b.p.parts + ((int64_t)q.part_base + (int64_t)piece * steps_of(q.longest) + s) * kTile +
                                              (tok - s * kTile));
                        f32x2 y = {sum[0], sum[1]};
                        if (at > from) y += *to;  // (this workgroup's own, of the window before)
                        *to = y;
                    } else if (tok < most && in_cache(page_of(s))) {
                        float *to = a.weights + a.weight_offsets[r] + tok;
                        to[0] += sum[0];
                        if (tok + 1 < most) to[1] += sum[1];
                    }
                }
            }
            // a piece of several windows begins with all of its steps
            if (size > 1 && all > size && at == from && g == 0)
                for (int s = end; s < s1; ++s)
                    *(f32x2 *)(b.p.parts + ((int64_t)q.part_base + (int64_t)piece * steps_of(q.longest) + s) * kTile +
                               (token(s) - s * kTile)) = f32x2{0.0f, 0.0f};
        }
    }
}

// Steps whose sums lie in parts: 64 tokens of one to a workgroup, its parts over 16 groups of threads.
__global__ __launch_bounds__(1024) void join_kernel(BlockArgs b) {
    constexpr int GROUPS = 16, AHEAD = 12;
    __shared__ float sums[GROUPS][64];
    const WeighArgs &a = b.a;
    const int lane = threadIdx.x & 63, group = threadIdx.x >> 6;
    const int total = b.p.requests[b.n].step_base, size = *b.p.size;
    for (int64_t i = blockIdx.x; i < (int64_t)total * (kTile / 64); i += gridDim.x) {
        const int at = (int)(i / (kTile / 64));
        const int r = last_base(b.n, at, [&](int j) { return (int64_t)b.p.requests[j].step_base; });
        const Request q = b.p.requests[r], next = b.p.requests[r + 1];
        const int step = at - q.step_base, steps = next.step_base - q.step_base, windows = next.window_base - q.window_base;
        const int pieces = (next.part_base - q.part_base) / steps, in = (int)(i % (kTile / 64)) * 64 + lane;
        const int tok = step * kTile + in;
        const float *parts = b.p.parts + ((int64_t)q.part_base + step) * kTile + in;
        float sum = 0.0f, old = 0.0f, *to = nullptr;
        if (group == 0 && tok < q.longest) {
            const int pg = a.table[(int64_t)r * a.table_stride + (tok >> a.lp)];
            to = a.weights + a.weight_offsets[r] + tok;
            old = *to;
            if (pg < 0 || pg >= a.n_pages) to = nullptr;
        }
        for (int p0 = group; p0 < pieces; p0 += AHEAD * GROUPS) {
            float x[AHEAD];
            int most[AHEAD];
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) {
                const int p = min(p0 + j * GROUPS, pieces - 1);
                x[j] = parts[(int64_t)p * steps * kTile];
                most[j] = b.p.window_max[q.window_base + p % windows];
            }
            // (a piece of one window has no parts of steps that it does not see: what lies there is anything)
#pragma unroll
            for (int j = 0; j < AHEAD; ++j)
                sum += p0 + j * GROUPS < pieces && (size > 1 || most[j] > step * kTile) ? x[j] : 0.0f;
        }
        sums[group][lane] = sum;
        __syncthreads();
        if (to) {
#pragma unroll
            for (int j = 1; j < GROUPS; ++j) sum += sums[j][lane];
            *to = old + sum;
        }
        __syncthreads();
    }
}

// A call's division into windows, and the workspace's.
struct Sizes {
    int rows, parts;
    int64_t max_windows;
    size_t bytes;
};
Sizes sizes_of(int64_t n_rows, int64_t n_requests, int per, int cols) {
    Sizes s;
    s.parts = (per + cols - 1) / cols;
    s.rows = s.parts > 1 ? 1 : cols / per;
    s.max_windows = s.parts > 1 ? n_rows * s.parts : n_rows / s.rows + n_requests;
    s.bytes = 256 + sizeof(Request) * (size_t)(n_requests + 1) + 12 * (size_t)s.max_windows +
              (size_t)kParts * kTile * sizeof(float);
    return s;
}

// Requests of up to so many rows x heads read the cache by themselves, without queries in windows (64 of 16384
// tokens, 16 heads: 8 rows each 96 us, and 180 in windows; 16 rows 169 and 203; one of 131072 tokens, 32 heads:
// 8 rows 40 and 52, 16 rows 66 and 57), where tokens make workgroups enough (four requests of up to 2635 tokens, 16
// heads, 7 to 68 rows: 52 us, and 27 with all in windows).  This and the rules of launch_types() go by the tokens that
// the table has room for, since the host knows no lengths; they were measured with tables as wide as the longest
// request.  Under one of 131072 tokens 4 rows of up to 3392 tokens take 48 us for 7.5, 64 rows of 2000 260 us for 26.
constexpr int kFew = 256;
inline int64_t tiles_of(int64_t cap, int n_requests) { return (cap + kTile - 1) / kTile * n_requests; }

// Whether a call may have others.  (Where rows are no more than requests, as single tokens are, none is looked
// for: the plan would cost as much as a short call.)
inline bool many(int n_rows, int n_requests, int heads) { return n_rows > n_requests && (int64_t)n_rows * heads > kFew; }

template <int D, class T, class C>
int launch_types(BlockArgs &b, bool block, int n_requests, void *stream) {
    WeighArgs &a = b.a;
    const int64_t cap = (int64_t)a.table_width << a.lp;
    while (a.steps < 4 && cap / (2 * a.steps * kTile) * n_requests >= 1024) a.steps *= 2;
    // Where workgroups are fewer than half of the CUs, the heads over four times as many waves (one row of
    // 31 tokens, 128 heads: 17 us, and 26 without; 52 rows of up to 162 tokens, 32 heads: 8.9 and 13.9; but 29 of 1874
    // tokens, 64 heads, 232 workgroups: 17.8 and 14.5).
    const bool split = a.kv_heads > 1 && tiles_of(cap, n_requests) <= 128;
    const int64_t tokens = split ? kTile / 4 : (int64_t)kTile * a.steps;
    const dim3 grid((unsigned)((cap + tokens - 1) / tokens), (unsigned)n_requests);
    int rc = PAGED_KV_OK;
    if (a.limit > 0)
        rc = split ? launch(weigh_rows_kernel<D, T, C, 4>, grid, dim3(kBlock), stream, a)
                   : launch(weigh_rows_kernel<D, T, C, 1>, grid, dim3(kBlock), stream, a);
    if (rc != PAGED_KV_OK || !block) return rc;
    return launch(weigh_block_kernel<D, T, C>, dim3((unsigned)device_cus() * 2), dim3(kBlock), stream, b);
}

template <int D>
int launch_dim(BlockArgs &b, int act, int code, bool block, int n, void *stream) {
    if (code == PAGED_KV_E4M3)
        return act == PAGED_KV_BF16 ? launch_types<D, bf16, E4M3>(b, block, n, stream) : launch_types<D, f16, E4M3>(b, block, n, stream);
    return act == PAGED_KV_BF16 ? launch_types<D, bf16, Int8>(b, block, n, stream) : launch_types<D, f16, Int8>(b, block, n, stream);
}

}  // namespace
}  // namespace paged

extern "C" size_t serve_weigh_workspace(int32_t n_rows, int32_t n_requests, int32_t heads, int32_t kv_heads) {
    using namespace paged;
    if (n_rows < 0 || n_requests < 0 || heads < 1 || kv_heads < 1 || heads % kv_heads != 0) return 0;
    if (device_cus() == 0) return 0;
    // (the smaller windows of heads of 256 are more)
    return many(n_rows, n_requests, heads) ? sizes_of(n_rows, n_requests, heads / kv_heads, window_of(256)).bytes : 256;
}

extern "C" int serve_weigh(const paged_kv_cache *cache, int32_t act, const void *q, int64_t q_row, int64_t q_head,
                           int32_t heads, const float *lse, const int32_t *table, int32_t table_stride,
                           int32_t table_width, const int32_t *row_starts, int32_t n_requests,
                           const int32_t *row_lengths, int32_t n_rows, float scale, float *weights,
                           const int64_t *weight_offsets, void *workspace, size_t workspace_bytes, void *stream) {
    using namespace paged;
    int rc = check_cache(cache, false);
    if (rc != PAGED_KV_OK) return rc;
    if ((act != PAGED_KV_BF16 && act != PAGED_KV_F16) || n_rows < 0 || n_requests < 0 || heads < 1 ||
        heads % cache->n_heads != 0 || table_width < 1 || table_stride < table_width || !(scale >= 0.0f) ||
        scale - scale != 0.0f)
        return PAGED_KV_EINVAL;
    // (products are scaled by scale * log2(e))
    if ((double)scale * 1.4426950408889634 > FLT_MAX) return PAGED_KV_EUNSUPPORTED;
    if (n_rows == 0 || n_requests == 0) return PAGED_KV_OK;
    const bool block = many(n_rows, n_requests, heads);
    if (!q || !lse || !table || !row_starts || !row_lengths || !weights || !weight_offsets || !aligned16(q) ||
        q_row % 8 || q_head % 8 || (block && !workspace) || (uintptr_t)workspace % 256)
        return PAGED_KV_EINVAL;
    const int lp = log2_page(cache->page);
    if (((int64_t)table_width << lp) > 0x7FFFFFFF - 65536 || n_requests > 65535) return PAGED_KV_EUNSUPPORTED;
    const size_t need = serve_weigh_workspace(n_rows, n_requests, heads, cache->n_heads);
    if (need == 0) return PAGED_KV_EUNSUPPORTED;
    if (block && workspace_bytes < need) return PAGED_KV_EWORKSPACE;
    const int64_t cap = (int64_t)table_width << lp;
    const double exact = (double)scale * 1.4426950408889634;
    const float scale2 = (float)exact;
    // (a scale below the normal numbers has few bits: what its rounding leaves is then no small part of lse, and scores
    // are far too small for it to matter)
    const float stretch = scale2 >= FLT_MIN ? (float)(exact / scale2 - 1.0) : 0.0f;
    BlockArgs b = {};
    b.a = {(const uint8_t *)cache->k, cache->k_scale, cache->page_stride, cache->scale_stride, cache->n_pages,
           lp, cache->n_heads, q, q_row, q_head, heads, heads / cache->n_heads, lse, table, table_stride,
           table_width, row_starts, row_lengths, n_rows, 1, !block ? INT64_MAX : tiles_of(cap, n_requests) >= 512 ? kFew : 0,
           (u32)(cache->page_stride / cache->head_dim), scale2, stretch,
           weights, weight_offsets};
    if (block) {
        const Sizes s = sizes_of(n_rows, n_requests, b.a.per, window_of(cache->head_dim));
        if (s.max_windows > 0x7FFFFFF0) return PAGED_KV_EUNSUPPORTED;
        b.n = n_requests;
        b.rows = s.rows;
        b.parts = s.parts;
        b.max_windows = (int)s.max_windows;
        b.per_inverse = 65536u / b.a.per + 1;
        const int stride = kBlock / (cache->head_dim / 8), rows = s.parts > 1 ? 0 : stride / b.a.per;
        b.skip_heads = stride - rows * b.a.per;
        b.skip = 2 * (rows * q_row + b.skip_heads * q_head);
        b.wrap = 2 * (q_row - b.a.per * q_head);
        char *at = (char *)workspace;
        const auto take = [&](size_t bytes) {
            char *p = at;
            at += bytes;
            return p;
        };
        b.p.parts = (float *)take((size_t)kParts * kTile * sizeof(float));
        b.p.counter = (int *)take(128);
        b.p.size = (int *)take(128);
        b.p.requests = (Request *)take(sizeof(Request) * (size_t)(n_requests + 1));
        b.p.window_max = (int *)take(4 * (size_t)s.max_windows);
        b.p.window_min = (int *)take(4 * (size_t)s.max_windows);
        b.p.window_steps = (int *)take(4 * (size_t)s.max_windows);
        rc = launch(plan_kernel, dim3(1), dim3(kPlan), stream, b);
        if (rc != PAGED_KV_OK) return rc;
    }
    rc = cache->head_dim == 64    ? launch_dim<64>(b, act, cache->code, block, n_requests, stream)
         : cache->head_dim == 128 ? launch_dim<128>(b, act, cache->code, block, n_requests, stream)
                                  : launch_dim<256>(b, act, cache->code, block, n_requests, stream);
    if (rc == PAGED_KV_OK && block) rc = launch(join_kernel, dim3(512), dim3(1024), stream, b);
    return rc;
}
