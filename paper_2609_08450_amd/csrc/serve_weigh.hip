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
    return {hi, exp2_(fmaf(hi, stretch, -rest))};
}

// Query columns in LDS.
constexpr int columns_of(int dim) { return dim == 256 ? 64 : 128; }

template <int D>
struct Columns {
    alignas(16) uint8_t q[columns_of(D)][2 * D + 16];
    alignas(16) float lse2[columns_of(D) + 32], fine[columns_of(D) + 32];
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
                Softmax x = {__builtin_inff(), 0.0f};
                int len = 0;
                if (i < heads * cols) {
                    const int h = i / cols;
                    const int64_t col = col0 + i - h * cols;
                    const int row = row0 + (int)(col / a.per);
                    x = softmax_of(a.lse[(int64_t)row * a.heads + (head0 + h) * a.per + (int)(col % a.per)], a.stretch);
                    len = (int)min((int64_t)max(a.row_lengths[row], 0), cap);
                }
                b.lse2[i] = x.lse2;
                b.fine[i] = x.fine;
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
                                const float l = b.lse2[at + col], f = b.fine[at + col];
                                const int len = masked ? b.len[at + col] : 0x7FFFFFFF;
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
                    if (g == 0 && there && tok + t < longest) weights[tok + t] += sum[t];
                }
            }
        }
}

// Many rows.  A chunk is the queries of some rows to one cache head, up to 64 columns; a
// request's tiles of tokens each meet its heads' chunks, counted head by head.  A unit is a tile
// with a piece of up to `size` of these; a tile in several pieces has a part of its sums from
// each, which a launch of its own joins in order.  Units of one piece follow each other: what
// runs at a time reads the same queries.

constexpr int kPlan = 1024;
constexpr int kChunk = 64;
constexpr int kUnits = 9216;  // about so many units to a call: 12 to a resident workgroup
constexpr int kLeast = 8;     // chunks of a unit, where there are so many

struct Plan {
    int64_t *unit_base;  // [n + 1] prefix sum of the requests' units
    int *counter;        // units taken
    int *size;           // chunks of a unit
    int *slot_base;      // [n + 1] of the parts
    int *tile_base;      // [n + 1] of the tiles that lie in parts
    int *chunk_base;     // [n + 1] of the chunks of a head
    int *longest;        // [n]
    int *chunk_max, *chunk_min;  // [max_chunks] lengths of a chunk's rows
    float *parts;        // [2 * kUnits][kTile]
};

struct BlockArgs {
    WeighArgs a;
    int n, rows, parts;  // requests; rows of a chunk; chunks of a row, where a head's queries are more than a chunk
    int max_chunks;
    Plan p;
};

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

// Last i in [0, n) with base[i] <= x (base rises, base[0] <= x).
template <class I>
__device__ int last_base(const I *base, int n, int64_t x) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (base[mid] <= x) lo = mid; else hi = mid;
    }
    return lo;
}

__global__ __launch_bounds__(kPlan) void plan_kernel(BlockArgs b) {
    __shared__ int64_t waves[kPlan / 64];
    const WeighArgs &a = b.a;
    const Plan &p = b.p;
    const int tid = threadIdx.x;
    const int64_t cap = (int64_t)a.table_width << a.lp;
    int64_t base = 0, all = 0;
    for (int r0 = 0; r0 < b.n; r0 += kPlan) {
        const int r = r0 + tid;
        int64_t chunks = 0;
        if (r < b.n) {
            const int rows = max(bounded(a, r + 1) - bounded(a, r), 0);
            chunks = b.parts > 1 ? (int64_t)rows * b.parts : (rows + b.rows - 1) / b.rows;
            p.longest[r] = 0;
        }
        const int64_t at = min(base + prefix(chunks, waves, &all), (int64_t)b.max_chunks);
        if (r < b.n) p.chunk_base[r] = (int)at;
        base += all;
    }
    const int chunks = (int)min(base, (int64_t)b.max_chunks);
    if (tid == 0) p.chunk_base[b.n] = chunks;
    __syncthreads();
    for (int c = tid; c < chunks; c += kPlan) {
        const int r = last_base(p.chunk_base, b.n, c), i = c - p.chunk_base[r];
        const int from = bounded(a, r) + (b.parts > 1 ? i / b.parts : i * b.rows);
        const int to = min(from + (b.parts > 1 ? 1 : b.rows), bounded(a, r + 1));
        int most = 0, least = 0x7FFFFFFF;
        for (int row = from; row < to; row += 8) {
            int len[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) len[j] = a.row_lengths[min(row + j, to - 1)];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                most = max(most, len[j]);
                least = min(least, max(len[j], 0));
            }
        }
        most = (int)min((int64_t)most, cap);
        least = (int)min((int64_t)least, cap);
        p.chunk_max[c] = most;
        p.chunk_min[c] = least;
        atomicMax(&p.longest[r], most);
    }
    __syncthreads();
    const auto tiles_of = [&](int r) { return ((int64_t)p.longest[r] + kTile - 1) / kTile; };
    const auto chunks_of = [&](int r) { return (int64_t)(p.chunk_base[r + 1] - p.chunk_base[r]) * a.kv_heads; };
    int64_t work = 0;
    for (int r0 = 0; r0 < b.n; r0 += kPlan) {
        const int r = r0 + tid;
        prefix(r < b.n ? tiles_of(r) * chunks_of(r) : 0, waves, &all);
        work += all;
    }
    const int64_t size = max((work + kUnits - 1) / kUnits, (int64_t)kLeast);
    int64_t units = 0, slots = 0, tiles = 0;
    for (int r0 = 0; r0 < b.n; r0 += kPlan) {
        const int r = r0 + tid;
        int64_t mine = 0, pieces = 0;
        if (r < b.n) {
            pieces = (chunks_of(r) + size - 1) / size;
            mine = tiles_of(r) * pieces;
        }
        const int64_t at = units + prefix(mine, waves, &all);
        units += all;
        const int64_t slot = slots + prefix(pieces > 1 ? mine : 0, waves, &all);
        slots += all;
        const int64_t tile = tiles + prefix(pieces > 1 ? tiles_of(r) : 0, waves, &all);
        tiles += all;
        if (r < b.n) {
            p.unit_base[r] = at;
            p.slot_base[r] = (int)slot;
            p.tile_base[r] = (int)tile;
        }
    }
    if (tid == 0) {
        p.unit_base[b.n] = units;
        p.slot_base[b.n] = (int)slots;
        p.tile_base[b.n] = (int)tiles;
        *p.size = (int)min(size, (int64_t)0x7FFFFFFF);
        *p.counter = 0;
    }
}

// One buffer of a chunk.
template <int D>
struct Chunk {
    alignas(16) uint8_t q[kChunk][2 * D + 16];
    alignas(16) float lse2[kChunk], fine[kChunk];
    alignas(16) int len[kChunk];
};

template <int D, class T, class C>
__global__ __launch_bounds__(kBlock, D == 256 ? 2 : 3) void weigh_block_kernel(BlockArgs b) {
    constexpr int NT = kTokens, PIECES = D / 8 / 4;  // 16-byte pieces of a thread: four threads to a column
    typedef typename Act<T>::frag frag;
    __shared__ Chunk<D> buf[2];
    __shared__ int64_t taken;
    const WeighArgs &a = b.a;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = lane & 31, g = lane >> 5;
    const int64_t cap = (int64_t)a.table_width << a.lp;
    const int size = *b.p.size;
    const int64_t total = b.p.unit_base[b.n];
    // this thread's column of every chunk
    const int col = tid >> 2;
    const int crow = b.parts > 1 ? 0 : col / a.per, chead = b.parts > 1 ? col : col - crow * a.per;
    const int part_heads = b.parts > 1 ? (a.per + b.parts - 1) / b.parts : a.per;

    for (;;) {
        __syncthreads();
        if (tid == 0) taken = atomicAdd(b.p.counter, 1);
        __syncthreads();
        const int64_t unit = taken;
        if (unit >= total) return;
        const int r = last_base(b.p.unit_base, b.n, unit);
        const int longest = b.p.longest[r], tiles = (longest + kTile - 1) / kTile;
        const int i = (int)(unit - b.p.unit_base[r]), piece = i / tiles, tile = i - piece * tiles;
        const int first_chunk = b.p.chunk_base[r], chunks = b.p.chunk_base[r + 1] - first_chunk;
        const int64_t all = (int64_t)chunks * a.kv_heads;
        const int64_t from = (int64_t)piece * size, to = min(from + size, all);
        const int row0 = bounded(a, r), row1 = bounded(a, r + 1);
        const int tile0 = tile * kTile, base = tile0 + 32 * NT * wave, tok = base + NT * n;
        const int pg = a.table[(int64_t)r * a.table_stride + (min((int64_t)tok, cap - 1) >> a.lp)];
        const bool there = pg >= 0 && pg < a.n_pages;
        const uint8_t *codes = a.k + (there ? pg : 0) * a.page_stride + (int64_t)(tok & ((1 << a.lp) - 1)) * D + 16 * g;
        const float *scales = a.ks + (there ? pg : 0) * a.scale_stride;
        float sum[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) sum[t] = 0.0f;

        for (int64_t at = from; at < to;) {
            const int head = (int)(at / chunks), c0 = (int)(at - (int64_t)head * chunks);
            const int c1 = (int)min((int64_t)chunks, c0 + (to - at));
            at += c1 - c0;
            frag k[NT][D / 16];
            float scale;
            bool loaded = false;
            for (int cs = c0; cs < c1; cs += 64) {
                // the chunks that see this tile, and those whose rows all see all of it
                const int mine = cs + lane;
                const int most = mine < c1 ? b.p.chunk_max[first_chunk + mine] : 0;
                const int least = mine < c1 ? b.p.chunk_min[first_chunk + mine] : 0;
                uint64_t some = __ballot(most > tile0);
                const uint64_t whole = __ballot(least >= tile0 + kTile);
                if (some == 0) continue;
                if (!loaded) {
                    u32x4 raw[NT][D / 32];
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int j = 0; j < D / 32; ++j)
                            raw[t][j] = *(const u32x4 *)(codes + ((int64_t)head << a.lp) * D + t * D + 32 * j);
                    scale = scales[head] * a.scale2;
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int j = 0; j < D / 32; ++j) {
                            k[t][2 * j] = eight<C, T>(raw[t][j][0], raw[t][j][1]);
                            k[t][2 * j + 1] = eight<C, T>(raw[t][j][2], raw[t][j][3]);
                        }
                    loaded = true;
                }
                u32x4 x[PIECES];
                float lse = 0.0f;
                int len = 0;
                const auto fetch = [&](int c) {
                    int row = row0, h = head * a.per;
                    bool on = col < (b.parts > 1 ? part_heads : b.rows * a.per);
                    if (b.parts > 1) {
                        row += c / b.parts;
                        const int at = c % b.parts * part_heads + chead;
                        on = on && at < a.per;
                        h += at;
                    } else {
                        row += c * b.rows + crow;
                        h += chead;
                    }
                    on = on && row < row1;
                    lse = -__builtin_inff();
                    len = 0;
#pragma unroll
                    for (int j = 0; j < PIECES; ++j) x[j] = u32x4{0, 0, 0, 0};
                    if (!on) return;
                    const char *q = (const char *)a.q + 2 * (row * a.q_row + h * a.q_head) + 16 * (tid & 3);
#pragma unroll
                    for (int j = 0; j < PIECES; ++j) x[j] = *(const u32x4 *)(q + 64 * j);
                    lse = a.lse[(int64_t)row * a.heads + h];
                    len = (int)min((int64_t)max(a.row_lengths[row], 0), cap);
                };
                const auto lay_out = [&](Chunk<D> &o) {
                    const Softmax s = softmax_of(lse, a.stretch);
                    // (what a row without a softmax holds is not looked at)
#pragma unroll
                    for (int j = 0; j < PIECES; ++j)
                        *(u32x4 *)&o.q[col][16 * (tid & 3) + 64 * j] = s.fine == 0.0f ? u32x4{0, 0, 0, 0} : x[j];
                    if ((tid & 3) == 0) {
                        o.lse2[col] = s.lse2;
                        o.fine[col] = s.fine;
                        o.len[col] = len;
                    }
                };
                int c = __builtin_ctzll(some), turn = 0;
                fetch(cs + c);
                __syncthreads();  // the chunk that was in the first buffer is done with
                lay_out(buf[0]);
                __syncthreads();
                while (some) {
                    const Chunk<D> &o = buf[turn];
                    some &= some - 1;
                    const int next = some ? __builtin_ctzll(some) : -1;
                    if (next >= 0) fetch(cs + next);
                    const bool masked = !(whole >> c & 1);
                    const int left = min(kChunk, b.parts > 1 ? part_heads : min(b.rows, row1 - row0 - (cs + c) * b.rows) * a.per);
#pragma unroll
                    for (int c32 = 0; c32 < kChunk; c32 += 32) {
                        if (c32 >= left) break;
                        f32x16 y[NT];
#pragma unroll
                        for (int t = 0; t < NT; ++t)
#pragma unroll
                            for (int i = 0; i < 16; ++i) y[t][i] = 0.0f;
                        const uint8_t *q = o.q[c32 + n] + 32 * g;
#pragma unroll
                        for (int j = 0; j < D / 16; ++j) {
                            const frag z = __builtin_bit_cast(frag, *(const u32x4 *)(q + 64 * (j >> 1) + 16 * (j & 1)));
#pragma unroll
                            for (int t = 0; t < NT; ++t) y[t] = Act<T>::mfma32(z, k[t][j], y[t]);
                        }
                        // place i of half g is column 8 (i / 4) + 4 g + i % 4
#pragma unroll
                        for (int i0 = 0; i0 < 16; i0 += 4) {
                            const int at = c32 + 2 * i0 + 4 * g;
                            const f32x4 l = *(const f32x4 *)&o.lse2[at], f = *(const f32x4 *)&o.fine[at];
                            if (masked) {
#pragma unroll
                                for (int i = 0; i < 4; ++i) {
                                    const int len = o.len[at + i];
#pragma unroll
                                    for (int t = 0; t < NT; ++t) {
                                        const float p = exp2_(fmaf(y[t][i0 + i], scale, -l[i])) * f[i];
                                        sum[t] += tok + t < len ? p : 0.0f;
                                    }
                                }
                            } else {
#pragma unroll
                                for (int i = 0; i < 4; ++i)
#pragma unroll
                                    for (int t = 0; t < NT; ++t)
                                        sum[t] = fmaf(exp2_(fmaf(y[t][i0 + i], scale, -l[i])), f[i], sum[t]);
                            }
                        }
                    }
                    if (next >= 0) lay_out(buf[turn ^ 1]);
                    __syncthreads();
                    turn ^= 1;
                    c = next;
                }
            }
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) sum[t] += __shfl_xor(sum[t], 32);
        if (g == 0) {
            if (all <= size) {
                float *w = a.weights + a.weight_offsets[r];
#pragma unroll
                for (int t = 0; t < NT; ++t)
                    if (there && tok + t < longest) w[tok + t] += sum[t];
            } else {
                float *w = b.p.parts + ((int64_t)b.p.slot_base[r] + i) * kTile + 32 * NT * wave + NT * n;
#pragma unroll
                for (int t = 0; t < NT; ++t) w[t] = sum[t];
            }
        }
    }
}

// Tiles whose sums lie in parts: a thread to a token.
__global__ __launch_bounds__(kTile) void join_kernel(BlockArgs b) {
    const WeighArgs &a = b.a;
    const int tid = threadIdx.x, total = b.p.tile_base[b.n];
    for (int i = blockIdx.x; i < total; i += gridDim.x) {
        const int r = last_base(b.p.tile_base, b.n, i), tile = i - b.p.tile_base[r];
        const int tiles = b.p.tile_base[r + 1] - b.p.tile_base[r], slot = b.p.slot_base[r];
        const int pieces = (b.p.slot_base[r + 1] - slot) / tiles, tok = tile * kTile + tid;
        if (tok >= b.p.longest[r]) continue;
        const int pg = a.table[(int64_t)r * a.table_stride + (tok >> a.lp)];
        const float *parts = b.p.parts + ((int64_t)slot + tile) * kTile + tid;
        float sum = 0.0f;
        for (int p0 = 0; p0 < pieces; p0 += 8) {
            float x[8];
#pragma unroll
            for (int p = 0; p < 8; ++p) x[p] = p0 + p < pieces ? parts[(int64_t)(p0 + p) * tiles * kTile] : 0.0f;
#pragma unroll
            for (int p = 0; p < 8; ++p) sum += x[p];
        }
        if (pg >= 0 && pg < a.n_pages) a.weights[a.weight_offsets[r] + tok] += sum;
    }
}

// A call's division into chunks, and the workspace's.
struct Sizes {
    int rows, parts, max_chunks;
    size_t bytes;
};
Sizes sizes_of(int64_t n_rows, int64_t n_requests, int per) {
    Sizes s;
    s.parts = (per + kChunk - 1) / kChunk;
    s.rows = s.parts > 1 ? 1 : kChunk / per;
    const int64_t chunks = s.parts > 1 ? n_rows * s.parts : n_rows / s.rows + n_requests;
    s.max_chunks = (int)(chunks < 0x7FFFFFF0 ? chunks : 0x7FFFFFF0);
    s.bytes = 256 + 8 * (size_t)(n_requests + 1) + 4 * (4 * (size_t)(n_requests + 1) + 2 * (size_t)chunks) + 256 +
              (size_t)2 * kUnits * kTile * sizeof(float);
    return s;
}

struct Launch {
    bool block;
    dim3 grid;
};

template <int D, class T, class C>
int launch_types(const BlockArgs &b, Launch l, void *stream) {
    return l.block ? launch(weigh_block_kernel<D, T, C>, l.grid, dim3(kBlock), stream, b)
                   : launch(weigh_rows_kernel<D, T, C>, l.grid, dim3(kBlock), stream, b.a);
}

template <int D>
int launch_dim(const BlockArgs &b, int act, int code, Launch l, void *stream) {
    if (code == PAGED_KV_E4M3)
        return act == PAGED_KV_BF16 ? launch_types<D, bf16, E4M3>(b, l, stream) : launch_types<D, f16, E4M3>(b, l, stream);
    return act == PAGED_KV_BF16 ? launch_types<D, bf16, Int8>(b, l, stream) : launch_types<D, f16, Int8>(b, l, stream);
}

// More rows than requests: rows share their keys.
inline bool many(int n_rows, int n_requests) { return n_rows > n_requests; }

}  // namespace
}  // namespace paged

extern "C" size_t serve_weigh_workspace(int32_t n_rows, int32_t n_requests, int32_t heads, int32_t kv_heads) {
    using namespace paged;
    if (n_rows < 0 || n_requests < 0 || heads < 1 || kv_heads < 1 || heads % kv_heads != 0) return 0;
    if (device_cus() == 0) return 0;
    return many(n_rows, n_requests) ? sizes_of(n_rows, n_requests, heads / kv_heads).bytes : 256;
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
    if (n_rows == 0 || n_requests == 0) return PAGED_KV_OK;
    if (!q || !lse || !table || !row_starts || !row_lengths || !weights || !weight_offsets || !aligned16(q) ||
        q_row % 8 || q_head % 8 || (many(n_rows, n_requests) && !workspace) || (uintptr_t)workspace % 256)
        return PAGED_KV_EINVAL;
    const int lp = log2_page(cache->page);
    if (((int64_t)table_width << lp) > 0x7FFFFFFF - 65536 || n_requests > 65535) return PAGED_KV_EUNSUPPORTED;
    const size_t need = serve_weigh_workspace(n_rows, n_requests, heads, cache->n_heads);
    if (need == 0) return PAGED_KV_EUNSUPPORTED;
    if (many(n_rows, n_requests) && workspace_bytes < need) return PAGED_KV_EWORKSPACE;
    const double exact = (double)scale * 1.4426950408889634;
    const float scale2 = (float)exact;
    BlockArgs b = {};
    b.a = {(const uint8_t *)cache->k, cache->k_scale, cache->page_stride, cache->scale_stride, cache->n_pages,
           lp, cache->n_heads, q, q_row, q_head, heads, heads / cache->n_heads, lse, table, table_stride,
           table_width, row_starts, row_lengths, n_rows, 1, scale2, scale2 > 0.0f ? (float)(exact / scale2 - 1.0) : 0.0f,
           weights, weight_offsets};
    const int64_t cap = (int64_t)table_width << lp;
    const bool block = many(n_rows, n_requests);
    dim3 grid;
    if (block) {
        const Sizes s = sizes_of(n_rows, n_requests, b.a.per);
        if (s.max_chunks == 0x7FFFFFF0) return PAGED_KV_EUNSUPPORTED;
        b.n = n_requests;
        b.rows = s.rows;
        b.parts = s.parts;
        b.max_chunks = s.max_chunks;
        char *at = (char *)workspace;
        const auto take = [&](size_t bytes) {
            char *p = at;
            at += bytes;
            return p;
        };
        b.p.parts = (float *)take((size_t)2 * kUnits * kTile * sizeof(float));
        b.p.counter = (int *)take(128);
        b.p.size = (int *)take(128);
        b.p.unit_base = (int64_t *)take(8 * (size_t)(n_requests + 1));
        b.p.slot_base = (int *)take(4 * (size_t)(n_requests + 1));
        b.p.tile_base = (int *)take(4 * (size_t)(n_requests + 1));
        b.p.chunk_base = (int *)take(4 * (size_t)(n_requests + 1));
        b.p.longest = (int *)take(4 * (size_t)(n_requests + 1));
        b.p.chunk_max = (int *)take(4 * (size_t)s.max_chunks);
        b.p.chunk_min = (int *)take(4 * (size_t)s.max_chunks);
        rc = launch(plan_kernel, dim3(1), dim3(kPlan), stream, b);
        if (rc != PAGED_KV_OK) return rc;
        grid = dim3((unsigned)(device_cus() * (cache->head_dim == 256 ? 2 : 3)));
    } else {
        while (b.a.steps < 4 && cap / (2 * b.a.steps * kTile) * n_requests >= 1024) b.a.steps *= 2;
        const int64_t tokens = (int64_t)kTile * b.a.steps;
        grid = dim3((unsigned)((cap + tokens - 1) / tokens), (unsigned)n_requests);
    }
    const Launch l = {block, grid};
    rc = cache->head_dim == 64    ? launch_dim<64>(b, act, cache->code, l, stream)
         : cache->head_dim == 128 ? launch_dim<128>(b, act, cache->code, l, stream)
                                  : launch_dim<256>(b, act, cache->code, l, stream);
    if (rc == PAGED_KV_OK && block) rc = launch(join_kernel, dim3(256), dim3(kTile), stream, b);
    return rc;
}
