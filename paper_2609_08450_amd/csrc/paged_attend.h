// What the two attention kernels share: the arguments, the plan that deals the
// work to workgroups, and the joining of a row's parts.
//
// Work is counted in units (a fixed number of tokens of one group of rows and
// one cache head) and laid out in one line: requests, of a request its cache
// heads, of a head its groups, of a group its units (for single rows: rows, of a
// row its heads, of a head its units).  Workgroup w of W takes
// the units [w T / W, (w + 1) T / W) of T, whatever rows they belong to, so
// all end together however long the rows are.  A group that lies in several
// workgroups' shares is joined from its parts, each with a maximum, a sum and the
// weighted values in FP32: for single rows by the last workgroup to arrive, for
// prompts, whose parts are 16 times as large, by a launch of its own.
#pragma once

#include "paged_common.h"

namespace paged {

constexpr int kMaxShares = 2048;  // workgroups of a launch; one ticket each
constexpr int kStreamRows = 1024; // rows of a launch of the kernel for single rows
constexpr int kSelectedUnit = 256; // selected tokens that a workgroup takes at a time
constexpr float kLow = -1e30f;    // below every score: the maximum of nothing
constexpr float kSlack = 8.0f;    // a maximum may be passed by this much (powers of 2) before it moves

struct Group {
    int row0, rows, request, len;  // len: the longest of its rows
};

struct AttendArgs {
    const uint8_t *k, *v;
    const float *ks, *vs;
    int64_t page_stride, scale_stride;
    int n_pages, lp, kv_heads;
    const void *q;
    int64_t q_row, q_head;
    void *out;
    float *lse;
    const int *table;
    int table_stride, table_width;
    const int *row_starts, *row_lengths;
    int n_rows, n_requests;
    int row0;         // first row of this launch, in the kernel for single rows
    int heads, per;   // query heads, and those of a cache head
    int parts;        // cuts of those `per` heads, each a "head" of the plan
    float scale2;     // scale * log2(e): scores are powers of 2
    // the plan
    int rows_per_group, max_groups, shares, unit;
    int *tickets;     // [kMaxShares], zero between calls
    Group *groups;    // [max_groups]
    int *group_units; // [max_groups + 1] prefix sum of the groups' units
    int *group_base;  // [n_requests + 1] first group of each request
    int4 *starts;     // [shares] group, head, unit, request at a share's start
    int64_t *total;   // [2] units in all, shares in use
    float *left;      // [2 * shares] parts: per column maximum, sum, then values
    // selected rows
    const int *idx, *row_request;
    int K, splits;
};

__device__ inline int64_t share_start(int64_t w, int64_t total, int64_t shares) { return w * total / shares; }
__device__ inline int share_of(int64_t unit, int64_t total, int64_t shares) {
    return (int)(((unit + 1) * shares - 1) / total);
}

// Parts go from one workgroup to another in relaxed agent-scope accesses, which
// pass the XCDs' own caches; a wait for them, then the ticket, orders them.  (A
// fence instead writes the whole L2 back: the decode batch took 682 us with it
// instead of 436.)
__device__ inline void give(float *p, float a, float b) {
    __hip_atomic_store((uint64_t *)p, __builtin_bit_cast(uint64_t, f32x2{a, b}), __ATOMIC_RELAXED,
                       __HIP_MEMORY_SCOPE_AGENT);
}
__device__ inline void give4(float *p, f32x4 x) {
    give(p, x[0], x[1]);
    give(p + 2, x[2], x[3]);
}
__device__ inline f32x2 taken(const float *p) {
    return __builtin_bit_cast(
        f32x2, __hip_atomic_load((const uint64_t *)p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
}
__device__ inline f32x4 taken4(const float *p) {
    const f32x2 a = taken(p), b = taken(p + 2);
    return f32x4{a[0], a[1], b[0], b[1]};
}
// After the workgroup's stores of its part: is it the last of `parts` to arrive?
// The ticket is back at 0 then.
__device__ inline bool arrived_last(int *ticket, int parts, int *flag) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0) {
        const int n = __hip_atomic_fetch_add(ticket, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (n == parts - 1) __hip_atomic_store(ticket, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        *flag = n == parts - 1;
    }
    __syncthreads();
    return *flag != 0;
}

// Joins the parts of a group's columns [first, cols); `part` gives part p's place.
// A thread holds four values of a column and goes through parts of its own, eight
// at once with their maximum and sum beside them: one after the other each would
// cost a trip to memory (one row of 131071 tokens, 32 parts to a head: 57 us, and
// 67 with maxima and values in passes of their own).
template <int BLOCK>
struct Joined {
    f32x4 o[BLOCK];
    float m[BLOCK], l[BLOCK];
};

// LIVE: the parts were written by workgroups of this launch.
template <int D, int COLS, int BLOCK, bool LIVE, class Part, class Out>
__device__ void join_parts(Joined<BLOCK> &j, int parts, int first, int cols, Part part, Out out) {
    constexpr int PER = BLOCK / (D / 4), AHEAD = 8;  // columns of a pass
    const int tid = threadIdx.x, d = tid % (D / 4) * 4;
    for (int c0 = first; c0 < cols; c0 += PER) {
        // where a pass has fewer columns, its threads share out the parts
        int width = PER;
        while (width / 2 >= cols - c0) width /= 2;
        const int spans = PER / width, col = c0 + tid / (D / 4) % width, span = tid / (D / 4) / width;
        f32x4 o = {0, 0, 0, 0};
        float m = kLow, l = 0.0f;
        if (col < cols)
            for (int p0 = span; p0 < parts; p0 += AHEAD * spans) {
                f32x2 ml[AHEAD];
                f32x4 v[AHEAD];
#pragma unroll
                for (int i = 0; i < AHEAD; ++i) {
                    const float *from = part(min(p0 + i * spans, parts - 1));
                    const float *values = from + 2 * COLS + col * D + d;
                    ml[i] = LIVE ? taken(from + 2 * col) : *(const f32x2 *)(from + 2 * col);
                    v[i] = LIVE ? taken4(values) : *(const f32x4 *)values;
                }
                float to = m;
#pragma unroll
                for (int i = 0; i < AHEAD; ++i) {
                    if (p0 + i * spans >= parts) ml[i] = f32x2{kLow, 0.0f};
                    to = fmaxf(to, ml[i][0]);
                }
                const float by = exp2_(m - to);
                o *= by;
                l *= by;
#pragma unroll
                for (int i = 0; i < AHEAD; ++i) {
                    // (a part that saw nothing has no values either; a sum that is NaN stays one)
                    const float w = ml[i][1] != 0.0f ? exp2_(ml[i][0] - to) : 0.0f;
                    l += ml[i][1] * w;
                    o += v[i] * w;
                }
                m = to;
            }
        if (spans > 1) {
            j.o[tid] = o;
            j.m[tid] = m;
            j.l[tid] = l;
            __syncthreads();
            if (span == 0)
                for (int i = 1; i < spans; ++i) {
                    const int at = tid + i * width * (D / 4);
                    const float to = fmaxf(m, j.m[at]), x = exp2_(m - to), y = exp2_(j.m[at] - to);
                    o = o * x + j.o[at] * y;
                    l = l * x + j.l[at] * y;
                    m = to;
                }
            __syncthreads();
        }
        if (col < cols && span == 0) out(col, d, o, m, l);
    }
}

template <int D, class T>
__device__ void write_out(const AttendArgs &a, int64_t at, int d, f32x4 o, float top, float sum) {
    o *= sum != 0.0f ? 1.0f / sum : 0.0f;
    *(u32x2 *)((uint16_t *)a.out + at * D + d) = u32x2{pack2<T>(o[0], o[1]), pack2<T>(o[2], o[3])};
    if (d == 0 && a.lse)
        a.lse[at] = sum != 0.0f ? (top + __log2f(sum)) * 0.6931471805599453f : -__builtin_inff();
}

// A group's first `cols` columns, in LDS: red[col][D + 4] the weighted values, top
// and sum the softmax's.  `place` gives a column's output row.
template <int D, int COLS, int BLOCK, class T, class Place>
__device__ void finish(const AttendArgs &a, float (*red)[D + 4], float *top, float *sum, Joined<BLOCK> &joined,
                       int cols, bool whole, int slot, int first_share, int parts, int first_slot, Place place) {
    __shared__ int last;
    const int tid = threadIdx.x;
    constexpr int PART = COLS * (D + 2);
    if (whole) {
        for (int i = tid; i < cols * (D / 4); i += BLOCK) {
            const int c = i / (D / 4), d = i % (D / 4) * 4;
            write_out<D, T>(a, place(c), d, *(const f32x4 *)&red[c][d], top[c], sum[c]);
        }
        __syncthreads();
        return;
    }
    // a part: pairs of maximum and sum, then the values
    float *mine = a.left + (int64_t)slot * PART;
    for (int i = tid; i < cols * (D / 4); i += BLOCK) {
        const int c = i / (D / 4), d = i % (D / 4) * 4;
        give4(mine + 2 * COLS + c * D + d, *(const f32x4 *)&red[c][d]);
    }
    for (int c = tid; c < cols; c += BLOCK) give(mine + 2 * c, top[c], sum[c]);
    if (!arrived_last(&a.tickets[first_share], parts, &last)) return;
    // part p lies in slot 0 of share first_share + p, the first one in first_slot
    join_parts<D, COLS, BLOCK, true>(
        joined, parts, 0, cols,
        [&](int p) { return a.left + (int64_t)(p == 0 ? first_slot : 2 * (first_share + p)) * PART; },
        [&](int c, int d, f32x4 o, float m, float l) { write_out<D, T>(a, place(c), d, o, m, l); });
}

int launch_stream(const AttendArgs &a, int head_dim, int act, int code, bool selected, int tiles, int grid, void *stream);
int launch_prompt(const AttendArgs &a, int head_dim, int act, int code, int grid, void *stream);

}  // namespace paged
