// Rotary positions: pairs of a head's elements, turned by position * frequency.
//
// The angle in turns is position * turns, a 64-bit fixed-point fraction that wraps
// at whole turns by itself: nothing is lost at far positions, and no large argument
// is reduced.  A workgroup makes the cosines and sines of its rows in LDS once for
// all heads; then a thread takes V pairs, or V elements that are only copied, at a time.
// Cosines, sines and products are FP32, rounded once to the type.  Bound by memory where rows are
// many (8192 rows of 40 heads of 128: 33.5 us, 5.0 TB/s), by the chain of trips where few (64 rows: 3.6 us).
#include "../../include/serve_step.h"
#include "paged_common.h"

namespace paged {
namespace {

constexpr int kBlock = 256;
constexpr int kAngles = 2048;  // cosines of a workgroup
constexpr int kAhead = 2;      // pieces of a thread whose loads are on their way at once

struct Heads {
    const char *in;
    char *out;
    int64_t in_row, in_head, out_row, out_head;  // bytes
};

struct RotateArgs {
    Heads q, k;
    int q_heads, heads;  // heads from q_heads on are k's
    const uint64_t *turns;
    float magnitude, sine;  // the sine's magnitude has the direction's sign
    const void *positions;
    int wide, n_rows, half, start, pieces, rotated;  // pieces of a head, and those of them that are pairs
    int rows;        // of a workgroup
    int per;         // heads of a workgroup (blockIdx.y)
};

template <class T, int V>
struct Piece {
    typedef T type __attribute__((ext_vector_type(V)));
};
template <class T>
struct Piece<T, 1> {
    typedef T type;
};

template <class T, int V>
__device__ void unpack(typename Piece<T, V>::type x, float *y) {
    if constexpr (V == 1) y[0] = (float)x;
    else
#pragma unroll
        for (int i = 0; i < V; ++i) y[i] = (float)x[i];
}
template <class T, int V>
__device__ typename Piece<T, V>::type packed(const float *y) {
    typename Piece<T, V>::type x;
    if constexpr (V == 1) x = (T)y[0];
    else
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = (T)y[i];
    return x;
}

// Cosine and sine of t / 2^32 turns: the quarter turn apart, which is exact, so that
// what is left, at most an eighth of a turn, converts to a float within 2^-25 of that: 2^-28 of a turn.
__device__ inline void cos_sin(int t, float &c, float &s) {
    const int quarter = (int)((u32)t + (1u << 29)) >> 30;  // -2 .. 1
    const int rest = (int)((u32)t - ((u32)quarter << 30));
    float x, y;
    sincospif((float)rest * 0x1p-31f, &y, &x);
    c = quarter & 1 ? -y : x;
    s = quarter & 1 ? x : y;
    if (quarter & 2) {
        c = -c;
        s = -s;
    }
}

// PAST: results are written past the caches.
template <class T, int V, bool INTERLEAVED, bool PAST>
__global__ __launch_bounds__(kBlock) void rotate_kernel(RotateArgs a) {
    typedef typename Piece<T, V>::type piece;
    __shared__ alignas(16) float cosines[kAngles], sines[kAngles];
    const int tid = threadIdx.x, row0 = blockIdx.x * a.rows, rows = min(a.rows, a.n_rows - row0);
    const int head0 = blockIdx.y * a.per, heads = min(a.per, a.heads - head0);
    for (int i = tid; i < rows * a.half; i += kBlock) {
        const int r = i / a.half, p = i - r * a.half;
        const int64_t at = a.wide ? ((const int64_t *)a.positions)[row0 + r] : ((const int32_t *)a.positions)[row0 + r];
        float c, s;
        cos_sin((int)(u32)(((uint64_t)at * a.turns[p]) >> 32), c, s);
        cosines[i] = c * a.magnitude;
        sines[i] = s * a.sine;
    }
    __syncthreads();

    // a thread's items: every kBlock-th of (row, head, piece)
    int piece0 = tid % a.pieces, head = tid / a.pieces, row = head / heads;
    head -= row * heads;
    const int step_piece = kBlock % a.pieces, steps = kBlock / a.pieces, step_row = steps / heads,
              step_head = steps % heads;
    const auto next = [&] {
        piece0 += step_piece;
        head += step_head;
        row += step_row;
        if (piece0 >= a.pieces) {
            piece0 -= a.pieces;
            ++head;
        }
        if (head >= heads) {
            head -= heads;
            ++row;
        }
    };
    const auto put = [&](char *o, piece z) {
        if constexpr (PAST) __builtin_nontemporal_store(z, (piece *)o);
        else *(piece *)o = z;
    };
    while (row < rows) {
        piece x[kAhead], y[kAhead];
        char *to[kAhead];
        int at[kAhead], place[kAhead], second[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            place[i] = -1;
            if (row >= rows) continue;
            const int h = head0 + head;
            const bool is_q = h < a.q_heads;
            const Heads &o = is_q ? a.q : a.k;
            const int hh = is_q ? h : h - a.q_heads;
            const char *from = o.in + (row0 + row) * o.in_row + hh * o.in_head;
            to[i] = o.out + (row0 + row) * o.out_row + hh * o.out_head;
            int e;
            second[i] = 0;
            if (piece0 < a.rotated) {
                const int p = piece0 * V;
                e = a.start + (INTERLEAVED ? 2 * p : p);
                second[i] = (INTERLEAVED ? V : a.half) * (int)sizeof(T);
                at[i] = row * a.half + p;
            } else {
                e = (piece0 - a.rotated) * V;
                if (e >= a.start) e += 2 * a.half;
            }
            place[i] = e * (int)sizeof(T);
            x[i] = *(const piece *)(from + place[i]);
            if (second[i]) y[i] = *(const piece *)(from + place[i] + second[i]);
            next();
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            if (place[i] < 0) continue;
            char *o = to[i] + place[i];
            if (second[i] == 0) {
                put(o, x[i]);
                continue;
            }
            float u[2 * V], z[2 * V];
            unpack<T, V>(x[i], u);
            unpack<T, V>(y[i], u + V);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const int m = INTERLEAVED ? 2 * j : j, n = INTERLEAVED ? 2 * j + 1 : V + j;
                const float c = cosines[at[i] + j], s = sines[at[i] + j];
                z[m] = u[m] * c - u[n] * s;
                z[n] = u[m] * s + u[n] * c;
            }
            put(o, packed<T, V>(z));
            put(o + second[i], packed<T, V>(z + V));
        }
    }
}

template <class T, int V>
int launch_layout(const RotateArgs &a, bool interleaved, bool past, dim3 grid, void *stream) {
    if constexpr (V * sizeof(T) == 16)
        if (past)
            return interleaved ? launch(rotate_kernel<T, V, true, true>, grid, dim3(kBlock), stream, a)
                               : launch(rotate_kernel<T, V, false, true>, grid, dim3(kBlock), stream, a);
    return interleaved ? launch(rotate_kernel<T, V, true, false>, grid, dim3(kBlock), stream, a)
                       : launch(rotate_kernel<T, V, false, false>, grid, dim3(kBlock), stream, a);
}

}  // namespace
}  // namespace paged

extern "C" int serve_rotate(int32_t act, const serve_rotary *rotary, const void *positions, int32_t wide,
                            int32_t n_rows, int32_t dim, const serve_heads *q, const serve_heads *k,
                            int32_t transposed, void *stream) {
    using namespace paged;
    if (!rotary || !q || n_rows < 0 || act < PAGED_KV_BF16 || act > SERVE_F32) return PAGED_KV_EINVAL;
    const int rot = rotary->rot, start = rotary->start;
    if (!rotary->turns || rot < 2 || rot % 2 || start < 0 || dim < 1 || (int64_t)start + rot > dim ||
        !(rotary->magnitude - rotary->magnitude == 0.0f))
        return PAGED_KV_EINVAL;
    if (q->heads < 1 || (k && k->heads < 1)) return PAGED_KV_EINVAL;
    if (rot > 1024 || dim > 65536 || (int64_t)q->heads + (k ? k->heads : 0) > 1 << 20) return PAGED_KV_EUNSUPPORTED;
    if (n_rows == 0) return PAGED_KV_OK;
    const int size = act == SERVE_F32 ? 4 : 2;
    if (!positions || (uintptr_t)positions % (wide ? 8 : 4) || (uintptr_t)rotary->turns % 8) return PAGED_KV_EINVAL;
    // the widest pieces that everything is a multiple of
    uint64_t any = (uint64_t)(rot / 2) | start | dim;
    const serve_heads *both[2] = {q, k};
    for (const serve_heads *h : both) {
        if (!h) continue;
        if (!h->in || !h->out || (uintptr_t)h->in % size || (uintptr_t)h->out % size) return PAGED_KV_EINVAL;
        if (h->in == h->out && ((n_rows > 1 && h->in_row != h->out_row) || (h->heads > 1 && h->in_head != h->out_head)))
            return PAGED_KV_EINVAL;
        any |= (uint64_t)h->in_row | (uint64_t)h->in_head | (uint64_t)h->out_row | (uint64_t)h->out_head |
               (uintptr_t)h->in / size | (uintptr_t)h->out / size;
    }
    if (device_cus() == 0) return PAGED_KV_EUNSUPPORTED;
    int v = 16 / size;
    while (any % v) v /= 2;
    const auto heads_of = [&](const serve_heads *h) {
        return h ? Heads{(const char *)h->in, (char *)h->out, h->in_row * size, h->in_head * size, h->out_row * size,
                         h->out_head * size}
                 : Heads{};
    };
    RotateArgs a = {};
    a.q = heads_of(q);
    a.k = heads_of(k);
    a.q_heads = q->heads;
    a.heads = q->heads + (k ? k->heads : 0);
    a.turns = rotary->turns;
    a.magnitude = rotary->magnitude;
    a.sine = transposed ? -rotary->magnitude : rotary->magnitude;
    a.positions = positions;
    a.wide = wide != 0;
    a.n_rows = n_rows;
    a.half = rot / 2;
    a.start = start;
    a.rotated = rot / 2 / v;
    bool in_place = true;
    for (const serve_heads *h : both)
        in_place = in_place && (!h || (h->in == h->out && h->in_row == h->out_row && h->in_head == h->out_head));
    a.pieces = a.rotated + (in_place ? 0 : (dim - rot) / v);
    // few rows: their heads over several workgroups; many: several rows to one
    a.rows = 1;
    a.per = a.heads;
    while (a.per > 1 && (int64_t)a.per * a.pieces > kBlock && (int64_t)n_rows * ((a.heads + a.per - 1) / a.per) < 512)
        a.per = (a.per + 1) / 2;
    if (a.per == a.heads)
        while (2 * a.rows * a.half <= kAngles && (int64_t)a.rows * a.heads * a.pieces < 4 * kBlock &&
               n_rows / (2 * a.rows) >= 1024)
            a.rows *= 2;
    // what the L2s (32 MB) do not hold anyway goes past them (8192 rows of 40 heads of 128: 33.5 us,
    // and 39.9 with stores that stay in them; with the store of its keys and one reader of its queries behind
    // it 91 and 99, but 35.2 and 31.7 for 2048 rows, 21 MB, which the last-level cache holds)
    const bool past = (int64_t)n_rows * a.heads * dim * size > 16 << 20;
    const dim3 grid((unsigned)(((int64_t)n_rows + a.rows - 1) / a.rows), (unsigned)((a.heads + a.per - 1) / a.per));
    if (grid.y > 65535) return PAGED_KV_EUNSUPPORTED;
    const bool il = rotary->interleaved != 0;
    if (act == SERVE_F32)
        return v == 4   ? launch_layout<float, 4>(a, il, past, grid, stream)
               : v == 2 ? launch_layout<float, 2>(a, il, past, grid, stream)
                        : launch_layout<float, 1>(a, il, past, grid, stream);
    const auto go = [&](auto t) {
        typedef decltype(t) T;
        return v == 8   ? launch_layout<T, 8>(a, il, past, grid, stream)
               : v == 4 ? launch_layout<T, 4>(a, il, past, grid, stream)
               : v == 2 ? launch_layout<T, 2>(a, il, past, grid, stream)
                        : launch_layout<T, 1>(a, il, past, grid, stream);
    };
    return act == PAGED_KV_BF16 ? go(bf16()) : go(f16());
}
