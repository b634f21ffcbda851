// A step's block tables, row tables and slots from request lengths.
//
// Three prefix sums over the requests: rows, pages released, pages taken.  One
// workgroup makes them (requests are few: a thread to each, in rounds) and moves
// the pages, a thread to a page, which finds its request in the sums.  The rows'
// table is written by the same workgroup when it is short and by a grid of its own
// when it is long.  The call is bound by its chain of dependent steps, not by its
// bytes: lengths, sums, pages out of the ring, slots.  64 requests of one token:
// 3.2 us; 1021 requests, 16384 rows and 16000 pages given back: 20 + 4 us.
#include "paged_common.h"

namespace paged {
namespace {

constexpr int kLarge = 1024;   // threads of the planning workgroup; 256 for few requests
constexpr int kOwnRows = 4096; // rows that it writes itself
constexpr int kStarts = 4097;  // requests' starts and lengths kept in LDS, plus one

struct TablesArgs {
    int32_t *ring;
    int32_t ring_size;
    const int32_t *pool_in;
    int32_t *pool_out;
    const int32_t *lens_in, *new_lens;
    int32_t *lens_out;
    int32_t n;
    int32_t *table;
    int32_t stride, width, lp, n_rows;
    int32_t *row_starts, *row_request, *row_lengths;
    int64_t *slots;
};

// What the step does to one request.
struct Change {
    int64_t len, to;  // tokens before and after, were it granted
    int held, need;   // pages
    int rows, give, take;
    bool wide;
};

__device__ Change change_of(const TablesArgs &a, int r) {
    Change c;
    const int64_t cap = (int64_t)a.width << a.lp;
    const int64_t add = a.new_lens[r];
    c.len = min((int64_t)max(a.lens_in[r], 0), cap);
    c.to = max(c.len + add, (int64_t)0);
    c.held = (int)((c.len + (1 << a.lp) - 1) >> a.lp);
    const int64_t need = (c.to + (1 << a.lp) - 1) >> a.lp;
    c.wide = need > a.width;
    c.need = c.wide ? c.held : (int)need;
    c.rows = (int)max(add, (int64_t)0);
    c.give = max(c.held - c.need, 0);
    c.take = max(c.need - c.held, 0);
    return c;
}

struct Sums {
    int64_t give, take, rows;
};

// Exclusive prefix of x over the workgroup; totals in *all.
template <int BLOCK>
__device__ Sums prefix(Sums x, Sums *waves, Sums *all) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    Sums s = x;
    for (int d = 1; d < 64; d <<= 1) {
        const int64_t g = __shfl_up(s.give, d), t = __shfl_up(s.take, d), r = __shfl_up(s.rows, d);
        if (lane >= d) s = {s.give + g, s.take + t, s.rows + r};
    }
    __syncthreads();
    if (lane == 63) waves[w] = s;
    __syncthreads();
    Sums before = {0, 0, 0};
    *all = {0, 0, 0};
#pragma unroll
    for (int i = 0; i < BLOCK / 64; ++i) {
        if (i == w) before = *all;
        *all = {all->give + waves[i].give, all->take + waves[i].take, all->rows + waves[i].rows};
    }
    return {before.give + s.give - x.give, before.take + s.take - x.take, before.rows + s.rows - x.rows};
}

// Counts of rows past 32 bits stay at the largest: were they to wrap, a row's search in
// them could end at a request that it does not belong to, outside its table.
__device__ int held(int64_t rows) { return (int)min(rows, (int64_t)0x7FFFFFFF); }

// Last i in [0, n) with starts[i] <= x (starts rise, starts[0] <= x).
__device__ int last_start(const int32_t *starts, int n, int x) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (starts[mid] <= x) lo = mid; else hi = mid;
    }
    return lo;
}

// Row i of request r, whose length was `len`, and negative where the step refuses it.
__device__ void write_row(const TablesArgs &a, int i, int r, int start, int64_t len) {
    int length = 0;
    int64_t slot = -1;
    if (len >= 0) {
        const int64_t pos = len + (i - start);
        const int page = a.table[(int64_t)r * a.stride + (pos >> a.lp)];
        slot = ((int64_t)page << a.lp) + (pos & ((1 << a.lp) - 1));
        length = (int)pos + 1;
    }
    a.row_request[i] = r;
    a.row_lengths[i] = length;
    a.slots[i] = slot;
}
__device__ void no_row(const TablesArgs &a, int i) {
    a.row_request[i] = -1;
    a.row_lengths[i] = 0;
    a.slots[i] = -1;
}

// `own`: the rows too.
template <int BLOCK>
__global__ __launch_bounds__(BLOCK) void tables_kernel(TablesArgs a, bool own) {
    __shared__ Sums waves[BLOCK / 64];
    __shared__ int32_t starts[kStarts], lens[kStarts];
    __shared__ int32_t order[BLOCK + 1];  // prefix sum of a round's moved pages
    __shared__ int32_t column[BLOCK];     // their first column in the table
    __shared__ int refused;
    __shared__ unsigned long long taken;
    const int tid = threadIdx.x;
    const int64_t size = a.ring_size;
    const int64_t head = (u32)a.pool_in[0] % (u32)a.ring_size;  // any state stays inside the ring
    const int64_t free_in = min(max((int64_t)a.pool_in[1], (int64_t)0), size);
    if (tid == 0) {
        refused = 0;
        taken = 0;
    }
    // Moves a round's `count` pages between table and ring, which holds them from `at` on.
    const auto move = [&](int base, int count, int64_t at, bool to_ring) {
        __syncthreads();
        const int n = min(BLOCK, a.n - base);
        const u32 first = (u32)(at % size);
        // four pages of a thread at once: one after the other each would cost its trips to memory
        for (int i0 = tid; i0 < count; i0 += 4 * BLOCK) {
            int32_t *entry[4], *place[4], page[4];
            int i[4], k[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                i[j] = min(i0 + j * BLOCK, count - 1);
                k[j] = 0;
            }
            for (int step = BLOCK / 2; step; step >>= 1)  // the last request that starts at or before page i
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int to = k[j] + step;
                    if (to < n && order[min(to, n - 1)] <= i[j]) k[j] = to;
                }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                entry[j] = a.table + (int64_t)(base + k[j]) * a.stride + column[k[j]] + (i[j] - order[k[j]]);
                place[j] = a.ring + (first + (u32)i[j]) % (u32)size;
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) page[j] = to_ring ? *entry[j] : *place[j];
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (i0 + j * BLOCK < count) *(to_ring ? place[j] : entry[j]) = page[j];
        }
        __syncthreads();
    };

    const bool single = a.n <= BLOCK;  // one round
    Sums done = {0, 0, 0}, all;
    int64_t given = 0;
    if (!single)
        for (int base = 0; base < a.n; base += BLOCK) {
            const int r = base + tid;
            const Change c = r < a.n ? change_of(a, r) : Change{};
            const Sums at = prefix<BLOCK>({c.give, 0, 0}, waves, &all);
            order[tid] = (int)at.give;
            column[tid] = c.need;
            // pages that go back, in the requests' order, to the ring's end
            if (all.give > 0) move(base, (int)all.give, head + free_in + given, true);
            given += all.give;
        }
    for (int base = 0; base < a.n; base += BLOCK) {
        const int r = base + tid;
        const Change c = r < a.n ? change_of(a, r) : Change{};
        const Sums at = prefix<BLOCK>({c.give, c.take, c.rows}, waves, &all);
        if (single) {
            order[tid] = (int)at.give;
            column[tid] = c.need;
            if (all.give > 0) move(base, (int)all.give, head + free_in, true);
            given = all.give;
        }
        // pages that are taken from its front: by the first requests that ask, up to
        // the last whose pages are all there
        const int64_t from = done.take + at.take, upto = from + c.take;
        const bool granted = upto <= free_in + given && !c.wide;
        const bool no = !granted && c.rows > 0 && (c.wide || c.take > 0);
        if (no) atomicAdd(&refused, 1);
        if (granted && c.take > 0) atomicMax(&taken, (unsigned long long)upto);
        if (r < a.n) {
            const int start = held(done.rows + at.rows);
            a.lens_out[r] = (int32_t)(no ? c.len : c.to);
            a.row_starts[r] = start;
            if (own) {
                starts[r] = start;
                lens[r] = no ? -1 : (int32_t)c.len;
            }
        }
        if (all.take > 0) {
            __syncthreads();
            order[tid] = (int)at.take;
            column[tid] = c.held;
            __syncthreads();
            const int64_t count = min((int64_t)taken - done.take, all.take);
            if (count > 0) move(base, (int)count, head + done.take, false);
        }
        done = {done.give + all.give, done.take + all.take, done.rows + all.rows};
    }
    __syncthreads();
    if (tid == 0) {
        a.row_starts[a.n] = held(done.rows);
        a.pool_out[0] = (int32_t)((head + (int64_t)taken) % size);
        a.pool_out[1] = (int32_t)(free_in + given - (int64_t)taken);
        a.pool_out[2] = refused;
        a.pool_out[3] = 0;
    }
    if (!own) return;
    for (int i = tid; i < a.n_rows; i += BLOCK) {
        if (i >= done.rows) {
            no_row(a, i);
            continue;
        }
        const int r = last_start(starts, a.n, i);
        write_row(a, i, r, starts[r], lens[r]);
    }
}

// The rows of a long step, after tables_kernel.
__global__ __launch_bounds__(256) void rows_kernel(TablesArgs a) {
    __shared__ int32_t starts[kStarts];
    const bool lds = a.n < kStarts;
    if (lds)
        for (int i = threadIdx.x; i <= a.n; i += 256) starts[i] = a.row_starts[i];
    __syncthreads();
    const int32_t *all = lds ? starts : a.row_starts;
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i >= a.n_rows) return;
    if (i >= all[a.n]) return no_row(a, i);
    const int r = last_start(all, a.n, i);
    const int64_t len = min((int64_t)max(a.lens_in[r], 0), (int64_t)a.width << a.lp);
    // a refused request keeps its length
    write_row(a, i, r, all[r], a.lens_out[r] != len ? len : -1);
}

}  // namespace
}  // namespace paged

extern "C" int paged_kv_tables(int32_t *ring, int32_t ring_size, const int32_t *pool_in, int32_t *pool_out,
                               const int32_t *lens_in, const int32_t *new_lens, int32_t *lens_out,
                               int32_t n_requests, int32_t *table, int32_t table_stride, int32_t table_width,
                               int32_t page, int32_t n_rows, int32_t *row_starts, int32_t *row_request,
                               int32_t *row_lengths, int64_t *slots, void *stream) {
    using namespace paged;
    if (n_requests < 0 || n_rows < 0 || ring_size < 1 || table_width < 1 || table_stride < table_width)
        return PAGED_KV_EINVAL;
    if (!ring || !pool_in || !pool_out || !row_starts) return PAGED_KV_EINVAL;
    if (n_requests > 0 && (!lens_in || !new_lens || !lens_out || !table || lens_in == lens_out)) return PAGED_KV_EINVAL;
    if (n_rows > 0 && (!row_request || !row_lengths || !slots)) return PAGED_KV_EINVAL;
    const int lp = log2_page(page);
    if (lp < 0) return PAGED_KV_EUNSUPPORTED;
    if (((int64_t)table_width << lp) > 0x7FFFFFFF) return PAGED_KV_EUNSUPPORTED;
    if (device_cus() == 0) return PAGED_KV_EUNSUPPORTED;
    const TablesArgs a = {ring, ring_size, pool_in, pool_out, lens_in, new_lens, lens_out, n_requests, table,
                          table_stride, table_width, lp, n_rows, row_starts, row_request, row_lengths, slots};
    const bool own = n_rows <= kOwnRows && n_requests < kStarts;
    int rc = n_requests <= 256 && n_rows <= 1024 ? launch(tables_kernel<256>, dim3(1), dim3(256), stream, a, own)
                                                 : launch(tables_kernel<kLarge>, dim3(1), dim3(kLarge), stream, a, own);
    if (rc == PAGED_KV_OK && !own)
        rc = launch(rows_kernel, dim3((unsigned)((n_rows + 255) / 256)), dim3(256), stream, a);
    return rc;
}

extern "C" const char *paged_kv_status_str(int status) {
    switch (status) {
    case PAGED_KV_OK: return "ok";
    case PAGED_KV_EINVAL: return "invalid argument";
    case PAGED_KV_EUNSUPPORTED: return "unsupported size, type or device (gfx950 required)";
    case PAGED_KV_ELAUNCH: return "HIP launch or runtime error";
    case PAGED_KV_EWORKSPACE: return "workspace too small";
    default: return "unknown status";
    }
}
