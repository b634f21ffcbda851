// A step's block tables, row tables and slots from request lengths.
//
// Three prefix sums over the requests: rows, pages released, pages taken.  One
// workgroup makes them (requests are few: 1024 to a round) and moves the
// pages, one wave to a request; the rows' table is written by the same
// workgroup when it is short and by a grid of its own when it is long.  The
// call is bound by its chain of dependent steps, not by its bytes.
#include "paged_common.h"

namespace paged {
namespace {

constexpr int kPlan = 1024;    // threads of the planning workgroup
constexpr int kOwnRows = 4096; // rows that it writes itself
constexpr int kStarts = 4097;  // starts kept in LDS

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

// Exclusive prefix of x over the workgroup; total in *sum.
__device__ int64_t prefix(int64_t x, int64_t *waves, int64_t *sum) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, n = blockDim.x >> 6;
    int64_t s = x;
    for (int d = 1; d < 64; d <<= 1) {
        const int64_t y = __shfl_up(s, d);
        if (lane >= d) s += y;
    }
    __syncthreads();
    if (lane == 63) waves[w] = s;
    __syncthreads();
    int64_t before = 0, all = 0;
    for (int i = 0; i < n; ++i) {
        if (i == w) before = all;
        all += waves[i];
    }
    *sum = all;
    return before + s - x;
}

// Row i: its request is the last one that starts at or before it.
__device__ void write_row(const TablesArgs &a, const int32_t *starts, int i) {
    int request = -1, length = 0;
    int64_t slot = -1;
    if (i < starts[a.n]) {
        int lo = 0, hi = a.n;  // starts[lo] <= i < starts[hi]
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (starts[mid] <= i) lo = mid; else hi = mid;
        }
        request = lo;
        const int64_t cap = (int64_t)a.width << a.lp;
        const int64_t len = min((int64_t)max(a.lens_in[lo], 0), cap);
        if (a.lens_out[lo] != len) {  // granted: a refused request keeps its length
            const int64_t pos = len + (i - starts[lo]);
            const int page = a.table[(int64_t)lo * a.stride + (pos >> a.lp)];
            slot = ((int64_t)page << a.lp) + (pos & ((1 << a.lp) - 1));
            length = (int)pos + 1;
        }
    }
    a.row_request[i] = request;
    a.row_lengths[i] = length;
    a.slots[i] = slot;
}

// `own`: the rows too.
__global__ __launch_bounds__(kPlan) void tables_kernel(TablesArgs a, bool own) {
    __shared__ int64_t waves[kPlan / 64];
    __shared__ int32_t starts[kStarts];
    __shared__ int moves[kPlan][3];  // of a round's requests: first page in the table, count, place in the ring
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t size = a.ring_size;
    const int64_t head = (u32)a.pool_in[0] % (u32)a.ring_size;  // any state stays inside the ring
    const int64_t free_in = min(max((int64_t)a.pool_in[1], (int64_t)0), size);

    // pages that go back, in the requests' order, to the ring's end
    int64_t given = 0;
    for (int base = 0; base < a.n; base += kPlan) {
        const int r = base + tid;
        const Change c = r < a.n ? change_of(a, r) : Change{};
        int64_t all;
        const int64_t before = prefix(c.give, waves, &all);
        if (all > 0) {
            moves[tid][0] = c.need;
            moves[tid][1] = c.give;
            moves[tid][2] = (int)((head + free_in + given + before) % size);
            __syncthreads();
            for (int k = wave; k < kPlan && base + k < a.n; k += kPlan / 64)
                for (int j = lane; j < moves[k][1]; j += 64)
                    a.ring[((int64_t)moves[k][2] + j) % size] =
                        a.table[(int64_t)(base + k) * a.stride + moves[k][0] + j];
        }
        given += all;
        __syncthreads();
    }

    // pages that are taken from its front, and the rows' starts
    const int64_t free_now = free_in + given;
    int64_t taken = 0, asked = 0, rows = 0, refused = 0;
    for (int base = 0; base < a.n; base += kPlan) {
        const int r = base + tid;
        const Change c = r < a.n ? change_of(a, r) : Change{};
        int64_t all, got;
        const int64_t upto = asked + prefix(c.take, waves, &all) + c.take;
        asked += all;
        const bool granted = upto <= free_now && !c.wide;
        const int take = granted ? c.take : 0;
        moves[tid][0] = c.held;
        moves[tid][1] = take;
        moves[tid][2] = (int)((head + upto - c.take) % size);
        const bool no = !granted && c.rows > 0 && (c.wide || c.take > 0);
        const int64_t lost = __popcll(__ballot(no));
        // refusals above, pages taken below: one sum for both
        prefix(((lane == 0 ? lost : 0) << 40) + take, waves, &got);
        refused += got >> 40;
        taken += got & (((int64_t)1 << 40) - 1);
        const int64_t start = rows + prefix(c.rows, waves, &got);
        rows += got;
        if (r < a.n) {
            a.lens_out[r] = (int32_t)(no ? c.len : c.to);
            a.row_starts[r] = (int32_t)start;
            if (own && r < kStarts) starts[r] = (int32_t)start;
        }
        if (all > 0)
            for (int k = wave; k < kPlan && base + k < a.n; k += kPlan / 64)
                for (int j = lane; j < moves[k][1]; j += 64)
                    a.table[(int64_t)(base + k) * a.stride + moves[k][0] + j] =
                        a.ring[((int64_t)moves[k][2] + j) % size];
        __syncthreads();
    }
    if (tid == 0) {
        a.row_starts[a.n] = (int32_t)rows;
        if (own) starts[a.n] = (int32_t)rows;
        a.pool_out[0] = (int32_t)((head + taken) % size);
        a.pool_out[1] = (int32_t)(free_now - taken);
        a.pool_out[2] = (int32_t)refused;
        a.pool_out[3] = 0;
    }
    if (!own) return;
    __syncthreads();
    for (int i = tid; i < a.n_rows; i += kPlan) write_row(a, starts, i);
}

// The rows of a long step, after tables_kernel.
__global__ __launch_bounds__(256) void rows_kernel(TablesArgs a) {
    __shared__ int32_t starts[kStarts];
    const bool lds = a.n < kStarts;
    if (lds)
        for (int i = threadIdx.x; i <= a.n; i += 256) starts[i] = a.row_starts[i];
    __syncthreads();
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i < a.n_rows) write_row(a, lds ? starts : a.row_starts, i);
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
    int rc = launch(tables_kernel, dim3(1), dim3(kPlan), stream, a, own);
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
