// The attention calls: their checks, workspace and plan.
#include "paged_attend.h"

namespace paged {
namespace {

constexpr int kPlan = 1024;

// Exclusive prefix of x over the workgroup; total in *sum.
__device__ int prefix(int x, int *waves, int *sum) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    int s = x;
    for (int d = 1; d < 64; d <<= 1) {
        const int y = __shfl_up(s, d);
        if (lane >= d) s += y;
    }
    __syncthreads();
    if (lane == 63) waves[w] = s;
    __syncthreads();
    int before = 0, all = 0;
    for (int i = 0; i < kPlan / 64; ++i) {
        if (i == w) before = all;
        all += waves[i];
    }
    *sum = all;
    return before + s - x;
}

// Largest i in [lo, hi) with f(i) <= x, f rising and f(lo) <= x.
template <class F>
__device__ int find(int lo, int hi, int64_t x, F f) {
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (f(mid) <= x) lo = mid; else hi = mid;
    }
    return lo;
}

// One workgroup: groups of rows, their units, and where each share starts.
__global__ __launch_bounds__(kPlan) void plan_kernel(AttendArgs a) {
    __shared__ int waves[kPlan / 64];
    const int tid = threadIdx.x, n = a.n_requests, R = a.rows_per_group;
    const auto bounded = [&](int r) { return min(max(a.row_starts[r], 0), a.n_rows); };
    int base = 0, all = 0;
    for (int r0 = 0; r0 < n; r0 += kPlan) {
        const int r = r0 + tid;
        const int rows = r < n ? max(bounded(r + 1) - bounded(r), 0) : 0;
        const int mine = base + prefix((rows + R - 1) / R, waves, &all);
        if (r < n) a.group_base[r] = min(mine, a.max_groups);
        base += all;
    }
    const int groups = min(base, a.max_groups);
    if (tid == 0) a.group_base[n] = groups;
    __syncthreads();
    const int64_t cap = (int64_t)a.table_width << a.lp;
    int units = 0;
    for (int g0 = 0; g0 < groups; g0 += kPlan) {
        const int g = g0 + tid;
        int mine = 0;
        if (g < groups) {
            const int r = find(0, n, g, [&](int i) { return (int64_t)a.group_base[i]; });
            Group gr;
            gr.request = r;
            gr.row0 = bounded(r) + (g - a.group_base[r]) * R;
            gr.rows = min(R, bounded(r + 1) - gr.row0);
            gr.len = 0;
            // eight at a time: one after the other each would cost a trip to memory
            for (int i = 0; i < gr.rows; i += 8) {
                int x[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] = a.row_lengths[gr.row0 + min(i + j, gr.rows - 1)];
#pragma unroll
                for (int j = 0; j < 8; ++j) gr.len = max(gr.len, x[j]);
            }
            gr.len = (int)min((int64_t)gr.len, cap);
            mine = max((gr.len + a.unit - 1) / a.unit, 1);
            a.groups[g] = gr;
        }
        const int before = units + prefix(mine, waves, &all);
        if (g < groups) a.group_units[g] = before;
        units += all;
    }
    if (tid == 0) a.group_units[groups] = units;
    __syncthreads();
    const int vheads = a.kv_heads * a.parts;
    const int64_t total = (int64_t)units * vheads;
    // a share of fewer than two units is not worth the joining
    const int64_t shares = min((int64_t)a.shares, (total + 1) / 2);
    if (tid == 0) {
        a.total[0] = total;
        a.total[1] = shares;
    }
    for (int w = tid; w < shares; w += kPlan) {
        const int64_t x = share_start(w, total, shares);
        const auto first = [&](int r) { return (int64_t)a.group_units[a.group_base[r]]; };
        const int r = find(0, n, x, [&](int i) { return first(i) * vheads; });
        const int64_t ru = first(r + 1) - first(r), in = x - first(r) * vheads;
        const int head = (int)(in / ru);
        const int64_t y = first(r) + (in - head * ru);
        const int g = find(a.group_base[r], a.group_base[r + 1], y, [&](int i) { return (int64_t)a.group_units[i]; });
        a.starts[w] = int4{g, head, (int)(y - a.group_units[g]), r};
    }
}

// What one call needs, from its sizes.
struct Shape {
    bool prompt;
    int tiles, cols, parts, rows_per_group, unit, shares, splits;
};

Shape shape_of(int n_rows, int n_requests, int heads, int kv_heads, int dim, bool selected, int K, int cus) {
    Shape s = {};
    const int per = heads / kv_heads;
    s.tiles = per > 16 && dim < 256 ? 2 : 1;
    s.cols = 16 * s.tiles;
    s.rows_per_group = 1;
    s.unit = 128;
    s.splits = 1;
    if (selected) {
        s.parts = (per + s.cols - 1) / s.cols;
        const int64_t items = (int64_t)n_rows * kv_heads * s.parts;
        const int units = (K + kSelectedUnit - 1) / kSelectedUnit;
        // rows are split while all workgroups are resident at once, two to a CU (the
        // decode batch: 25.7 us, and 31.0 with two rounds of them)
        while (s.splits < units && items * (s.splits + 1) <= 2 * cus) ++s.splits;
        s.shares = s.splits > 1 ? (int)(items * s.splits) : 0;
        return s;
    }
    // up to three rows to a request each row reads the cache by itself (64 rows of 32
    // requests at 16384 to 32768 tokens: 127 us, and 227 as a
    // prompt; three to a request: 180 and 230).  One rule for the call, in which
    // n_requests is the table's height: a prompt among many single rows, or in a table
    // of many idle requests, is read row by row.
    s.prompt = n_rows > 3 * (int64_t)n_requests;
    if (s.prompt) {
        s.cols = dim == 256 ? 128 : 256;
        s.unit = 64;
        s.rows_per_group = per >= s.cols ? 1 : s.cols / per;
        s.shares = cus;
    } else {
        s.shares = 2 * cus;
    }
    if (s.shares > kMaxShares) s.shares = kMaxShares;
    s.parts = (per + s.cols - 1) / s.cols;
    return s;
}

size_t up(size_t x) { return (x + 255) & ~(size_t)255; }

// Lays the workspace out; bytes in all.
size_t lay_out(AttendArgs *a, char *at, const Shape &s, int n_rows, int n_requests, int dim) {
    char *p = at;
    const auto take = [&](size_t bytes) {
        char *q = p;
        p += up(bytes);
        return q;
    };
    AttendArgs dummy;
    if (!a) a = &dummy;
    a->tickets = (int *)take(PAGED_KV_WORKSPACE_ZEROED);
    a->total = (int64_t *)take(2 * sizeof(int64_t));
    a->starts = (int4 *)take(sizeof(int4) * kMaxShares);
    a->groups = (Group *)take(sizeof(Group) * (size_t)n_rows);
    a->group_units = (int *)take(sizeof(int) * ((size_t)n_rows + 1));
    a->group_base = (int *)take(sizeof(int) * ((size_t)n_requests + 1));
    a->left = (float *)take(sizeof(float) * 2 * (size_t)s.shares * s.cols * (dim + 2));
    return (size_t)(p - at);
}

bool fits(int n_rows, int n_requests, int heads, int kv_heads, int dim) {
    return n_rows >= 0 && n_requests >= 0 && heads >= 1 && kv_heads >= 1 && heads % kv_heads == 0 &&
           (dim == 64 || dim == 128 || dim == 256) && (int64_t)n_rows * heads < 0x7FFFFFFF;
}

int attend(const paged_kv_cache *cache, int act, const void *q, int64_t q_row, int64_t q_head, int heads,
           const int *idx, int K, const int *table, int table_stride, int table_width, const int *row_starts,
           const int *row_request, int n_requests, const int *row_lengths, int n_rows, float scale, void *out,
           float *lse, void *workspace, size_t bytes, void *stream) {
    const bool selected = idx != nullptr || row_request != nullptr;
    const int rc = check_cache(cache, true);
    if (rc != PAGED_KV_OK) return rc;
    if ((act != PAGED_KV_BF16 && act != PAGED_KV_F16) || n_rows < 0 || n_requests < 0 || heads < 1 ||
        heads % cache->n_heads != 0 || table_width < 1 || table_stride < table_width)
        return PAGED_KV_EINVAL;
    if ((selected && K < 1) || !(scale >= 0.0f) || scale > 3e38f) return PAGED_KV_EINVAL;
    if (n_rows == 0) return PAGED_KV_OK;
    if (!q || !out || !row_lengths || (n_requests > 0 && !table) || !aligned16(q) || !aligned16(out) || q_row % 8 ||
        q_head % 8)
        return PAGED_KV_EINVAL;
    if (selected ? !idx || !row_request : !row_starts) return PAGED_KV_EINVAL;
    if (!workspace || ((uintptr_t)workspace & 255) != 0) return PAGED_KV_EINVAL;
    if (!fits(n_rows, n_requests, heads, cache->n_heads, cache->head_dim) ||
        K > 0x7FFFFF00)
        return PAGED_KV_EUNSUPPORTED;
    // tokens, a few tiles past the last, are 32-bit numbers
    const int64_t cap = (int64_t)table_width << log2_page(cache->page);
    if (cap > 0x7FFFFFFF - 8192) return PAGED_KV_EUNSUPPORTED;
    const int cus = device_cus();
    if (cus == 0) return PAGED_KV_EUNSUPPORTED;
    const Shape s = shape_of(n_rows, n_requests, heads, cache->n_heads, cache->head_dim, selected, K, cus);
    // and so are a plan's units
    const int64_t groups = s.prompt ? n_rows / s.rows_per_group + (int64_t)n_requests
                                    : n_rows < kStreamRows ? n_rows : kStreamRows;
    if (!selected && (double)groups * (double)(cap / s.unit + 1) > 2e9) return PAGED_KV_EUNSUPPORTED;
    AttendArgs a = {};
    if (lay_out(&a, (char *)workspace, s, n_rows, n_requests, cache->head_dim) > bytes) return PAGED_KV_EWORKSPACE;
    a.k = (const uint8_t *)cache->k;
    a.v = (const uint8_t *)cache->v;
    a.ks = cache->k_scale;
    a.vs = cache->v_scale;
    a.page_stride = cache->page_stride;
    a.scale_stride = cache->scale_stride;
    a.n_pages = cache->n_pages;
    a.lp = log2_page(cache->page);
    a.kv_heads = cache->n_heads;
    a.q = q;
    a.q_row = q_row;
    a.q_head = q_head;
    a.out = out;
    a.lse = lse;
    a.table = table;
    a.table_stride = table_stride;
    a.table_width = table_width;
    a.row_starts = row_starts;
    a.row_lengths = row_lengths;
    a.n_rows = n_rows;
    a.n_requests = n_requests;
    a.heads = heads;
    a.per = heads / cache->n_heads;
    a.parts = s.parts;
    a.scale2 = scale * 1.4426950408889634f;
    a.rows_per_group = s.rows_per_group;
    a.max_groups = n_rows;
    a.shares = s.shares;
    a.unit = s.unit;
    a.idx = idx;
    a.row_request = row_request;
    a.K = K;
    a.splits = s.splits;
    if (selected) {
        const int64_t grid = (int64_t)n_rows * a.kv_heads * s.parts * s.splits;
        if (grid > 0x7FFFFFFF) return PAGED_KV_EUNSUPPORTED;
        return launch_stream(a, cache->head_dim, act, cache->code, true, s.tiles, (int)grid, stream);
    }
    if (!s.prompt) {
        int rc2 = PAGED_KV_OK;
        for (int r = 0; r < n_rows && rc2 == PAGED_KV_OK; r += kStreamRows) {
            a.row0 = r;
            a.n_rows = n_rows - r < kStreamRows ? n_rows - r : kStreamRows;
            rc2 = launch_stream(a, cache->head_dim, act, cache->code, false, s.tiles, s.shares, stream);
        }
        return rc2;
    }
    const int planned = launch(plan_kernel, dim3(1), dim3(kPlan), stream, a);
    if (planned != PAGED_KV_OK) return planned;
    return launch_prompt(a, cache->head_dim, act, cache->code, s.shares, stream);
}

}  // namespace
}  // namespace paged

extern "C" size_t paged_kv_attend_workspace(int32_t n_rows, int32_t n_requests, int32_t heads, int32_t kv_heads,
                                            int32_t head_dim) {
    using namespace paged;
    const int cus = device_cus();
    if (!fits(n_rows, n_requests, heads, kv_heads, head_dim) || cus == 0) return 0;
    size_t most = 0;
    for (int selected = 0; selected < 2; ++selected) {
        const Shape s = shape_of(n_rows, n_requests, heads, kv_heads, head_dim, selected, 0x7FFFFF00, cus);
        const size_t b = lay_out(nullptr, nullptr, s, n_rows, n_requests, head_dim);
        most = b > most ? b : most;
    }
    return most;
}

extern "C" int paged_kv_attend(const paged_kv_cache *cache, int32_t act, const void *q, int64_t q_row, int64_t q_head,
                               int32_t heads, const int32_t *table, int32_t table_stride, int32_t table_width,
                               const int32_t *row_starts, int32_t n_requests, const int32_t *row_lengths,
                               int32_t n_rows, float scale, void *out, float *lse, void *workspace,
                               size_t workspace_bytes, void *stream) {
    return paged::attend(cache, act, q, q_row, q_head, heads, nullptr, 0, table, table_stride, table_width, row_starts,
                         nullptr, n_requests, row_lengths, n_rows, scale, out, lse, workspace, workspace_bytes, stream);
}

extern "C" int paged_kv_attend_selected(const paged_kv_cache *cache, int32_t act, const void *q, int64_t q_row,
                                        int64_t q_head, int32_t heads, const int32_t *idx, int32_t K,
                                        const int32_t *table, int32_t table_stride, int32_t table_width,
                                        const int32_t *row_request, int32_t n_requests, const int32_t *row_lengths,
                                        int32_t n_rows, float scale, void *out, float *lse, void *workspace,
                                        size_t workspace_bytes, void *stream) {
    if (n_rows > 0 && (!idx || !row_request)) return PAGED_KV_EINVAL;
    static const int32_t none = 0;  // tells the two calls apart where there are no rows
    return paged::attend(cache, act, q, q_row, q_head, heads, idx ? idx : &none, K, table, table_stride, table_width,
                         nullptr, row_request, n_requests, row_lengths, n_rows, scale, out, lse, workspace,
                         workspace_bytes, stream);
}
