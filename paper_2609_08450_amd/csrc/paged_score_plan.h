// How the score kernel for many rows divides query rows and heads into products,
// and how many rows fit a workgroup's LDS.  Plain C++, so that the host can check it.
#pragma once

namespace paged {

// Product rows (query rows x heads) that a workgroup holds in LDS.
constexpr int window_of(int dim) { return dim == 64 ? 512 : 256; }

// Heads of a query row in one product of 32 rows: a power of two up to 16; more
// heads take further products.
constexpr int product_heads(int heads) {
    return heads > 8 ? 16 : heads > 4 ? 8 : heads > 2 ? 4 : heads;
}
constexpr int product_chunks(int heads) { return (heads + product_heads(heads) - 1) / product_heads(heads); }

// Products that `rows` query rows of one request take.
constexpr int products_of(int rows, int heads) {
    const int count = 32 / product_heads(heads);
    return (rows + count - 1) / count * product_chunks(heads);
}

// Query rows of a workgroup: those of as many whole products as it holds.  (Rows
// that fill a product in part take all of its 32 places.)
constexpr int rows_of_window(int dim, int heads) {
    return window_of(dim) / (32 * product_chunks(heads)) * (32 / product_heads(heads));
}

// (A window of one row stands for the kernel of single rows.)
constexpr bool windows_fit() {
    for (int dim = 64; dim <= 128; dim += 64)
        for (int heads = 1; heads <= 128; ++heads) {
            const int rows = rows_of_window(dim, heads);
            if (rows < 2 || 32 * products_of(rows, heads) > window_of(dim)) return false;
        }
    return true;
}
static_assert(windows_fit(), "a window's products fit its LDS");

}  // namespace paged
