// Rows by index: what the kernels of lookups, expert order and weighted sums share, and their launchers.
#pragma once
#include "fg_internal.hpp"

namespace fg {

// x / d for 0 <= x < 2^31 by a product: M = ceil(2^(31+s) / d), s = ceil(log2 d).  M d exceeds 2^(31+s) by less than d <= 2^s, which x times
// stays below 2^(31+s): the quotient is exact, and M < 2^32.
struct Divide {
    uint32_t mul, shift;
    Divide() = default;
    explicit Divide(uint32_t d)
    {
        uint32_t s = 0;
        while (((uint64_t)1 << s) < d) ++s;
        mul = (uint32_t)((((uint64_t)1 << (31 + s)) + d - 1) / d);
        shift = 31 + s;
    }
    __device__ __forceinline__ uint32_t operator()(uint32_t x) const { return (uint32_t)(((uint64_t)x * mul) >> shift); }
};

// A view of rows: `stride` elements from one to the next.
struct RowsIn { const void* at; int64_t stride; };
struct RowsOut { void* at; int64_t stride; };

size_t index_sort_workspace_bytes(int64_t m, int64_t n_rows);
hipError_t launch_index_sort(const int32_t* index, int64_t m, int64_t n_rows, int32_t* order, int32_t* place, int32_t* bounds, void* workspace,
                             hipStream_t stream);

hipError_t launch_lookup(int32_t type, RowsIn table, int64_t n_rows, int64_t c, const int32_t* index, int64_t m, float scale, RowsOut out,
                         hipStream_t stream);
hipError_t launch_dispatch(int32_t type, RowsIn x, int64_t t, int64_t c, const int32_t* place, int32_t k, int64_t n_rows, RowsOut out,
                           hipStream_t stream);
hipError_t launch_combine(int32_t type, RowsIn rows, int64_t n_rows, int64_t c, const int32_t* index, const float* weights, int64_t t, int32_t k,
                          const int32_t* walk /* or NULL */, RowsOut out, hipStream_t stream);

// grad_weights, and with grad_rows.at (every row named once at most) the rows' gradient too
hipError_t launch_combine_grad(int32_t type, RowsIn grad_out, int64_t t, int64_t c, RowsIn rows, int64_t n_rows, const int32_t* index,
                               const float* weights, int32_t k, RowsOut grad_rows, float* grad_weights, hipStream_t stream);

// Rows of grad (entry j of the sorted index stands for row j / fan, times weights[j]) summed by index, times scale; all n_rows are written.
struct RowSums {
    int32_t type, out_type;
    RowsIn grad;
    RowsOut out;
    const int32_t *index, *order, *bounds;
    const float* weights;
    const int32_t* walk;     // the order in which rows are taken, or NULL
    RowsIn rows;             // with grad_weights (sums_with_products): the rows that the entries name
    float* grad_weights;     // or NULL
    int64_t m, n_rows, c;
    int32_t fan;
    float scale;
    int32_t accumulate;
    float* partials;     // row_sums_workspace_bytes()
};
// Widths of rows whose products with the summed rows, the weights' gradient, are made along with the sums.
bool sums_with_products(int32_t type, int64_t c);
size_t row_sums_workspace_bytes(int32_t type, int64_t m, int64_t n_rows, int64_t c, bool products);
hipError_t launch_row_sums(const RowSums& a, hipStream_t stream);

}  // namespace fg
