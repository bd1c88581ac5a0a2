// Internal declarations of the row operators: row order by group, grouped products, adapters.
#ifndef CGTP_ROWS_H
#define CGTP_ROWS_H

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "cgtp.h"

namespace cgtp {

// Rows in group order: position p of the sequence is row order[p] (p if order is NULL); group g
// owns the positions [offsets[g], offsets[g + 1]), no group those from offsets[G] on.
struct RowOrder {
    int64_t n;  // rows
    int G;
    const int32_t *offsets, *order;
};

size_t group_rows_bytes(int64_t n_rows, int G);
hipError_t launch_group_rows(int64_t n_rows, int G, const int32_t *ids, int32_t *offsets,
                             int32_t *order, void *ws, hipStream_t s);

// out_i = in_i W_g for the rows of every group, zero (or, with a shared W, in_i W) elsewhere.
struct RowProduct {
    const void *in;
    int64_t in_stride;
    int K;             // width of the input rows
    const void *w;     // per group [K][N], or [N][K] where w_nk
    int64_t w_group;   // elements from one group's weights to the next; 0: shared by all rows
    bool w_nk;
    int N;
    void *out;
    int64_t out_stride;
    // adapters: out_i += scale_g H_i V_g with H from a narrow product before, V per group [r][N] or
    // [N][r] (as W). NULL: none.
    const void *h;
    const void *a;     // instead of h: the adapters' first matrices, [K][r] or [r][K] as W, from which the
                       // kernel forms H itself (where *_takes says so); narrow_scale is its factor
    void *h_out;       // then, if not NULL: H, as a narrow product leaves it
    const void *v;
    int r;
    bool narrow;       // out is a narrow product: in sequence order, fp32 [n][N]
    const float *narrow_scale;  // its factor per group, or NULL
};
hipError_t launch_row_product(int dtype, const RowOrder &o, const RowProduct &p, hipStream_t s);
// The form for short inputs and wide outputs (rows_wide.hip), and whether it covers a product.
bool row_wide_takes(int dtype, const RowProduct &p);
hipError_t launch_row_wide(int dtype, const RowOrder &o, const RowProduct &p, hipStream_t s);
// Products with p.a: whether some form covers one (the launch is that of launch_row_product).
bool adapter_wide_takes(int dtype, const RowOrder &o, const RowProduct &p);
bool adapter_product_takes(int dtype, const RowOrder &o, const RowProduct &p);

// out_g = sum over the rows of group g of a_i b_i^T, [A][B]; with h, the result of a narrow product,
// in place of b: [A][r], or [r][A] where transposed.
struct RowOuter {
    const void *a;
    int64_t a_stride;
    int A;
    const void *b;
    int64_t b_stride;
    int B;
    const void *h;
    int r;
    bool transposed;
    void *out;
};
size_t row_outer_bytes(int dtype, int64_t n_rows, int G, int A, int B);
hipError_t launch_row_outer(int dtype, const RowOrder &o, const RowOuter &p, void *ws,
                            hipStream_t s);
// The forms for groups of few rows (rows_few.hip), up to kFewMean on the mean, and whether that of products
// covers one. Of weight gradients, groups of more than kFewRows rows are left to the tiled kernel.
constexpr int kFewMean = 4, kFewRows = 64;
bool row_few_takes(int dtype, const RowOrder &o, const RowProduct &p);
hipError_t launch_row_few(const RowOrder &o, const RowProduct &p, hipStream_t s);
hipError_t launch_row_outer_few(int dtype, const RowOrder &o, const RowOuter &q, hipStream_t s);
size_t narrow_bytes(int dtype, int64_t n_rows, int N);

}  // namespace cgtp

#endif
