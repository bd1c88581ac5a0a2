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
// Whether adapters get tiles of 128 rows of their own, in which the product forms the narrow rows itself: where they
// have 64 rows on the mean, or all tiles run at once anyway. Us in one launch, and with a narrow product of its own
// and tiles that adapters share: 300 adapters of 1, 8 and 48 rows, bf16, y 64 -> 896, rank 16 23 and 94, 28 and 33,
// 29 and 40, dx 896 -> 128 34 and 207, 35 and 86, 34 and 55; fp32 y 49 and 138, 66 and 58, 62 and 68, dx 101 and
// 323, 102 and 168, 98 and 126. 4,000 adapters: bf16 y 120 and 116, 188 and 156, 202 and 222, dx 208 and 276, 269
// and 175, 291 and 266; fp32 y 329 and 226, 485 and 353, 580 and 527, dx 601 and 492, 809 and 396, 899 and 691. 100
// of 1,000 rows: bf16 dx 71 and 105, fp32 265 and 298; 800 of 125: y 41 and 66, 101 and 125.
inline bool own_tiles(const RowOrder &o) { return o.n >= 64 * (int64_t)o.G || o.n / 128 + o.G < 512; }
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
