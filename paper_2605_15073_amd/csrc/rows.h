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
    // layers (rows_layer.h): row i is of input row i / per, out_i = act(in W_g + bias_g) + residual_i, and z_i,
    // if not NULL, what the activation took. 0: a plain product.
    int per;
    const void *bias;  // [G][N], or NULL
    int act;           // CGTP_ACT_*
    const void *residual;  // or NULL
    int64_t residual_stride;
    void *z;
    int64_t z_stride;
    int64_t xcd_tiles; // 0, or tiles of an XCD, which follow each other there (rows_index.h)
    bool split_k;      // sums may be split over k (rows_thin.hip); layers' may
    bool out_f32;      // row gradients of rows that share their input: out is fp32 whatever the type
    // row gradients of layers in bf16: row i of the input is in_i act'(slope_z_i), or in_i + slope_z_i where act is
    // kDzHeld, or in_i where NULL
    const void *slope_z;
    int64_t slope_stride;
};
constexpr int kDzHeld = -1;
hipError_t launch_row_product(int dtype, const RowOrder &o, const RowProduct &p, hipStream_t s);
// The form for short inputs and wide outputs (rows_wide.hip), and whether it covers a product.
bool row_wide_takes(int dtype, const RowProduct &p);
hipError_t launch_row_wide(int dtype, const RowOrder &o, const RowProduct &p, hipStream_t s);
// Layers (RowProduct::per) in that form.
bool layer_wide_takes(int dtype, const RowProduct &p);
hipError_t launch_layer_wide(int dtype, const RowOrder &o, const RowProduct &p, hipStream_t s);
hipError_t launch_layer_wide_bf16(const RowOrder &o, const RowProduct &p, hipStream_t s);
hipError_t launch_layer_wide_f32(const RowOrder &o, const RowProduct &p, hipStream_t s);
// The form for long inputs and few tiles (rows_thin.hip), and whether it covers a product.
bool row_thin_takes(int dtype, const RowOrder &o, const RowProduct &p);
hipError_t launch_row_thin(int dtype, const RowOrder &o, const RowProduct &p, hipStream_t s);
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
    int per;     // row i of the order is row i / per of a; 0: row i
    void *sums;  // if not NULL: the sum over the rows of group g of b_i, [G][B], beside out
    // weight gradients of layers in bf16: row i of b is b_i act'(slope_z_i), or b_i + slope_z_i where act is kDzHeld, or
    // b_i where NULL
    const void *slope_z;
    int64_t slope_stride;
    int act;
};
// parts: b is formed from slope_z.
size_t row_outer_bytes(int dtype, int64_t n_rows, int G, int A, int B, bool sums = false, bool parts = false);
hipError_t launch_row_outer(int dtype, const RowOrder &o, const RowOuter &p, void *ws,
                            hipStream_t s);
// The forms for groups of few rows (rows_few.hip), up to kFewMean on the mean, and whether that of products
// covers one. Of weight gradients, groups of more than kFewRows rows are left to the tiled kernel.
constexpr int kFewMean = 4, kFewRows = 64;
bool row_few_takes(int dtype, const RowOrder &o, const RowProduct &p);
hipError_t launch_row_few(const RowOrder &o, const RowProduct &p, hipStream_t s);
hipError_t launch_row_outer_few(int dtype, const RowOrder &o, const RowOuter &q, hipStream_t s);
size_t narrow_bytes(int dtype, int64_t n_rows, int N);

// dz_i = dy_i act'(z_i), rows of N fp32 values at a stride of N, or in bf16 two parts of N values, one behind the other.
hipError_t launch_layer_dz(int dtype, int64_t n, int N, int act, const void *dy, int64_t dy_stride, const void *z,
                           int64_t z_stride, void *dz, hipStream_t s);

// Both products of a narrow layer's gradient in one pass (layer_grad.hip): dx, dw and dbias where not NULL; x for dw
// alone, w for dx alone.
struct LayerGrad {
    const void *x;
    int64_t x_stride;
    int K, per;
    const void *w, *z;
    int64_t z_stride;
    int act;
    const void *dy;
    int64_t dy_stride;
    int N;
    void *dx;
    int64_t dx_stride;
    bool dx_f32;  // dx is fp32 whatever the type
    void *dw, *dbias;
};
bool layer_grad_takes(int dtype, int64_t n, int G, int K, int N);
size_t layer_grad_slots(int dtype, int64_t n, int G, int K, int N);
hipError_t launch_layer_grad(int dtype, const RowOrder &o, const LayerGrad &q, void *slots, hipStream_t s);
// out [G][A][B], and sums [G][B] where not NULL, of the groups of more than one chunk, from their slots.
hipError_t launch_row_join(int dtype, const RowOrder &o, int chunk_rows, int A, int B, const float *slots, void *out,
                           void *sums, hipStream_t s);

// Row t of out (n rows) from rows t k .. t k + k - 1 of y, with a weight each.
struct RowMix {
    int64_t n;
    int k, N;
    const void *y;          // [n k][N]
    int64_t y_stride;
    const float *weights;   // [n][k], or NULL: 1
    const void *residual;   // [n][N], or NULL
    int64_t residual_stride;
    void *out;
    int64_t out_stride;
};
// y_f32: y is fp32 whatever the type of out.
hipError_t launch_mix_rows(int dtype, const RowMix &p, bool y_f32, hipStream_t s);
struct RowMixGrad {
    int64_t n;
    int k, N;
    const void *dout;
    int64_t dout_stride;
    const float *weights;  // or NULL
    const void *y;         // for dweights
    int64_t y_stride;
    void *dy;              // or NULL
    int64_t dy_stride;
    float *dweights;       // or NULL
};
hipError_t launch_mix_rows_grad(int dtype, const RowMixGrad &p, hipStream_t s);

struct RowRoute {
    int64_t n;
    int E, k;
    const void *logits;
    int64_t stride;
    const float *bias;
    int score, blocks, keep;
    bool renorm;
    float scale;
    int32_t *ids;      // written by the choice, read by the gradient
    float *weights;    // the choice's
    const float *dweights;
    void *dlogits;
    int64_t dstride;
};
hipError_t launch_route_rows(int dtype, const RowRoute &p, hipStream_t s);
hipError_t launch_route_rows_grad(int dtype, const RowRoute &p, hipStream_t s);

}  // namespace cgtp

#endif
