// Entry points of the row operators: argument validation, workspaces, launch sequences.
#include "internal.h"
#include "rows.h"

namespace {

using cgtp::report;

size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }

size_t elem(int dtype) { return dtype == CGTP_BF16 ? 2 : 4; }

int hip_fail(hipError_t e, const char *what)
{
    return report(CGTP_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

int check_sizes(int dtype, int64_t n_rows, int n_groups, int n_in, int n_out)
{
    if (dtype != CGTP_F32 && dtype != CGTP_BF16)
        return report(CGTP_ERR_ARG, "dtype %d is neither CGTP_F32 nor CGTP_BF16", dtype);
    if (n_rows < 0 || n_rows > 0x7fffffffLL)
        return report(CGTP_ERR_ARG, "n_rows %lld outside [0, 2^31)", (long long)n_rows);
    if (n_groups < 1 || n_groups > CGTP_MAX_GROUPS)
        return report(CGTP_ERR_ARG, "n_groups %d outside [1, %d]", n_groups, CGTP_MAX_GROUPS);
    if (n_in < 1 || n_in > CGTP_MAX_WIDTH || n_out < 1 || n_out > CGTP_MAX_WIDTH)
        return report(CGTP_ERR_ARG, "widths %d, %d outside [1, %d]", n_in, n_out, CGTP_MAX_WIDTH);
    return CGTP_OK;
}

int check_rank(int rank)
{
    if (rank < 1 || rank > CGTP_MAX_ADAPTER_RANK)
        return report(CGTP_ERR_ARG, "rank %d outside [1, %d]", rank, CGTP_MAX_ADAPTER_RANK);
    return CGTP_OK;
}

int check_ptr(const void *p, const char *name, size_t align)
{
    if (!p) return report(CGTP_ERR_ARG, "%s is NULL", name);
    if (reinterpret_cast<uintptr_t>(p) % align != 0)
        return report(CGTP_ERR_ARG, "%s %p is not aligned to its %zu-byte elements", name, p, align);
    return CGTP_OK;
}

// rows of the given width; n_rows 0 needs no pointer
int check_rows(const void *p, const char *name, int64_t stride, int width, int64_t n_rows, size_t es)
{
    if (n_rows == 0) return CGTP_OK;
    if (stride < width || stride > ((int64_t)1 << 31))
        return report(CGTP_ERR_ARG, "%s_stride %lld outside [%d, 2^31]", name, (long long)stride, width);
    return check_ptr(p, name, es);
}

int check_ws(void *ws, size_t ws_bytes, size_t need)
{
    if (need == 0) return CGTP_OK;
    if (!ws) return report(CGTP_ERR_WORKSPACE, "no workspace, %zu bytes needed", need);
    if (reinterpret_cast<uintptr_t>(ws) % 256 != 0)
        return report(CGTP_ERR_ARG, "workspace %p is not 256-byte aligned", ws);
    if (ws_bytes < need)
        return report(CGTP_ERR_WORKSPACE, "workspace of %zu bytes, %zu needed", ws_bytes, need);
    return CGTP_OK;
}

// offsets are always read; order may be NULL
int check_order(const int32_t *offsets, const int32_t *order)
{
    int st = check_ptr(offsets, "offsets", 4);
    if (st == CGTP_OK && order) st = check_ptr(order, "order", 4);
    return st;
}

size_t grouped_grad_bytes(int dtype, int64_t n, int G, int n_in, int n_out)
{
    return cgtp::row_outer_bytes(dtype, n, G, n_in, n_out);
}

size_t adapter_bytes(int dtype, int64_t n, int rank)
{
    return align256(cgtp::narrow_bytes(dtype, n, rank));
}

// The product y of adapters, but for the pointers: what forms cover it does not depend on them.
cgtp::RowProduct adapter_product(int n_in, int n_out, int rank, const void *a)
{
    cgtp::RowProduct p{};
    p.K = n_in;
    p.N = n_out;
    p.a = a;
    p.r = rank;
    return p;
}

// h, where the product does not form it itself
size_t adapter_forward_bytes(int dtype, int64_t n, int G, const cgtp::RowProduct &p)
{
    return cgtp::adapter_wide_takes(dtype, {n, G, nullptr, nullptr}, p) ? 0 : adapter_bytes(dtype, n, p.r);
}

// h and u, then the sums of da and of db, which use the same space one after the other
size_t adapter_grad_bytes(int dtype, int64_t n, int G, int n_in, int n_out, int rank)
{
    const size_t sa = cgtp::row_outer_bytes(dtype, n, G, n_in, rank);
    const size_t sb = cgtp::row_outer_bytes(dtype, n, G, n_out, rank);
    return 2 * adapter_bytes(dtype, n, rank) + (sa > sb ? sa : sb);
}

}  // namespace

#define CGTP_TRY(call)                        \
    do {                                      \
        const int st_ = (call);               \
        if (st_ != CGTP_OK) return st_;       \
    } while (0)

extern "C" int cgtp_group_rows_bytes(int64_t n_rows, int n_groups, size_t *bytes)
{
    cgtp::clear_error();
    CGTP_TRY(check_sizes(CGTP_F32, n_rows, n_groups, 1, 1));
    if (!bytes) return report(CGTP_ERR_ARG, "bytes is NULL");
    *bytes = cgtp::group_rows_bytes(n_rows, n_groups);
    return CGTP_OK;
}

extern "C" int cgtp_group_rows(int64_t n_rows, int n_groups, const int32_t *ids, int32_t *offsets,
                               int32_t *order, void *workspace, size_t ws_bytes, void *stream)
{
    cgtp::clear_error();
    CGTP_TRY(check_sizes(CGTP_F32, n_rows, n_groups, 1, 1));
    CGTP_TRY(check_ptr(offsets, "offsets", 4));
    if (n_rows > 0) {
        CGTP_TRY(check_ptr(ids, "ids", 4));
        CGTP_TRY(check_ptr(order, "order", 4));
    }
    CGTP_TRY(check_ws(workspace, ws_bytes, cgtp::group_rows_bytes(n_rows, n_groups)));
    const hipError_t e = cgtp::launch_group_rows(n_rows, n_groups, ids, offsets, order, workspace,
                                                 static_cast<hipStream_t>(stream));
    return e == hipSuccess ? CGTP_OK : hip_fail(e, "group rows");
}

extern "C" int cgtp_grouped_linear(int dtype, int64_t n_rows, int n_groups, int n_in, int n_out,
                                   const int32_t *offsets, const int32_t *order, const void *x,
                                   int64_t x_stride, const void *w, void *y, int64_t y_stride,
                                   void *stream)
{
    cgtp::clear_error();
    CGTP_TRY(check_sizes(dtype, n_rows, n_groups, n_in, n_out));
    if (n_rows == 0) return CGTP_OK;
    const size_t es = elem(dtype);
    CGTP_TRY(check_order(offsets, order));
    CGTP_TRY(check_rows(x, "x", x_stride, n_in, n_rows, es));
    CGTP_TRY(check_ptr(w, "w", es));
    CGTP_TRY(check_rows(y, "y", y_stride, n_out, n_rows, es));
    cgtp::RowProduct p{};
    p.in = x;
    p.in_stride = x_stride;
    p.K = n_in;
    p.w = w;
    p.w_group = (int64_t)n_in * n_out;
    p.N = n_out;
    p.out = y;
    p.out_stride = y_stride;
    const hipError_t e = cgtp::launch_row_product(dtype, {n_rows, n_groups, offsets, order}, p,
                                                  static_cast<hipStream_t>(stream));
    return e == hipSuccess ? CGTP_OK : hip_fail(e, "grouped product");
}

extern "C" int cgtp_grouped_linear_grad_bytes(int dtype, int64_t n_rows, int n_groups, int n_in,
                                              int n_out, size_t *bytes)
{
    cgtp::clear_error();
    CGTP_TRY(check_sizes(dtype, n_rows, n_groups, n_in, n_out));
    if (!bytes) return report(CGTP_ERR_ARG, "bytes is NULL");
    *bytes = grouped_grad_bytes(dtype, n_rows, n_groups, n_in, n_out);
    return CGTP_OK;
}

extern "C" int cgtp_grouped_linear_grad(int dtype, int64_t n_rows, int n_groups, int n_in,
                                        int n_out, const int32_t *offsets, const int32_t *order,
                                        const void *x, int64_t x_stride, const void *w,
                                        const void *dy, int64_t dy_stride, void *dx,
                                        int64_t dx_stride, void *dw, void *workspace,
                                        size_t ws_bytes, void *stream)
{
    cgtp::clear_error();
    CGTP_TRY(check_sizes(dtype, n_rows, n_groups, n_in, n_out));
    if (!dw && n_rows == 0) return CGTP_OK;
    if (!dx && !dw) return report(CGTP_ERR_ARG, "dx and dw are both NULL");
    const size_t es = elem(dtype);
    CGTP_TRY(check_order(offsets, order));
    CGTP_TRY(check_rows(dy, "dy", dy_stride, n_out, n_rows, es));
    if (dx) {
        CGTP_TRY(check_ptr(w, "w", es));
        CGTP_TRY(check_rows(dx, "dx", dx_stride, n_in, n_rows, es));
    }
    if (dw) {
        CGTP_TRY(check_rows(x, "x", x_stride, n_in, n_rows, es));
        CGTP_TRY(check_ptr(dw, "dw", es));
        CGTP_TRY(check_ws(workspace, ws_bytes,
                          grouped_grad_bytes(dtype, n_rows, n_groups, n_in, n_out)));
    }
    const cgtp::RowOrder o{n_rows, n_groups, offsets, order};
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (dx && n_rows > 0) {
        cgtp::RowProduct p{};
        p.in = dy;
        p.in_stride = dy_stride;
        p.K = n_out;
        p.w = w;
        p.w_group = (int64_t)n_in * n_out;
        p.w_nk = true;
        p.N = n_in;
        p.out = dx;
        p.out_stride = dx_stride;
        const hipError_t e = cgtp::launch_row_product(dtype, o, p, s);
        if (e != hipSuccess) return hip_fail(e, "row gradient");
    }
    if (dw) {
        cgtp::RowOuter q{};
        q.a = x;
        q.a_stride = x_stride;
        q.A = n_in;
        q.b = dy;
        q.b_stride = dy_stride;
        q.B = n_out;
        q.out = dw;
        const hipError_t e = cgtp::launch_row_outer(dtype, o, q, workspace, s);
        if (e != hipSuccess) return hip_fail(e, "weight gradient");
    }
    return CGTP_OK;
}

extern "C" int cgtp_adapter_linear_bytes(int dtype, int64_t n_rows, int n_groups, int n_in,
                                         int n_out, int rank, size_t *bytes)
{
    cgtp::clear_error();
    CGTP_TRY(check_sizes(dtype, n_rows, n_groups, n_in, n_out));
    CGTP_TRY(check_rank(rank));
    if (!bytes) return report(CGTP_ERR_ARG, "bytes is NULL");
    const cgtp::RowProduct p = adapter_product(n_in, n_out, rank, bytes);  // a: any pointer, for "adapters"
    *bytes = adapter_forward_bytes(dtype, n_rows, n_groups, p);
    return CGTP_OK;
}

extern "C" int cgtp_adapter_linear(int dtype, int64_t n_rows, int n_groups, int n_in, int n_out,
                                   int rank, const int32_t *offsets, const int32_t *order,
                                   const void *x, int64_t x_stride, const void *w, const void *a,
                                   const void *b, const float *scale, void *y, int64_t y_stride,
                                   void *workspace, size_t ws_bytes, void *stream)
{
    cgtp::clear_error();
    CGTP_TRY(check_sizes(dtype, n_rows, n_groups, n_in, n_out));
    CGTP_TRY(check_rank(rank));
    if (n_rows == 0) return CGTP_OK;
    const size_t es = elem(dtype);
    CGTP_TRY(check_order(offsets, order));
    CGTP_TRY(check_rows(x, "x", x_stride, n_in, n_rows, es));
    CGTP_TRY(check_ptr(w, "w", es));
    CGTP_TRY(check_ptr(a, "a", es));
    CGTP_TRY(check_ptr(b, "b", es));
    if (scale) CGTP_TRY(check_ptr(scale, "scale", 4));
    CGTP_TRY(check_rows(y, "y", y_stride, n_out, n_rows, es));
    cgtp::RowProduct p = adapter_product(n_in, n_out, rank, a);
    CGTP_TRY(check_ws(workspace, ws_bytes, adapter_forward_bytes(dtype, n_rows, n_groups, p)));
    const cgtp::RowOrder o{n_rows, n_groups, offsets, order};
    const hipStream_t s = static_cast<hipStream_t>(stream);
    p.in = x;
    p.in_stride = x_stride;
    p.w = w;
    p.out = y;
    p.out_stride = y_stride;
    p.v = b;
    p.narrow_scale = scale;
    hipError_t e;
    if (cgtp::adapter_wide_takes(dtype, o, p)) {
        e = cgtp::launch_row_product(dtype, o, p, s);
        return e == hipSuccess ? CGTP_OK : hip_fail(e, "adapter product");
    }
    cgtp::RowProduct q{};  // h = scale a^T x
    q.in = x;
    q.in_stride = x_stride;
    q.K = n_in;
    q.w = a;
    q.w_group = (int64_t)n_in * rank;
    q.N = rank;
    q.out = workspace;
    q.narrow = true;
    q.narrow_scale = scale;
    e = cgtp::launch_row_product(dtype, o, q, s);
    if (e != hipSuccess) return hip_fail(e, "adapter's first product");
    p.a = nullptr;
    p.narrow_scale = nullptr;
    p.h = workspace;
    e = cgtp::launch_row_product(dtype, o, p, s);
    return e == hipSuccess ? CGTP_OK : hip_fail(e, "shared product");
}

extern "C" int cgtp_adapter_linear_grad_bytes(int dtype, int64_t n_rows, int n_groups, int n_in,
                                              int n_out, int rank, size_t *bytes)
{
    cgtp::clear_error();
    CGTP_TRY(check_sizes(dtype, n_rows, n_groups, n_in, n_out));
    CGTP_TRY(check_rank(rank));
    if (!bytes) return report(CGTP_ERR_ARG, "bytes is NULL");
    *bytes = adapter_grad_bytes(dtype, n_rows, n_groups, n_in, n_out, rank);
    return CGTP_OK;
}

extern "C" int cgtp_adapter_linear_grad(int dtype, int64_t n_rows, int n_groups, int n_in,
                                        int n_out, int rank, const int32_t *offsets,
                                        const int32_t *order, const void *x, int64_t x_stride,
                                        const void *w, const void *a, const void *b,
                                        const float *scale, const void *dy, int64_t dy_stride,
                                        void *dx, int64_t dx_stride, void *da, void *db,
                                        void *workspace, size_t ws_bytes, void *stream)
{
    cgtp::clear_error();
    CGTP_TRY(check_sizes(dtype, n_rows, n_groups, n_in, n_out));
    CGTP_TRY(check_rank(rank));
    if (!da && !db && n_rows == 0) return CGTP_OK;
    if (!dx && !da && !db) return report(CGTP_ERR_ARG, "dx, da and db are all NULL");
    const size_t es = elem(dtype);
    CGTP_TRY(check_order(offsets, order));
    CGTP_TRY(check_rows(x, "x", x_stride, n_in, n_rows, es));
    CGTP_TRY(check_ptr(w, "w", es));
    CGTP_TRY(check_ptr(a, "a", es));
    CGTP_TRY(check_ptr(b, "b", es));
    if (scale) CGTP_TRY(check_ptr(scale, "scale", 4));
    CGTP_TRY(check_rows(dy, "dy", dy_stride, n_out, n_rows, es));
    if (dx) CGTP_TRY(check_rows(dx, "dx", dx_stride, n_in, n_rows, es));
    if (da) CGTP_TRY(check_ptr(da, "da", es));
    if (db) CGTP_TRY(check_ptr(db, "db", es));
    CGTP_TRY(check_ws(workspace, ws_bytes,
                      adapter_grad_bytes(dtype, n_rows, n_groups, n_in, n_out, rank)));
    const cgtp::RowOrder o{n_rows, n_groups, offsets, order};
    const hipStream_t s = static_cast<hipStream_t>(stream);
    char *const h = static_cast<char *>(workspace);
    char *const u = h + adapter_bytes(dtype, n_rows, rank);
    char *const sums = u + adapter_bytes(dtype, n_rows, rank);
    hipError_t e;
    cgtp::RowProduct px{};  // dx = w dy + a u
    px.in = dy;
    px.in_stride = dy_stride;
    px.K = n_out;
    px.w = w;
    px.w_nk = true;
    px.N = n_in;
    px.out = dx;
    px.out_stride = dx_stride;
    px.a = b;
    px.h_out = u;
    px.v = a;
    px.r = rank;
    px.narrow_scale = scale;
    const bool together = dx && n_rows > 0 && cgtp::adapter_product_takes(dtype, o, px);
    if ((dx || da) && n_rows > 0 && !together) {  // u = scale b dy
        cgtp::RowProduct p{};
        p.in = dy;
        p.in_stride = dy_stride;
        p.K = n_out;
        p.w = b;
        p.w_group = (int64_t)rank * n_out;
        p.w_nk = true;
        p.N = rank;
        p.out = u;
        p.narrow = true;
        p.narrow_scale = scale;
        e = cgtp::launch_row_product(dtype, o, p, s);
        if (e != hipSuccess) return hip_fail(e, "adapter's row gradient");
    }
    if (db && n_rows > 0) {  // h = scale a^T x
        cgtp::RowProduct p{};
        p.in = x;
        p.in_stride = x_stride;
        p.K = n_in;
        p.w = a;
        p.w_group = (int64_t)n_in * rank;
        p.N = rank;
        p.out = h;
        p.narrow = true;
        p.narrow_scale = scale;
        e = cgtp::launch_row_product(dtype, o, p, s);
        if (e != hipSuccess) return hip_fail(e, "adapter's first product");
    }
    if (dx && n_rows > 0) {
        if (!together) {
            px.a = nullptr;
            px.h_out = nullptr;
            px.narrow_scale = nullptr;
            px.h = u;
        }
        e = cgtp::launch_row_product(dtype, o, px, s);
        if (e != hipSuccess) return hip_fail(e, "row gradient");
    }
    if (da) {
        cgtp::RowOuter q{};
        q.a = x;
        q.a_stride = x_stride;
        q.A = n_in;
        q.h = u;
        q.r = rank;
        q.out = da;
        e = cgtp::launch_row_outer(dtype, o, q, sums, s);
        if (e != hipSuccess) return hip_fail(e, "gradient of a");
    }
    if (db) {
        cgtp::RowOuter q{};
        q.a = dy;
        q.a_stride = dy_stride;
        q.A = n_out;
        q.h = h;
        q.r = rank;
        q.transposed = true;
        q.out = db;
        e = cgtp::launch_row_outer(dtype, o, q, sums, s);
        if (e != hipSuccess) return hip_fail(e, "gradient of b");
    }
    return CGTP_OK;
}
