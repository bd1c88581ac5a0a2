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

// ---------------------------------------------------------------- layers, routing, joining

namespace {

int check_per_row(int64_t n_rows, int per_row)
{
    if (per_row < 1 || per_row > CGTP_MAX_PER_ROW)
        return report(CGTP_ERR_ARG, "per_row %d outside [1, %d]", per_row, CGTP_MAX_PER_ROW);
    if (n_rows % per_row != 0)
        return report(CGTP_ERR_ARG, "n_rows %lld is no multiple of per_row %d", (long long)n_rows, per_row);
    return CGTP_OK;
}

int check_activation(int activation)
{
    if (activation < CGTP_ACT_NONE || activation > CGTP_ACT_RELU)
        return report(CGTP_ERR_ARG, "activation %d is not known", activation);
    return CGTP_OK;
}

// Whether dz is formed in a pass of its own, 4 bytes a value: fp32, or two bf16 parts. In bf16 the products form it themselves
// where each of them does so once, up to 128 inputs: they read dy and z in place of the parts. Us of all gradients with the
// pass and without, silu: 261,764 rows, 128 -> 448, 492 and 428, 525,308, 64 -> 128, 247 and 168, 262,144, 128 -> 128, 155 and
// 133; 100,000, 136 -> 64, 66 and 77, 192 -> 192 126 and 139, 60,000, 1344 -> 448, 503 and 759.
bool dz_apart(int dtype, int n_in, int activation)
{
    return activation != CGTP_ACT_NONE && (dtype == CGTP_F32 || n_in > 128);
}

// dz where it has a pass of its own, the row gradients (per_row 1 where they are not asked for) in fp32 where rows share
// their input, and sums of the weight gradients. The form of narrow layers has no dz, whatever it is asked for.
struct LayerGradBytes {
    size_t dz, rows, sums;
    size_t all() const { return dz + rows + sums; }
};

LayerGradBytes layer_grad_bytes(int dtype, int64_t n, int G, int n_in, int n_out, int per_row, int activation)
{
    const size_t rows = per_row == 1 ? 0 : align256((size_t)n * n_in * 4);
    if (cgtp::layer_grad_takes(dtype, n, G, n_in, n_out)) return {0, rows, cgtp::layer_grad_slots(dtype, n, G, n_in, n_out)};
    const bool parts = dtype == CGTP_BF16 && activation != CGTP_ACT_NONE;
    const size_t all = cgtp::row_outer_bytes(dtype, n, G, n_in, n_out, true, parts);
    const size_t alone = cgtp::row_outer_bytes(dtype, n, G, 1, n_out, true, parts);  // dbias
    return {dz_apart(dtype, n_in, activation) ? align256((size_t)n * n_out * 4) : 0, rows, all > alone ? all : alone};
}

int check_score(int score, int renormalize, float scale)
{
    if (score != CGTP_SCORE_SOFTMAX && score != CGTP_SCORE_SIGMOID)
        return report(CGTP_ERR_ARG, "score %d is neither CGTP_SCORE_SOFTMAX nor CGTP_SCORE_SIGMOID", score);
    if (renormalize != 0 && renormalize != 1) return report(CGTP_ERR_ARG, "renormalize %d is neither 0 nor 1", renormalize);
    if (!__builtin_isfinite(scale)) return report(CGTP_ERR_ARG, "scale %g is not finite", scale);
    return CGTP_OK;
}

int check_route(int dtype, int64_t n_rows, int n_experts, int top_k)
{
    CGTP_TRY(check_sizes(dtype, n_rows, n_experts, 1, 1));
    if (top_k < 1 || top_k > CGTP_MAX_TOP_K || top_k > n_experts)
        return report(CGTP_ERR_ARG, "top_k %d outside [1, %d] or above %d experts", top_k, CGTP_MAX_TOP_K, n_experts);
    if (n_rows * top_k > 0x7fffffffLL)
        return report(CGTP_ERR_ARG, "%lld rows of %d experts: 2^31 pairs or more", (long long)n_rows, top_k);
    return CGTP_OK;
}

}  // namespace

extern "C" int cgtp_route_rows(int dtype, int64_t n_rows, int n_experts, int top_k, const void *logits,
                               int64_t logits_stride, const float *bias, int score, int n_blocks, int keep_blocks,
                               int renormalize, float scale, int32_t *ids, float *weights, void *stream)
{
    cgtp::clear_error();
    CGTP_TRY(check_route(dtype, n_rows, n_experts, top_k));
    CGTP_TRY(check_score(score, renormalize, scale));
    if (n_blocks < 1 || n_blocks > CGTP_MAX_ROUTE_BLOCKS || n_experts % n_blocks != 0)
        return report(CGTP_ERR_ARG, "n_blocks %d outside [1, %d] or no divisor of %d experts", n_blocks,
                      CGTP_MAX_ROUTE_BLOCKS, n_experts);
    if (keep_blocks < 1 || keep_blocks > n_blocks)
        return report(CGTP_ERR_ARG, "keep_blocks %d outside [1, %d]", keep_blocks, n_blocks);
    if (top_k > n_experts / n_blocks * keep_blocks)
        return report(CGTP_ERR_ARG, "top_k %d above the %d experts of the blocks kept", top_k,
                      n_experts / n_blocks * keep_blocks);
    if (n_rows == 0) return CGTP_OK;
    CGTP_TRY(check_rows(logits, "logits", logits_stride, n_experts, n_rows, elem(dtype)));
    if (bias) CGTP_TRY(check_ptr(bias, "bias", 4));
    CGTP_TRY(check_ptr(ids, "ids", 4));
    CGTP_TRY(check_ptr(weights, "weights", 4));
    cgtp::RowRoute p{};
    p.n = n_rows;
    p.E = n_experts;
    p.k = top_k;
    p.logits = logits;
    p.stride = logits_stride;
    p.bias = bias;
    p.score = score;
    p.blocks = keep_blocks == n_blocks ? 1 : n_blocks;  // all are kept
    p.keep = keep_blocks;
    p.renorm = renormalize != 0;
    p.scale = scale;
    p.ids = ids;
    p.weights = weights;
    const hipError_t e = cgtp::launch_route_rows(dtype, p, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? CGTP_OK : hip_fail(e, "route");
}

extern "C" int cgtp_route_rows_grad(int dtype, int64_t n_rows, int n_experts, int top_k, const void *logits,
                                    int64_t logits_stride, const int32_t *ids, const float *dweights, int score,
                                    int renormalize, float scale, void *dlogits, int64_t dlogits_stride, void *stream)
{
    cgtp::clear_error();
    CGTP_TRY(check_route(dtype, n_rows, n_experts, top_k));
    CGTP_TRY(check_score(score, renormalize, scale));
    if (n_rows == 0) return CGTP_OK;
    const size_t es = elem(dtype);
    CGTP_TRY(check_rows(logits, "logits", logits_stride, n_experts, n_rows, es));
    CGTP_TRY(check_ptr(ids, "ids", 4));
    CGTP_TRY(check_ptr(dweights, "dweights", 4));
    CGTP_TRY(check_rows(dlogits, "dlogits", dlogits_stride, n_experts, n_rows, es));
    cgtp::RowRoute p{};
    p.n = n_rows;
    p.E = n_experts;
    p.k = top_k;
    p.logits = logits;
    p.stride = logits_stride;
    p.score = score;
    p.renorm = renormalize != 0;
    p.scale = scale;
    p.ids = const_cast<int32_t *>(ids);
    p.dweights = dweights;
    p.dlogits = dlogits;
    p.dstride = dlogits_stride;
    const hipError_t e = cgtp::launch_route_rows_grad(dtype, p, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? CGTP_OK : hip_fail(e, "route gradient");
}

extern "C" int cgtp_grouped_layer(int dtype, int64_t n_rows, int n_groups, int n_in, int n_out, int per_row,
                                  const int32_t *offsets, const int32_t *order, const void *x, int64_t x_stride,
                                  const void *w, const void *bias, int activation, const void *residual,
                                  int64_t residual_stride, void *y, int64_t y_stride, void *z, int64_t z_stride,
                                  void *stream)
{
    cgtp::clear_error();
    CGTP_TRY(check_sizes(dtype, n_rows, n_groups, n_in, n_out));
    CGTP_TRY(check_per_row(n_rows, per_row));
    CGTP_TRY(check_activation(activation));
    if (n_rows == 0) return CGTP_OK;
    const size_t es = elem(dtype);
    CGTP_TRY(check_order(offsets, order));
    CGTP_TRY(check_rows(x, "x", x_stride, n_in, n_rows, es));
    CGTP_TRY(check_ptr(w, "w", es));
    if (bias) CGTP_TRY(check_ptr(bias, "bias", es));
    if (residual) CGTP_TRY(check_rows(residual, "residual", residual_stride, n_out, n_rows, es));
    CGTP_TRY(check_rows(y, "y", y_stride, n_out, n_rows, es));
    if (z) CGTP_TRY(check_rows(z, "z", z_stride, n_out, n_rows, es));
    cgtp::RowProduct p{};
    p.in = x;
    p.in_stride = x_stride;
    p.K = n_in;
    p.w = w;
    p.w_group = (int64_t)n_in * n_out;
    p.N = n_out;
    p.out = y;
    p.out_stride = y_stride;
    p.per = per_row;
    p.bias = bias;
    p.act = activation;
    p.residual = residual;
    p.residual_stride = residual_stride;
    p.z = z;
    p.z_stride = z_stride;
    p.xcd_tiles = 1;
    const hipError_t e = cgtp::launch_row_product(dtype, {n_rows, n_groups, offsets, order}, p,
                                                  static_cast<hipStream_t>(stream));
    return e == hipSuccess ? CGTP_OK : hip_fail(e, "grouped layer");
}

extern "C" int cgtp_grouped_layer_grad_bytes(int dtype, int64_t n_rows, int n_groups, int n_in, int n_out, int per_row,
                                             int activation, size_t *bytes)
{
    cgtp::clear_error();
    CGTP_TRY(check_sizes(dtype, n_rows, n_groups, n_in, n_out));
    CGTP_TRY(check_per_row(n_rows, per_row));
    CGTP_TRY(check_activation(activation));
    if (!bytes) return report(CGTP_ERR_ARG, "bytes is NULL");
    *bytes = layer_grad_bytes(dtype, n_rows, n_groups, n_in, n_out, per_row, activation).all();
    return CGTP_OK;
}

extern "C" int cgtp_grouped_layer_grad(int dtype, int64_t n_rows, int n_groups, int n_in, int n_out, int per_row,
                                       const int32_t *offsets, const int32_t *order, const void *x, int64_t x_stride,
                                       const void *w, const void *z, int64_t z_stride, int activation, const void *dy,
                                       int64_t dy_stride, void *dx, int64_t dx_stride, void *dw, void *dbias,
                                       void *workspace, size_t ws_bytes, void *stream)
{
    cgtp::clear_error();
    CGTP_TRY(check_sizes(dtype, n_rows, n_groups, n_in, n_out));
    CGTP_TRY(check_per_row(n_rows, per_row));
    CGTP_TRY(check_activation(activation));
    if (!dw && !dbias && n_rows == 0) return CGTP_OK;
    if (!dx && !dw && !dbias) return report(CGTP_ERR_ARG, "dx, dw and dbias are all NULL");
    const size_t es = elem(dtype);
    CGTP_TRY(check_order(offsets, order));
    CGTP_TRY(check_rows(dy, "dy", dy_stride, n_out, n_rows, es));
    if (activation != CGTP_ACT_NONE) CGTP_TRY(check_rows(z, "z", z_stride, n_out, n_rows, es));
    if (dx) {
        CGTP_TRY(check_ptr(w, "w", es));
        CGTP_TRY(check_rows(dx, "dx", dx_stride, n_in, n_rows, es));
    }
    if (dw) {
        CGTP_TRY(check_rows(x, "x", x_stride, n_in, n_rows, es));
        CGTP_TRY(check_ptr(dw, "dw", es));
    }
    if (dbias) CGTP_TRY(check_ptr(dbias, "dbias", es));
    const LayerGradBytes need = layer_grad_bytes(dtype, n_rows, n_groups, n_in, n_out, dx ? per_row : 1, activation);
    CGTP_TRY(check_ws(workspace, ws_bytes, need.all()));
    const cgtp::RowOrder o{n_rows, n_groups, offsets, order};
    const hipStream_t s = static_cast<hipStream_t>(stream);
    char *const dz = static_cast<char *>(workspace), *const rows = dz + need.dz, *const sums = rows + need.rows;
    hipError_t e;
    auto add_shared = [&]() {  // dx from the rows that share an input
        cgtp::RowMix m{};
        m.n = n_rows / per_row;
        m.k = per_row;
        m.N = n_in;
        m.y = rows;
        m.y_stride = n_in;
        m.out = dx;
        m.out_stride = dx_stride;
        return cgtp::launch_mix_rows(dtype, m, true, s);
    };
    if (cgtp::layer_grad_takes(dtype, n_rows, n_groups, n_in, n_out)) {
        cgtp::LayerGrad q{};
        q.x = x;
        q.x_stride = x_stride;
        q.K = n_in;
        q.per = per_row;
        q.w = w;
        q.z = z;
        q.z_stride = z_stride;
        q.act = activation;
        q.dy = dy;
        q.dy_stride = dy_stride;
        q.N = n_out;
        q.dx = dx && per_row > 1 ? rows : dx;
        q.dx_stride = per_row > 1 ? n_in : dx_stride;
        q.dx_f32 = per_row > 1;
        q.dw = dw;
        q.dbias = dbias;
        e = cgtp::launch_layer_grad(dtype, o, q, sums, s);
        if (e != hipSuccess) return hip_fail(e, "layer gradient");
        if (dx && per_row > 1) e = add_shared();
        return e == hipSuccess ? CGTP_OK : hip_fail(e, "row gradient's sum");
    }
    // dz, one of the products' operands: dy itself, in a pass of its own, or in bf16 from dy and z within the products
    const void *b = dy, *slope_z = nullptr;
    int64_t b_stride = dy_stride, slope_stride = 0;
    int act = activation;
    if (need.dz > 0 && n_rows > 0) {
        e = cgtp::launch_layer_dz(dtype, n_rows, n_out, activation, dy, dy_stride, z, z_stride, dz, s);
        if (e != hipSuccess) return hip_fail(e, "activation's gradient");
        b = dz;
        b_stride = n_out;
        if (dtype == CGTP_BF16) {
            slope_z = dz + (size_t)n_out * es;
            b_stride = slope_stride = 2 * (int64_t)n_out;
            act = cgtp::kDzHeld;
        }
    } else if (activation != CGTP_ACT_NONE && dtype == CGTP_BF16) {
        slope_z = z;
        slope_stride = z_stride;
    }
    if (dx && n_rows > 0) {
        cgtp::RowProduct p{};
        p.in = b;
        p.in_stride = b_stride;
        p.K = n_out;
        p.w = w;
        p.w_group = (int64_t)n_in * n_out;
        p.w_nk = true;
        p.N = n_in;
        p.out = per_row > 1 ? rows : dx;
        p.out_stride = per_row > 1 ? n_in : dx_stride;
        p.out_f32 = per_row > 1 && dtype == CGTP_BF16;
        p.split_k = true;
        p.act = act;
        p.slope_z = slope_z;
        p.slope_stride = slope_stride;
        e = cgtp::launch_row_product(dtype, o, p, s);
        if (e != hipSuccess) return hip_fail(e, "row gradient");
        if (per_row > 1) {
            e = add_shared();
            if (e != hipSuccess) return hip_fail(e, "row gradient's sum");
        }
    }
    if (dw || dbias) {
        cgtp::RowOuter q{};
        q.a = dw ? x : b;
        q.a_stride = dw ? x_stride : b_stride;
        q.A = dw ? n_in : 1;  // no products are asked for: those with b's first column, which are not stored
        q.b = b;
        q.b_stride = b_stride;
        q.B = n_out;
        q.out = dw;
        q.per = dw ? per_row : 1;
        q.sums = dbias;
        q.act = act;
        q.slope_z = slope_z;
        q.slope_stride = slope_stride;
        e = cgtp::launch_row_outer(dtype, o, q, sums, s);
        if (e != hipSuccess) return hip_fail(e, "weight gradient");
    }
    return CGTP_OK;
}

extern "C" int cgtp_mix_rows(int dtype, int64_t n_rows, int per_row, int width, const void *y, int64_t y_stride,
                             const float *weights, const void *residual, int64_t residual_stride, void *out,
                             int64_t out_stride, void *stream)
{
    cgtp::clear_error();
    CGTP_TRY(check_sizes(dtype, n_rows, 1, width, width));
    CGTP_TRY(check_per_row(0, per_row));
    if (n_rows * per_row > 0x7fffffffLL)
        return report(CGTP_ERR_ARG, "%lld times %d rows: 2^31 or more", (long long)n_rows, per_row);
    if (n_rows == 0) return CGTP_OK;
    const size_t es = elem(dtype);
    CGTP_TRY(check_rows(y, "y", y_stride, width, n_rows, es));
    if (weights) CGTP_TRY(check_ptr(weights, "weights", 4));
    if (residual) CGTP_TRY(check_rows(residual, "residual", residual_stride, width, n_rows, es));
    CGTP_TRY(check_rows(out, "out", out_stride, width, n_rows, es));
    cgtp::RowMix p{};
    p.n = n_rows;
    p.k = per_row;
    p.N = width;
    p.y = y;
    p.y_stride = y_stride;
    p.weights = weights;
    p.residual = residual;
    p.residual_stride = residual_stride;
    p.out = out;
    p.out_stride = out_stride;
    const hipError_t e = cgtp::launch_mix_rows(dtype, p, false, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? CGTP_OK : hip_fail(e, "mix");
}

extern "C" int cgtp_mix_rows_grad(int dtype, int64_t n_rows, int per_row, int width, const void *dout,
                                  int64_t dout_stride, const float *weights, const void *y, int64_t y_stride, void *dy,
                                  int64_t dy_stride, float *dweights, void *stream)
{
    cgtp::clear_error();
    CGTP_TRY(check_sizes(dtype, n_rows, 1, width, width));
    CGTP_TRY(check_per_row(0, per_row));
    if (n_rows * per_row > 0x7fffffffLL)
        return report(CGTP_ERR_ARG, "%lld times %d rows: 2^31 or more", (long long)n_rows, per_row);
    if (n_rows == 0) return CGTP_OK;
    if (!dy && !dweights) return report(CGTP_ERR_ARG, "dy and dweights are both NULL");
    const size_t es = elem(dtype);
    CGTP_TRY(check_rows(dout, "dout", dout_stride, width, n_rows, es));
    if (weights) CGTP_TRY(check_ptr(weights, "weights", 4));
    if (dweights) {
        CGTP_TRY(check_rows(y, "y", y_stride, width, n_rows, es));
        CGTP_TRY(check_ptr(dweights, "dweights", 4));
    }
    if (dy) CGTP_TRY(check_rows(dy, "dy", dy_stride, width, n_rows, es));
    cgtp::RowMixGrad p{};
    p.n = n_rows;
    p.k = per_row;
    p.N = width;
    p.dout = dout;
    p.dout_stride = dout_stride;
    p.weights = weights;
    p.y = y;
    p.y_stride = y_stride;
    p.dy = dy;
    p.dy_stride = dy_stride;
    p.dweights = dweights;
    const hipError_t e = cgtp::launch_mix_rows_grad(dtype, p, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? CGTP_OK : hip_fail(e, "mix gradient");
}
