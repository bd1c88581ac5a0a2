// Products of grouped rows (cgtp_grouped_linear, cgtp_adapter_linear and their gradients).
#include "internal.h"
#include "rows.h"

namespace cgtp {

namespace {

typedef __bf16 bf16_t;

template <typename T> __device__ __forceinline__ float to_f32(T v) { return (float)v; }

__device__ __forceinline__ int clamp_offset(int v, int64_t n)
{
    return v < 0 ? 0 : (int64_t)v > n ? (int)n : v;
}

// Groups share the sequence of rows; a tile of R positions of one group has the index
// offsets[g] / R + g + j: since floor((o + m) / R) + 1 >= floor(o / R) + ceil(m / R), the tiles of
// different groups never meet, and no prefix sum of tile counts is needed. Group G holds the
// rows of no group.
struct Tile {
    int g;          // G: no group; -1: none at this index
    int64_t p0, p1; // positions
};

__device__ Tile find_tile(const RowOrder &o, int R, int64_t index)
{
    int lo = 0, hi = o.G;  // the last group whose first tile index is <= index
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if ((int64_t)clamp_offset(o.offsets[mid], o.n) / R + mid <= index) lo = mid;
        else hi = mid - 1;
    }
    const int64_t start = clamp_offset(o.offsets[lo], o.n);
    const int64_t end = lo < o.G ? clamp_offset(o.offsets[lo + 1], o.n) : o.n;
    const int64_t p0 = start + (index - (start / R + lo)) * R;
    if (p0 >= end) return {-1, 0, 0};
    return {lo, p0, p0 + R < end ? p0 + R : end};
}

__device__ __forceinline__ int64_t row_at(const RowOrder &o, int64_t p)
{
    return o.order ? o.order[p] : p;
}

__device__ __forceinline__ bool row_ok(const RowOrder &o, int64_t row)
{
    return row >= 0 && row < o.n;
}

constexpr int kTileRows = 16;

template <typename T>
__global__ __launch_bounds__(256) void k_row_product(RowOrder o, RowProduct p)
{
    const Tile t = find_tile(o, kTileRows, blockIdx.x);
    if (t.g < 0) return;
    const int c = blockIdx.y * 64 + (threadIdx.x & 63);
    if (c >= p.N) return;
    const T *w = (const T *)p.w + (p.w_group ? (int64_t)(t.g < o.G ? t.g : 0) * p.w_group : 0);
    const bool bare = t.g == o.G;
    const float scale = p.narrow_scale && !bare ? p.narrow_scale[t.g] : 1.f;
    for (int64_t pos = t.p0 + (threadIdx.x >> 6); pos < t.p1; pos += 4) {
        const int64_t row = row_at(o, pos);
        if (!row_ok(o, row)) continue;
        float acc = 0.f;
        if (!bare || !p.w_group) {
            const T *in = (const T *)p.in + row * p.in_stride;
            for (int k = 0; k < p.K; ++k)
                acc += to_f32(in[k]) * to_f32(w[p.w_nk ? (int64_t)c * p.K + k : (int64_t)k * p.N + c]);
        }
        if (p.h && !bare) {
            const T *v = (const T *)p.v + (int64_t)t.g * p.r * p.N;
            const float *h = (const float *)p.h + pos * p.r;
            for (int k = 0; k < p.r; ++k)
                acc += h[k] * to_f32(v[p.w_nk ? (int64_t)c * p.r + k : (int64_t)k * p.N + c]);
        }
        if (p.narrow) ((float *)p.out)[pos * p.N + c] = acc * scale;
        else ((T *)p.out)[row * p.out_stride + c] = (T)acc;
    }
}

template <typename T>
__global__ __launch_bounds__(256) void k_row_outer(RowOrder o, RowOuter q)
{
    const int g = blockIdx.x;
    const int64_t start = clamp_offset(o.offsets[g], o.n);
    const int64_t end = clamp_offset(o.offsets[g + 1], o.n);
    const int cols = q.r > 0 ? q.r : q.B;
    for (int64_t e = blockIdx.y * 256 + threadIdx.x; e < (int64_t)q.A * cols; e += 256 * gridDim.y) {
        const int i = (int)(e / cols), c = (int)(e % cols);
        float acc = 0.f;
        for (int64_t pos = start; pos < end; ++pos) {
            const int64_t row = row_at(o, pos);
            if (!row_ok(o, row)) continue;
            const float b = q.r > 0 ? ((const float *)q.h)[pos * q.r + c]
                                : to_f32(((const T *)q.b)[row * q.b_stride + c]);
            acc += to_f32(((const T *)q.a)[row * q.a_stride + i]) * b;
        }
        const int64_t at = q.transposed ? (int64_t)c * q.A + i : e;
        ((T *)q.out)[(int64_t)g * q.A * cols + at] = (T)acc;
    }
}

}  // namespace

size_t narrow_bytes(int dtype, int64_t n_rows, int N) { return (size_t)n_rows * N * 4; }

size_t row_outer_bytes(int dtype, int64_t n_rows, int G, int A, int B) { return 0; }

hipError_t launch_row_product(int dtype, const RowOrder &o, const RowProduct &p, hipStream_t s)
{
    const dim3 grid((unsigned)(o.n / kTileRows + o.G + 1), (unsigned)((p.N + 63) / 64));
    if (dtype == CGTP_BF16) hipLaunchKernelGGL(k_row_product<bf16_t>, grid, dim3(256), 0, s, o, p);
    else hipLaunchKernelGGL(k_row_product<float>, grid, dim3(256), 0, s, o, p);
    return hipGetLastError();
}

hipError_t launch_row_outer(int dtype, const RowOrder &o, const RowOuter &q, void *ws, hipStream_t s)
{
    const int64_t cells = (int64_t)q.A * (q.r > 0 ? q.r : q.B);
    const int64_t by = (cells + 255) / 256;
    const dim3 grid((unsigned)o.G, (unsigned)(by < 1024 ? by : 1024));
    if (dtype == CGTP_BF16) hipLaunchKernelGGL(k_row_outer<bf16_t>, grid, dim3(256), 0, s, o, q);
    else hipLaunchKernelGGL(k_row_outer<float>, grid, dim3(256), 0, s, o, q);
    return hipGetLastError();
}

}  // namespace cgtp
