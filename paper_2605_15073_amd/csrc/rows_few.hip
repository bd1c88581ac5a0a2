// Weight gradients of groups with few rows: a small batch of a model of many elements. A group's gradient is
// written once for a handful of rows: memory and latency bound, too little for the matrix cores' tiles. Sums
// are plain fp32, a thread has one column and kOuterA of them.
//
// Groups of more than kFewRows rows among them are left to the tiled kernel, which finds them by the
// multiples of kFewRows in the sequence (find_big).
//
// Measured as this form came in, with it and with the tiled one for all: 10,007 rows in 4,005 groups,
// 37 x 129 fp32, the whole gradient call 73 and 119 us; 1,000 rows in 500 groups, 256 x 256 63 and 78 us;
// 4,000 rows 138 and 134. The kernel alone takes 38 us of the first (2.2 TB/s, 76 MB of it written).
#include "internal.h"
#include "rows_tile.h"

namespace cgtp {

namespace {

using namespace rows;

constexpr int kOuterA = 32;      // values of a of a thread
constexpr int kOuterRows = 16;   // rows in LDS at once

// A workgroup takes COLS columns of b by 32 (256 / COLS) values of a of one group: a thread has one column
// and 32 sums.
template <typename T, int COLS, bool NARROW>
__global__ __launch_bounds__(kThreads) void k_row_outer_few(RowOrder o, RowOuter q)
{
    constexpr int kA = kOuterA * kThreads / COLS;
    __shared__ float4_t s_a[kOuterRows][kA / 4];
    __shared__ int s_row[kOuterRows];
    const int B = NARROW ? q.r : q.B, W = narrow_width(B);
    const int btiles = (B + COLS - 1) / COLS, tiles = btiles * ((q.A + kA - 1) / kA);
    const int g = blockIdx.x / tiles, tile = blockIdx.x % tiles;
    const int64_t start = clamp_offset(o.offsets[g], o.n), end = clamp_offset(o.offsets[g + 1], o.n);
    if (end - start > kFewRows) return;
    const int tid = threadIdx.x;
    const int a0 = tile / btiles * kA, b = tile % btiles * COLS + tid % COLS, ai = tid / COLS * kOuterA;
    float acc[kOuterA];
#pragma unroll
    for (int i = 0; i < kOuterA; ++i) acc[i] = 0.f;
    for (int64_t p0 = start; p0 < end; p0 += kOuterRows) {
        const int rows = end - p0 < kOuterRows ? (int)(end - p0) : kOuterRows;
        if (p0 > start) __syncthreads();
        if (tid < kOuterRows) s_row[tid] = tid < rows ? row_at(o, p0 + tid) : -1;
        __syncthreads();
        for (int i = tid; i < rows * kA; i += kThreads) {
            const int r = i / kA, a = i % kA, row = s_row[r];
            reinterpret_cast<float *>(&s_a[r])[a] =
                row >= 0 && a0 + a < q.A ? (float)static_cast<const T *>(q.a)[row * q.a_stride + a0 + a] : 0.f;
        }
        __syncthreads();
        for (int r0 = 0; r0 < rows; r0 += 4) {
            float f[4];  // of four rows at once: zero past the last (their a is zero, or not set)
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int row = s_row[r0 + u];
                f[u] = 0.f;
                if (row >= 0 && b < B)
                    f[u] = NARROW ? narrow_at<T>(q.h, p0 + r0 + u, W, b)
                                  : (float)static_cast<const T *>(q.b)[row * q.b_stride + b];
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                if (r0 + u >= rows) break;
#pragma unroll
                for (int i = 0; i < kOuterA; i += 4) {
                    const float4_t a = s_a[r0 + u][(ai + i) / 4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[i + e] += a[e] * f[u];
                }
            }
        }
    }
    if (b >= B) return;
    T *const out = static_cast<T *>(q.out) + (int64_t)g * q.A * B;
#pragma unroll
    for (int i = 0; i < kOuterA; ++i) {
        const int a = a0 + ai + i;
        if (a < q.A) out[q.transposed ? (int64_t)b * q.A + a : (int64_t)a * B + b] = (T)acc[i];
    }
}

template <typename T, int COLS> hipError_t outer(const RowOrder &o, const RowOuter &q, hipStream_t s)
{
    constexpr int kA = kOuterA * kThreads / COLS;
    const int B = q.r > 0 ? q.r : q.B;
    const int64_t blocks = (int64_t)o.G * ((q.A + kA - 1) / kA) * ((B + COLS - 1) / COLS);
    if (blocks > 0x7fffffffLL) return hipErrorInvalidConfiguration;
    auto *kernel = q.r > 0 ? k_row_outer_few<T, COLS, true> : k_row_outer_few<T, COLS, false>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(kThreads), 0, s, o, q);
    return hipGetLastError();
}

template <typename T> hipError_t outer(const RowOrder &o, const RowOuter &q, hipStream_t s)
{
    const int B = q.r > 0 ? q.r : q.B;
    auto tiles = [&](int cols) {
        const int a = kOuterA * kThreads / cols;
        return (int64_t)((q.A + a - 1) / a) * ((B + cols - 1) / cols);
    };
    if (tiles(64) < tiles(256) || B <= 64) return outer<T, 64>(o, q, s);
    return outer<T, 256>(o, q, s);
}

}  // namespace

hipError_t launch_row_outer_few(int dtype, const RowOrder &o, const RowOuter &q, hipStream_t s)
{
    return dtype == CGTP_BF16 ? outer<bf16_t>(o, q, s) : outer<float>(o, q, s);
}

}  // namespace cgtp
