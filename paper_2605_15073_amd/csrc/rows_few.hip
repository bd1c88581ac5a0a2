// Products and weight gradients of groups with few rows: single rows of many experts, a small batch of a
// model of many elements. A group's weights are read once, or written once, for a handful of rows: memory
// and latency bound, too little for the matrix cores' tiles. Sums are plain fp32.
//
// Groups of more than kFewRows rows among them are left to the tiled kernels, which find them by the
// multiples of kFewRows in the sequence (find_big).
#include "internal.h"
#include "rows_tile.h"

namespace cgtp {

namespace {

using namespace rows;

constexpr int kTileRows = 8;   // rows of a tile
constexpr int kTileCols = 64;  // columns of a workgroup
constexpr int kChunk = 512;    // k of the input rows in LDS at once

template <typename T> __device__ __forceinline__ float value(const uint4_t &v, int e)
{
    if (sizeof(T) == 4) return __builtin_bit_cast(float, (unsigned)v[e % 4]);
    const unsigned u = v[e / 2 % 4];
    return __builtin_bit_cast(float, e & 1 ? u & 0xffff0000u : u << 16);
}

template <typename T> __device__ __forceinline__ float value(const uint2_t &v, int e)
{
    if (sizeof(T) == 4) return __builtin_bit_cast(float, (unsigned)v[e % 2]);
    const unsigned u = v[e / 2 % 2];
    return __builtin_bit_cast(float, e & 1 ? u & 0xffff0000u : u << 16);
}

// A thread takes kWide columns (two or four) of every 8th or 16th k of [K][N] weights, or one column and
// every fourth 16 bytes of k of [N][K] ones; the partial sums meet in LDS, or between lanes.
template <typename T, bool WNK, bool VEC>
__global__ __launch_bounds__(kThreads) void k_row_few(RowOrder o, RowProduct p)
{
    constexpr int CW = kWide<T>, kLanes = kTileCols / CW, kSlices = kThreads / kLanes, V = 16 / (int)sizeof(T);
    constexpr int kUnroll = 4;
    __shared__ float4_t s_x[kChunk][kTileRows / 4];  // the rows, k first
    __shared__ float s_sum[WNK ? 1 : kSlices][kTileRows][kTileCols];
    __shared__ int s_row[kTileRows];
    const Tile t = find_tile(o, 3, blockIdx.x);
    if (t.g < 0 || t.p0 >= t.p1) return;
    const int rows = (int)(t.p1 - t.p0), tid = threadIdx.x;
    const int c0 = blockIdx.y * kTileCols;
    if (t.g < o.G && t.end - t.start > kFewRows) return;
    if (tid < kTileRows) s_row[tid] = tid < rows ? row_at(o, t.p0 + tid) : -1;
    __syncthreads();
    if (t.g == o.G) {
        if (!p.narrow) store_zeros<T>(p, s_row, rows, c0, c0 + kTileCols < p.N ? c0 + kTileCols : p.N);
        return;
    }
    const T *const w = static_cast<const T *>(p.w) + (int64_t)t.g * p.w_group;
    constexpr int NA = WNK ? 1 : CW;
    float acc[NA][kTileRows];
#pragma unroll
    for (int c = 0; c < NA; ++c)
#pragma unroll
        for (int r = 0; r < kTileRows; ++r) acc[c][r] = 0.f;
    const int quad = tid % kLanes, slice = tid / kLanes;  // [K][N]
    const int col = c0 + (WNK ? tid / 4 : CW * quad);
    for (int k0 = 0; k0 < p.K; k0 += kChunk) {
        const int kc = p.K - k0 < kChunk ? p.K - k0 : kChunk;
        if (k0 > 0) __syncthreads();
        for (int r = tid >> 6; r < kTileRows; r += kThreads / 64) {
            const int row = s_row[r];
            for (int k = tid & 63; k < kc; k += 64)
                reinterpret_cast<float *>(&s_x[k])[r] =
                    row < 0 ? 0.f : (float)static_cast<const T *>(p.in)[row * p.in_stride + k0 + k];
        }
        __syncthreads();
        if constexpr (WNK) {
            const T *const q = w + (int64_t)(col < p.N ? col : p.N - 1) * p.K + k0;
            for (int k = tid % 4 * V; k < kc; k += 4 * V) {
                const uint4_t v = load_16<T, VEC>(q + k, kc - k);
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    if (k + e >= kc) break;
                    const float4_t x0 = s_x[k + e][0], x1 = s_x[k + e][1];
                    const float f = value<T>(v, e);
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        acc[0][r] += f * x0[r];
                        acc[0][4 + r] += f * x1[r];
                    }
                }
            }
        } else if (col < p.N) {
            for (int k = slice; k < kc; k += kSlices * kUnroll) {
                uint2_t v[kUnroll];
#pragma unroll
                for (int u = 0; u < kUnroll; ++u) {
                    const int kk = k + u * kSlices;
                    v[u] = load_8<T, VEC>(w + (int64_t)(k0 + kk) * p.N + col, kk < kc ? p.N - col : 0);
                }
#pragma unroll
                for (int u = 0; u < kUnroll; ++u) {
                    const int kk = k + u * kSlices;
                    if (kk >= kc) break;
                    const float4_t x0 = s_x[kk][0], x1 = s_x[kk][1];
#pragma unroll
                    for (int c = 0; c < CW; ++c) {
                        const float f = value<T>(v[u], c);
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            acc[c][r] += f * x0[r];
                            acc[c][4 + r] += f * x1[r];
                        }
                    }
                }
            }
        }
    }
    const float scale = p.narrow_scale ? p.narrow_scale[t.g] : 1.f;
    const int No = narrow_width(p.N);
    auto store = [&](int r, int c, float sum) {
        if (p.narrow) {
            if (r >= rows || c >= No) return;
            T *const q = static_cast<T *>(p.out) + (t.p0 + r) * (kNarrow<T> * No) + c;
            sum = c < p.N ? sum * scale : 0.f;
            const T hi = (T)sum;
            q[0] = hi;
            if (kNarrow<T> == 2) q[No] = (T)(__builtin_isfinite((float)hi) ? sum - (float)hi : 0.f);
        } else if (s_row[r] >= 0 && c < p.N) {
            static_cast<T *>(p.out)[s_row[r] * p.out_stride + c] = (T)sum;
        }
    };
    if constexpr (WNK) {
#pragma unroll
        for (int r = 0; r < kTileRows; ++r) {
            acc[0][r] += __shfl_xor(acc[0][r], 1);
            acc[0][r] += __shfl_xor(acc[0][r], 2);
        }
#pragma unroll
        for (int r = 0; r < kTileRows; r += 4) {  // a column's four lanes store two rows each
            const int l = tid & 3;
            store(r + l, col, l == 0 ? acc[0][r] : l == 1 ? acc[0][r + 1] : l == 2 ? acc[0][r + 2] : acc[0][r + 3]);
        }
    } else {
#pragma unroll
        for (int r = 0; r < kTileRows; ++r)
#pragma unroll
            for (int c = 0; c < CW; ++c) s_sum[slice][r][CW * quad + c] = acc[c][r];
        __syncthreads();
        for (int i = tid; i < kTileRows * kTileCols; i += kThreads) {
            const int r = i / kTileCols, c = i % kTileCols;
            float sum = 0.f;
#pragma unroll
            for (int s = 0; s < kSlices; ++s) sum += s_sum[s][r][c];
            store(r, c0 + c, sum);
        }
    }
}

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
        for (int r = 0; r < rows; ++r) {
            const int row = s_row[r];
            if (row < 0 || b >= B) continue;
            const float f = NARROW ? narrow_at<T>(q.h, p0 + r, W, b)
                                   : (float)static_cast<const T *>(q.b)[row * q.b_stride + b];
#pragma unroll
            for (int i = 0; i < kOuterA; i += 4) {
                const float4_t a = s_a[r][(ai + i) / 4];
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[i + e] += a[e] * f;
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

template <typename T, bool WNK> hipError_t product(const RowOrder &o, const RowProduct &p, hipStream_t s)
{
    constexpr int V = 16 / (int)sizeof(T);
    const bool vec = aligned_rows<T>(p.w, 0) && (WNK ? p.K : p.N) % V == 0;
    auto *kernel = vec ? k_row_few<T, WNK, true> : k_row_few<T, WNK, false>;
    const dim3 grid((unsigned)(o.n / kTileRows + o.G + 1), (unsigned)((p.N + kTileCols - 1) / kTileCols));
    hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, s, o, p);
    return hipGetLastError();
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

hipError_t launch_row_few(int dtype, const RowOrder &o, const RowProduct &p, hipStream_t s)
{
    if (dtype == CGTP_BF16) return p.w_nk ? product<bf16_t, true>(o, p, s) : product<bf16_t, false>(o, p, s);
    return p.w_nk ? product<float, true>(o, p, s) : product<float, false>(o, p, s);
}

hipError_t launch_row_outer_few(int dtype, const RowOrder &o, const RowOuter &q, hipStream_t s)
{
    return dtype == CGTP_BF16 ? outer<bf16_t>(o, q, s) : outer<float>(o, q, s);
}

}  // namespace cgtp
