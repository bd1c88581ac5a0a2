// Products and weight gradients of groups with few rows: a small batch of a model of many elements. Each
// group's weights are read, or its gradient written, for a handful of rows: memory and latency bound, too
// little for the matrix cores' tiles. Sums are plain fp32.
#include "internal.h"
#include "rows_tile.h"

#include <type_traits>

namespace cgtp {

namespace {

using namespace rows;

constexpr int kHeld = 8;           // rows in LDS at once, 32 threads each
constexpr int kChunk = 512;        // k of them
constexpr int kColumns = 64;       // of a product's workgroup

// Products. Blocks 0 .. G take the first kHeld rows of a group (G: of no group, zeros). The further tiles of
// larger groups follow: block G + 1 + m is for the group that holds position (m + 1) kHeld, and the i-th such
// block of a group for its tile i + 1; a group of n rows holds at least floor((n - 1) / kHeld) such positions
// beyond its start, the number of those tiles.
//
// What counts is how few memory accesses wait for each other: no search, the rows of a workgroup go to LDS at
// once, and the weights of the next 64 k are loaded before a step is summed. [N][K] weights: eight lanes
// share a column, eight k a lane; a thread has two columns. [K][N]: a thread has four columns and four k of
// every 64.
//
// Of fp32 alone, whose tiles cost six matrix instructions a product and the splitting of the weights. This form
// and the tiles, 2.5 rows a group: 4,005 groups, 37 -> 129 45 and 66 us, 129 -> 37 as the row gradient 30 and 50
// (2.5 TB/s of weights); 4,000 groups, 64 -> 64 19 and 36; 500 groups, 256 -> 256 30 and 40. bf16: 44 and 33, 24
// and 26, 17 and 19, 21 and 17. At 8 rows a group the tiles are ahead (1,000 groups, 128 -> 128 29 and 25).
template <bool WNK>
__global__ __launch_bounds__(kThreads) void k_row_product_few(RowOrder o, RowProduct p)
{
    constexpr int kC = WNK ? 2 : 4;
    __shared__ float4_t s_x[kHeld][kChunk / 4];
    __shared__ float s_part[WNK ? 1 : 4][WNK ? 1 : kHeld][WNK ? 1 : kColumns];
    const int tid = threadIdx.x;
    int g = blockIdx.x;
    int64_t p0 = 0;
    if (g > o.G) {
        const int64_t m = g - (o.G + 1);
        g = group_at(o, (m + 1) * kHeld);
        const int64_t start = clamp_offset(o.offsets[g], o.n), i = m - start / kHeld;
        if (i < 0) return;
        p0 = start + (i + 1) * kHeld;
    } else {
        p0 = clamp_offset(o.offsets[g], o.n);
    }
    const int64_t end = g < o.G ? clamp_offset(o.offsets[g + 1], o.n) : o.n;
    if (p0 >= end) return;
    const int rows = end - p0 < kHeld ? (int)(end - p0) : kHeld;
    const int c0 = blockIdx.y * kColumns;

    // this thread's rows: the one it stages, and (WNK) the one it stores
    const int sr = tid / 32, sc = tid % 32;
    const int row = sr < rows ? row_at(o, p0 + sr) : -1;
    if (g == o.G) {
        if (row >= 0)
            for (int c = c0 + sc; c < c0 + kColumns && c < p.N; c += 32)
                static_cast<float *>(p.out)[row * p.out_stride + c] = 0.f;
        return;
    }

    // weights: column c0 + tid / 8 + 32 j, k from 8 (tid % 8) on, or columns from c0 + 4 (tid % 16) on, k from
    // 4 (tid / 16) on, both in steps of 64 k
    const float *const w = static_cast<const float *>(p.w) + g * p.w_group;
    const int kt = WNK ? tid % 8 * 8 : tid / 16 * 4;
    int col[kC];
    const float *wc[kC];
    const int cw = c0 + tid % 16 * 4, first = cw + 4 <= p.N ? cw : p.N - 4;  // [K][N]: early at a row's end
    if (WNK) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            col[j] = c0 + tid / 8 + 32 * j;
            wc[j] = w + (int64_t)(col[j] < p.N ? col[j] : p.N - 1) * p.K;
        }
    }
    using Load = typename std::conditional<WNK, Raw8<float>, float4_t>::type;
    Load now[kC], next[kC];
    auto load = [&](Load(&v)[kC], int k) {
        if constexpr (WNK) {
            const int at = start8(k + kt < p.K ? k + kt : p.K, p.K);
#pragma unroll
            for (int j = 0; j < 2; ++j)
                if (j == 0 || c0 + 32 < p.N) v[j] = load_any8(wc[j] + at);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int64_t at = k + kt + e < p.K ? k + kt + e : p.K - 1;
                v[e] = *reinterpret_cast<const float4_any *>(w + at * p.N + first);
            }
        }
    };
    load(now, 0);

    float acc[kC][kHeld];
#pragma unroll
    for (int j = 0; j < kC; ++j)
#pragma unroll
        for (int r = 0; r < kHeld; ++r) acc[j][r] = 0.f;
    const float *const in = static_cast<const float *>(p.in) + (row < 0 ? 0 : row) * p.in_stride;
    for (int kc = 0; kc < p.K; kc += kChunk) {
        const int width = p.K - kc < kChunk ? (p.K - kc + 63) / 64 * 64 : kChunk;
        if (kc > 0) __syncthreads();
        if (sr < rows)
            for (int c = sc; c < width; c += 32)
                reinterpret_cast<float *>(&s_x[sr])[c] = row >= 0 && kc + c < p.K ? in[kc + c] : 0.f;
        __syncthreads();
        for (int k = kc; k < kc + width; k += 64) {
            if (k + 64 < p.K) load(next, k + 64);
            if constexpr (WNK) {
                if (k + kt + 8 > p.K) {  // past the end: what was loaded early, and zeros
                    const int kk = k + kt < p.K ? k + kt : p.K;
#pragma unroll
                    for (int j = 0; j < 2; ++j) settle<float>(now[j], kk - start8(kk, p.K), p.K - kk);
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) {
#pragma unroll
                    for (int r = 0; r < kHeld; ++r) {
                        if (r >= rows) break;
                        const float4_t x = s_x[r][(k - kc + kt) / 4 + h];
#pragma unroll
                        for (int j = 0; j < 2; ++j)
#pragma unroll
                            for (int e = 0; e < 4; ++e) acc[j][r] += x[e] * __uint_as_float(now[j].v[h][e]);
                    }
                }
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (k + kt + e >= p.K) now[e] = float4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int r = 0; r < kHeld; ++r) {
                    if (r >= rows) break;
                    const float4_t x = s_x[r][(k - kc + kt) / 4];
#pragma unroll
                    for (int e = 0; e < 4; ++e)
#pragma unroll
                        for (int j = 0; j < 4; ++j) acc[j][r] += x[e] * now[e][j];
                }
            }
#pragma unroll
            for (int j = 0; j < kC; ++j) now[j] = next[j];
        }
    }

    if constexpr (WNK) {  // lane tid % 8 of a column stores row tid % 8
        float mine[2] = {0.f, 0.f};
#pragma unroll
        for (int r = 0; r < kHeld; ++r) {
            if (r >= rows) break;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                float v = acc[j][r];
                v += __shfl_xor(v, 1);
                v += __shfl_xor(v, 2);
                v += __shfl_xor(v, 4);
                if (tid % 8 == r) mine[j] = v;
            }
        }
        const int to = tid % 8 < rows ? row_at(o, p0 + tid % 8) : -1;
        if (to < 0) return;
#pragma unroll
        for (int j = 0; j < 2; ++j)
            if (col[j] < p.N) static_cast<float *>(p.out)[to * p.out_stride + col[j]] = mine[j];
    } else {
#pragma unroll
        for (int r = 0; r < kHeld; ++r) {
            if (r >= rows) break;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float v = acc[j][r];
                v += __shfl_xor(v, 16);
                v += __shfl_xor(v, 32);
                if ((tid & 63) < 16) s_part[tid / 64][r][tid % 16 * 4 + j] = v;
            }
        }
        __syncthreads();
        if (row < 0) return;
        for (int i = sc; i < kColumns; i += 32) {
            const int own = c0 + i / 4 * 4;  // the quad's first column, and what its load started early
            const int c = (own + 4 <= p.N ? own : p.N - 4) + i % 4;
            if (own >= p.N || c < own) continue;  // of the quad before
            const float v = s_part[0][sr][i] + s_part[1][sr][i] + (s_part[2][sr][i] + s_part[3][sr][i]);
            static_cast<float *>(p.out)[row * p.out_stride + c] = v;
        }
    }
}

constexpr int kOuterA = 32;      // values of a of a thread
constexpr int kOuterRows = 16;   // rows in LDS at once

// Weight gradients, in plain fp32 for both types. Groups of more than kFewRows rows are left to the tiled kernel,
// which finds them by the multiples of kFewRows in the sequence (find_big).
//
// A workgroup takes COLS columns of b by 32 (256 / COLS) values of a of one group: a thread has one column
// and 32 sums. (The gradient as one run of cells, so that all lanes have some at any widths, with both rows'
// values read from LDS for each product, took 45 us where this takes 33.)
//
// Measured as this form came in, with it and with the tiled one for all: 10,007 rows in 4,005 groups,
// 37 x 129 fp32, the whole gradient call 73 and 119 us; 1,000 rows in 500 groups, 256 x 256 63 and 78 us;
// 4,000 rows 138 and 134. The kernel alone takes 38 us of the first (2.2 TB/s, 76 MB of it written).
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

// [N][K] weights of up to half a step of k leave half of the lanes without any: 128 x 32, 18 us and 14 with tiles.
bool row_few_takes(int dtype, const RowOrder &o, const RowProduct &p)
{
    return dtype == CGTP_F32 && p.w_group && !p.h && !p.a && !p.narrow && o.n <= kFewMean * (int64_t)o.G &&
           (p.w_nk ? p.K > 32 : p.N >= 4);
}

hipError_t launch_row_few(const RowOrder &o, const RowProduct &p, hipStream_t s)
{
    const dim3 grid((unsigned)(o.G + 1 + o.n / kHeld), (unsigned)((p.N + kColumns - 1) / kColumns));
    auto *kernel = p.w_nk ? k_row_product_few<true> : k_row_product_few<false>;
    hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, s, o, p);
    return hipGetLastError();
}

}  // namespace cgtp
