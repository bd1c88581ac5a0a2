// Tiles of the row products in LDS and registers, shared by the kernels of rows_product.hip and
// rows_outer.hip.
//
// An operand tile of R lanes (rows of the input, columns of the weights, ...) by kGroups k-groups is
// held in 16-byte units of consecutive k: kU = 8 bf16 or 4 fp32 values. Unit (kg, r) lies at
// kg (R + 1) + r, so that the 32 lanes of a matrix instruction's half read consecutive units and the
// eight lanes that stage one row's eight units hit different banks.
//
// Operands whose k is contiguous in memory are staged a unit a load. The others (weights of the
// forward product, both operands of a weight gradient) are loaded four lanes wide, kU rows deep and
// transposed in registers; the four units of a thread then go to places 8 apart within a block of 32
// (place()), so that neighbouring threads write neighbouring units. The matrix instruction does not
// care which lane carries which column: lane_of() gives the column that a place holds.
#ifndef CGTP_ROWS_TILE_H
#define CGTP_ROWS_TILE_H

#include "rows.h"

namespace cgtp {
namespace rows {

typedef __bf16 bf16_t;
typedef float float4_t __attribute__((ext_vector_type(4)));
typedef float float16_t __attribute__((ext_vector_type(16)));
typedef unsigned uint2_t __attribute__((ext_vector_type(2)));
typedef unsigned uint4_t __attribute__((ext_vector_type(4)));
typedef bf16_t bf2_t __attribute__((ext_vector_type(2)));
typedef bf16_t bf4_t __attribute__((ext_vector_type(4)));
typedef bf16_t bf8_t __attribute__((ext_vector_type(8)));

constexpr int kThreads = 256;
constexpr int kGroups = 8;  // k-groups of a step

template <typename T> constexpr int kU = 16 / (int)sizeof(T);
template <typename T> constexpr int kStep = kGroups * kU<T>;  // k of a step: 64 bf16, 32 fp32

__device__ __forceinline__ int clamp_offset(int v, int64_t n)
{
    return v < 0 ? 0 : (int64_t)v > n ? (int)n : v;
}

// Groups share the sequence of rows. Cut into tiles of R = 2^shift positions of one group, tile j of
// group g has the index offsets[g] / R + g + j: since floor((o + m) / R) + 1 >= floor(o / R) +
// ceil(m / R), tiles of different groups never meet, and no prefix sum of tile counts is needed.
// Group G holds the rows of no group. An empty group has one empty tile.
struct Tile {
    int g;          // -1: no tile at this index
    int64_t p0, p1; // its positions
    int64_t start, end;  // the group's
};

// The wave searches 64 candidates at a time: three loads deep for 4096 groups.
__device__ __forceinline__ Tile find_tile(const RowOrder &o, int shift, int64_t index)
{
    const int lane = threadIdx.x & 63;
    int lo = 0, len = o.G + 1;  // the last g with offsets[g] / R + g <= index lies in [lo, lo + len)
    while (len > 1) {
        const int s = (len + 63) / 64;
        const int c = lo + lane * s;
        const bool ok = lane * s < len &&
                        (clamp_offset(o.offsets[lane * s < len ? c : lo], o.n) >> shift) + (int64_t)c <= index;
        const int cnt = __popcll(__ballot(ok));
        const int skip = (cnt > 0 ? cnt - 1 : 0) * s;
        lo += skip;
        len = len - skip < s ? len - skip : s;
    }
    lo = __builtin_amdgcn_readfirstlane(lo);
    Tile t;
    t.start = clamp_offset(o.offsets[lo], o.n);
    t.end = lo < o.G ? clamp_offset(o.offsets[lo + 1], o.n) : o.n;
    const int64_t j = index - ((t.start >> shift) + lo);
    t.p0 = t.start + (j << shift);
    t.p1 = t.p0 + ((int64_t)1 << shift) < t.end ? t.p0 + ((int64_t)1 << shift) : t.end;
    t.g = lo;
    if (j < 0 || (j > 0 && t.p0 >= t.end)) t.g = -1;
    return t;
}

// Row of a position, -1 where the order holds none.
__device__ __forceinline__ int row_at(const RowOrder &o, int64_t p)
{
    if (!o.order) return (int)p;
    const int r = o.order[p];
    return (unsigned)r < (unsigned)o.n ? r : -1;
}

// The segments of a tile's positions that share a group, for R = 32 .. 128 positions from p0 on: their
// groups seg_g[0 .. count), where they start seg_at[0 .. count), and seg_at[count], the end of the last.
// Positions of no group, and those from `rows` on, come after it. Returns the count. Called by the whole
// workgroup; g: R ints of LDS.
template <int R>
__device__ __forceinline__ int find_segments(const RowOrder &o, int64_t p0, int rows, int *g, int *seg_g,
                                             int *seg_at, int *count)
{
    const int tid = threadIdx.x, lane = tid & 63;
    if (tid < R) {
        int lo = 0, hi = o.G;  // the last group that starts at or before this position
        while (lo < hi) {
            const int mid = (lo + hi + 1) / 2;
            if (clamp_offset(o.offsets[mid], o.n) <= p0 + tid) lo = mid;
            else hi = mid - 1;
        }
        g[tid] = tid < rows ? lo : o.G;
    }
    __syncthreads();
    if (tid < 64) {
        int n = 0;
        for (int b = 0; b < R; b += 64) {
            const int r = b + lane;
            const int gr = r < R ? g[r] : o.G;
            const bool first = gr < o.G && (r == 0 || g[r - 1] != gr);
            const unsigned long long m = __ballot(first);
            const int at = n + __popcll(m & ((1ull << lane) - 1));
            if (first) {
                seg_g[at] = gr;
                seg_at[at] = r;
            }
            n += __popcll(m);
        }
        if (lane == 0) *count = n;
    }
    __syncthreads();
    const int n = __builtin_amdgcn_readfirstlane(*count);
    if (tid < R && g[tid] == o.G && (tid == 0 || g[tid - 1] != o.G)) seg_at[n] = tid;
    if (tid == 0 && g[R - 1] != o.G) seg_at[n] = R;
    __syncthreads();
    return n;
}

// One unit: kU values from p on, zero past the `left` that exist.
template <typename T, bool VEC>
__device__ __forceinline__ uint4_t load_unit(const T *p, int64_t left)
{
    uint4_t v = {0, 0, 0, 0};
    if (VEC) {
        if (left > 0) v = *reinterpret_cast<const uint4_t *>(p);
    } else if (sizeof(T) == 4) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (left > e) v[e] = reinterpret_cast<const unsigned *>(p)[e];
    } else {
        const unsigned short *h = reinterpret_cast<const unsigned short *>(p);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            unsigned lo = 0, hi = 0;
            if (left > 2 * e) lo = h[2 * e];
            if (left > 2 * e + 1) hi = h[2 * e + 1];
            v[e] = lo | hi << 16;
        }
    }
    return v;
}

// Four consecutive values, as loaded: 16 or 8 bytes.
template <typename T> struct Four;
template <> struct Four<float> { typedef uint4_t t; };
template <> struct Four<bf16_t> { typedef uint2_t t; };

template <typename T, bool VEC>
__device__ __forceinline__ typename Four<T>::t load_four(const T *p, int64_t left)
{
    typedef typename Four<T>::t F;
    F v = {};
    if (VEC) {
        if (left > 0) v = *reinterpret_cast<const F *>(p);
    } else if (sizeof(T) == 4) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (left > e) v[e] = reinterpret_cast<const unsigned *>(p)[e];
    } else {
        const unsigned short *h = reinterpret_cast<const unsigned short *>(p);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            unsigned lo = 0, hi = 0;
            if (left > 2 * e) lo = h[2 * e];
            if (left > 2 * e + 1) hi = h[2 * e + 1];
            v[e] = lo | hi << 16;
        }
    }
    return v;
}

// The units of four lanes from kU loads of four values each.
__device__ __forceinline__ void transpose4(const uint4_t (&in)[4], uint4_t (&out)[4])
{
#pragma unroll
    for (int j = 0; j < 4; ++j) out[j] = uint4_t{in[0][j], in[1][j], in[2][j], in[3][j]};
}

__device__ __forceinline__ void transpose4(const uint2_t (&in)[8], uint4_t (&out)[4])
{
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const unsigned a = in[2 * e][j >> 1], b = in[2 * e + 1][j >> 1];
            out[j][e] = __builtin_amdgcn_perm(b, a, (j & 1) ? 0x07060302u : 0x05040100u);
        }
}

// Where a transposed operand's lane r lies in its block of 32, and which lane a place holds.
__device__ __forceinline__ int place(int r) { return (r & ~31) | (r & 3) << 3 | (r >> 2 & 7); }
__device__ __forceinline__ int lane_of(int p) { return (p & ~31) | (p & 7) << 2 | (p >> 3 & 3); }

// acc += A B for one unit of each lane: lanes 0..31 carry k-group 2 s, lanes 32..63 2 s + 1.
__device__ __forceinline__ void mma(float16_t &acc, uint4_t a, uint4_t b, bf16_t)
{
    acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf8_t, a),
                                                  __builtin_bit_cast(bf8_t, b), acc, 0, 0, 0);
}

__device__ __forceinline__ void mma(float16_t &acc, uint4_t a, uint4_t b, float)
{
    const float4_t x = __builtin_bit_cast(float4_t, a), y = __builtin_bit_cast(float4_t, b);
#pragma unroll
    for (int e = 0; e < 4; ++e)
        acc = __builtin_amdgcn_mfma_f32_32x32x2f32(x[e], y[e], acc, 0, 0, 0);
}

// The products of a step: TC blocks of 32 columns (from unit column c0 of cols) by TR blocks of 32
// rows. acc[c][r][i]: column place 8 (i / 4) + 4 (lane / 32) + i % 4 of block c, row place lane % 32 of
// block r. All k-groups always, zeros past the end: a branch around a matrix instruction costs a copy of
// its sums.
template <typename T, int BN, int BM, int TC, int TR>
__device__ __forceinline__ void step_products(float16_t (&acc)[TC][TR], const uint4_t *cols,
                                              const uint4_t *rws, int c0, int r0)
{
    const int lane = threadIdx.x & 63, half = lane >> 5, n = lane & 31;
#pragma unroll
    for (int s = 0; s < kGroups / 2; ++s) {
        uint4_t a[TC], b[TR];
#pragma unroll
        for (int c = 0; c < TC; ++c) a[c] = cols[(2 * s + half) * (BN + 1) + c0 + 32 * c + n];
#pragma unroll
        for (int r = 0; r < TR; ++r) b[r] = rws[(2 * s + half) * (BM + 1) + r0 + 32 * r + n];
#pragma unroll
        for (int c = 0; c < TC; ++c)
#pragma unroll
            for (int r = 0; r < TR; ++r) mma(acc[c][r], a[c], b[r], T{});
    }
}

// Four consecutive columns of a lane's row: the first of vector v, and the values. With a
// transposed column operand they are the accumulators 4 apart.
template <bool TRANS>
__device__ __forceinline__ int vec_col(int v, int half) { return TRANS ? 4 * (4 * half + v) : 8 * v + 4 * half; }

template <bool TRANS>
__device__ __forceinline__ float4_t vec_val(const float16_t &acc, int v)
{
    return TRANS ? float4_t{acc[v], acc[4 + v], acc[8 + v], acc[12 + v]}
                 : float4_t{acc[4 * v], acc[4 * v + 1], acc[4 * v + 2], acc[4 * v + 3]};
}

// Stores four consecutive values, of which `left` exist.
template <bool VEC> __device__ __forceinline__ void store_four(float *p, float4_t v, int64_t left)
{
    if (VEC) {
        if (left > 0) *reinterpret_cast<float4_t *>(p) = v;
        return;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (left > e) p[e] = v[e];
}

template <bool VEC> __device__ __forceinline__ void store_four(bf16_t *p, float4_t v, int64_t left)
{
    const bf4_t h = {(bf16_t)v[0], (bf16_t)v[1], (bf16_t)v[2], (bf16_t)v[3]};
    if (VEC) {
        if (left > 0) *reinterpret_cast<bf4_t *>(p) = h;
        return;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (left > e) p[e] = h[e];
}

// Zeros in the columns [c0, c1) of the tile's rows: those of no group.
template <typename T>
__device__ __forceinline__ void store_zeros(const RowProduct &p, const int *row, int rows, int c0, int c1)
{
    for (int r = threadIdx.x >> 6; r < rows; r += kThreads / 64)
        if (row[r] >= 0)
            for (int c = c0 + (threadIdx.x & 63); c < c1; c += 64)
                static_cast<T *>(p.out)[row[r] * p.out_stride + c] = (T)0.f;
}

// Results of narrow products (width N <= 64, between the two products of an adapter), in sequence
// order: fp32 [n][W], or for bf16 two parts hi + lo [n][2][W], 16 bits of significand; W is N
// rounded up to a unit, the rest zero.
template <typename T> __host__ __device__ constexpr int narrow_width(int N) { return (N + kU<T> - 1) / kU<T> * kU<T>; }
template <typename T> constexpr int kParts = sizeof(T) == 2 ? 2 : 1;

__device__ __forceinline__ void store_narrow(float *p, int W, float4_t v)
{
    *reinterpret_cast<float4_t *>(p) = v;
}

__device__ __forceinline__ void store_narrow(bf16_t *p, int W, float4_t v)
{
    bf4_t hi, lo;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        hi[e] = (bf16_t)v[e];
        const float h = (float)hi[e];
        lo[e] = (bf16_t)(__builtin_isfinite(h) ? v[e] - h : 0.f);  // an infinity has no second part
    }
    *reinterpret_cast<bf4_t *>(p) = hi;
    *reinterpret_cast<bf4_t *>(p + W) = lo;
}

template <typename T> bool unit_aligned(const void *p, int64_t stride)
{
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride % kU<T> == 0;
}

}  // namespace rows
}  // namespace cgtp

#endif
