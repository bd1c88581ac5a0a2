// Tiles of the row products in LDS and registers, shared by rows_product.hip, rows_outer.hip and
// rows_wide.hip.
//
// An operand tile of R lanes (rows of the input, columns of the weights, ...) by kGroups k-groups is
// held in 16-byte units of 8 consecutive k in bf16. Unit (kg, r) lies at kg (R + 1) + r, so that the 32
// lanes of a matrix instruction's half read consecutive units and the eight lanes that stage one row's
// units hit different banks.
//
// fp32 operands are three bf16 parts each, 2^16 x = h + m + l (24 bits of significand), and a product is hh,
// hm, mh, mm, hl, lh, summed in fp32: six matrix instructions for 16 k, where the fp32 ones take eight
// of twice the time; what is left out is below 2^-24 of the term. 2^16 x is a multiple of 2^-133, bf16's smallest
// step, so that the parts hold every x up to 2^112 whole, however small, beside whatever others. Sums beyond
// 2^96, larger inputs, infinities and NaN leave results that are not finite, and so do an adapter's weights that
// are not, which rows of other adapters in a tile meet as zeros. Those results, and no others, are formed again in
// plain fp32, one result a thread at a time, up to the term that makes it NaN. 131,072 rows, 64 -> 896, 8 groups: y
// 122 us, with one infinite input 339, with one in every 128 rows 650; all gradients 361, 2,700 and 3,800 us (a cell of
// dw runs over its chunk's rows); 896 -> 128, dy all NaN, 2,060 us where numbers take 579.
//
// Operands whose k is contiguous in memory are staged eight k a load. The others (weights of the
// forward product, both operands of a weight gradient) are loaded 8 or 16 bytes wide (kWide, kFull lanes), 8
// rows deep, and transposed in registers; the units of a thread then go to places apart within a block of 32
// (place(), place_full()), so that neighbouring threads write neighbouring units. The matrix instruction does
// not care which lane carries which column; the stores find each column where its place is.
#ifndef CGTP_ROWS_TILE_H
#define CGTP_ROWS_TILE_H

#include "rows.h"
#include "rows_index.h"

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
constexpr int kU = 8;  // k of a unit

template <typename T> constexpr int kSplit = sizeof(T) == 2 ? 1 : 3;   // parts of an operand
template <typename T> constexpr int kGroups = sizeof(T) == 2 ? 8 : 4;  // k-groups of a step
template <typename T> constexpr int kStep = kGroups<T> * kU;           // k of a step: 64 bf16, 32 fp32
template <typename T> constexpr int kWide = 8 / (int)sizeof(T);        // lanes of a transposed load
template <typename T, int R> constexpr int kTile = kSplit<T> * kGroups<T> * (R + 1);  // units of a tile

__device__ __forceinline__ int clamp_offset(int v, int64_t n)
{
    return v < 0 ? 0 : (int64_t)v > n ? (int)n : v;
}

// Positions over the rows of a tile: R, a power of two known here, or the chunks of a weight gradient, a multiple
// of 64 up to 2^14. Of those the quotient is that of 64ths, x < 2^25 over q <= 256, by m = ceil(2^33 / q): what m
// exceeds 2^33 / q by adds x (m q - 2^33) / (2^33 q) < 1 / q.
template <int R> struct TileRows {
    static constexpr int rows = R;
    __device__ int of(int pos) const { return pos / R; }
};
struct ChunkRows {
    int rows;
    unsigned m;
    explicit ChunkRows(int r) : rows(r), m((unsigned)(((1ull << 33) + r / 64 - 1) / (r / 64))) {}
    __device__ int of(int pos) const { return (int)(((unsigned long long)(pos >> 6) * m) >> 33); }
};

// Groups share the sequence of rows. Cut into tiles of R positions of one group, tile j of
// group g has the index offsets[g] / R + g + j: since floor((o + m) / R) + 1 >= floor(o / R) +
// ceil(m / R), tiles of different groups never meet, and no prefix sum of tile counts is needed.
// Group G holds the rows of no group. An empty group has one empty tile.
struct Tile {
    int g;          // -1: no tile at this index
    int64_t p0, p1; // its positions
    int64_t start, end;  // the group's
};

// The wave searches 64 candidates at a time: three loads deep for 4096 groups.
template <typename Rows> __device__ __forceinline__ Tile find_tile(const RowOrder &o, Rows R, int64_t index)
{
    const int lane = threadIdx.x & 63;
    int lo = 0, len = o.G + 1;  // the last g with offsets[g] / R + g <= index lies in [lo, lo + len)
    while (len > 1) {
        const int s = (len + 63) / 64;
        const int c = lo + lane * s;
        const bool ok = lane * s < len &&
                        R.of(clamp_offset(o.offsets[lane * s < len ? c : lo], o.n)) + (int64_t)c <= index;
        const int cnt = __popcll(__ballot(ok));
        const int skip = (cnt > 0 ? cnt - 1 : 0) * s;
        lo += skip;
        len = len - skip < s ? len - skip : s;
    }
    lo = __builtin_amdgcn_readfirstlane(lo);
    Tile t;
    t.start = clamp_offset(o.offsets[lo], o.n);
    t.end = lo < o.G ? clamp_offset(o.offsets[lo + 1], o.n) : o.n;
    const int64_t j = index - (R.of((int)t.start) + lo);
    t.p0 = t.start + j * R.rows;
    t.p1 = t.p0 + R.rows < t.end ? t.p0 + R.rows : t.end;
    t.g = lo;
    if (j < 0 || (j > 0 && t.p0 >= t.end)) t.g = -1;
    return t;
}

// The last group, of G + 1, that starts at position pos or before it: the one that holds pos.
__device__ __forceinline__ int group_at(const RowOrder &o, int64_t pos)
{
    const int lane = threadIdx.x & 63;
    int lo = 0, len = o.G + 1;  // it lies in [lo, lo + len)
    while (len > 1) {
        const int s = (len + 63) / 64;
        const bool in = lane * s < len;
        const int cnt = __popcll(__ballot(in && clamp_offset(o.offsets[in ? lo + lane * s : lo], o.n) <= pos));
        const int skip = (cnt > 0 ? cnt - 1 : 0) * s;
        lo += skip;
        len = len - skip < s ? len - skip : s;
    }
    return __builtin_amdgcn_readfirstlane(lo);
}

// Tile j of a group of more than kFewRows rows, where the others are looked after elsewhere: index m is for
// the group that holds position (m + 1) kFewRows, and the i-th such index of a group for its tile i. A group of
// n rows, n > kFewRows, holds at least floor((n - 1) / kFewRows) such positions beyond its start, no fewer than
// tiles of 2 kFewRows.
__device__ __forceinline__ Tile find_big(const RowOrder &o, int R, int64_t m)
{
    const int lo = group_at(o, (m + 1) * kFewRows);
    Tile t;
    t.g = -1;
    if (lo >= o.G) return t;
    t.start = clamp_offset(o.offsets[lo], o.n);
    t.end = clamp_offset(o.offsets[lo + 1], o.n);
    const int64_t i = m - t.start / kFewRows;
    t.p0 = t.start + i * R;
    t.p1 = t.p0 + R < t.end ? t.p0 + R : t.end;
    if (t.end - t.start > kFewRows && i >= 0 && t.p0 < t.end) t.g = lo;
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

// 16 and 8 bytes of values at the alignment of one (global memory accesses need no more).
typedef uint4_t uint4_any __attribute__((aligned(2)));
typedef uint2_t uint2_any __attribute__((aligned(2)));
typedef float4_t float4_any __attribute__((aligned(4)));
typedef bf4_t bf4_any __attribute__((aligned(2)));

// 16 bytes of values from p on, zero past the `left` that exist.
template <typename T, bool VEC>
__device__ __forceinline__ uint4_t load_16(const T *p, int64_t left)
{
    constexpr int V = 16 / (int)sizeof(T);
    uint4_t v = {0, 0, 0, 0};
    if (left >= V) {
        if (VEC) v = *reinterpret_cast<const uint4_t *>(p);
        else v = *reinterpret_cast<const uint4_any *>(p);
    } else if (!VEC && left > 0) {
#pragma unroll
        for (int e = 0; e < V; ++e)
            if (left > e) {
                if (sizeof(T) == 4) v[e % 4] = reinterpret_cast<const unsigned *>(p)[e];
                else v[e / 2] |= (unsigned)reinterpret_cast<const unsigned short *>(p)[e] << (e % 2 * 16);
            }
    }
    return v;
}

// The same for 8 bytes: kWide values.
template <typename T, bool VEC>
__device__ __forceinline__ uint2_t load_8(const T *p, int64_t left)
{
    constexpr int V = 8 / (int)sizeof(T);
    uint2_t v = {0, 0};
    if (left >= V) {
        if (VEC) v = *reinterpret_cast<const uint2_t *>(p);
        else v = *reinterpret_cast<const uint2_any *>(p);
    } else if (!VEC && left > 0) {
#pragma unroll
        for (int e = 0; e < V; ++e)
            if (left > e) {
                if (sizeof(T) == 4) v[e % 2] = reinterpret_cast<const unsigned *>(p)[e];
                else v[e / 2] |= (unsigned)reinterpret_cast<const unsigned short *>(p)[e] << (e % 2 * 16);
            }
    }
    return v;
}

// Eight consecutive k of a lane as loaded: one unit of bf16, or 32 bytes of fp32.
template <typename T> struct Raw8 { uint4_t v[sizeof(T) / 2]; };

template <typename T, bool VEC>
__device__ __forceinline__ Raw8<T> load_row8(const T *p, int64_t left)
{
    Raw8<T> r;
    r.v[0] = load_16<T, VEC>(p, left);
    if constexpr (sizeof(T) == 4) r.v[1] = load_16<T, VEC>(p + 4, left - 4);
    return r;
}

// Loads that must not pass the end of a row, and must not be under a condition, start early enough to end
// with it; the values are moved down by what they started early when they are staged.

// Eight values at the alignment of one.
template <typename T> __device__ __forceinline__ Raw8<T> load_any8(const T *q)
{
    Raw8<T> r;
    r.v[0] = *reinterpret_cast<const uint4_any *>(q);
    if constexpr (sizeof(T) == 4) r.v[1] = *reinterpret_cast<const uint4_any *>(q + 4);
    return r;
}

// Moves the values down by `early`, and leaves zeros from value `left` on.
template <typename T> __device__ __forceinline__ void settle(Raw8<T> &r, int early, int left)
{
    constexpr int D = (int)sizeof(T) * 2;  // registers
    for (int i = 0; i < early; ++i) {
#pragma unroll
        for (int e = 0; e < D; ++e) {
            const unsigned v = r.v[e / 4][e % 4], up = e + 1 < D ? r.v[(e + 1) / 4 % (D / 4)][(e + 1) % 4] : 0u;
            r.v[e / 4][e % 4] = sizeof(T) == 4 ? up : v >> 16 | up << 16;
        }
    }
#pragma unroll
    for (int e = 0; e < D; ++e) {
        const int first = e * 4 / (int)sizeof(T);  // of the values in this register
        const unsigned v = r.v[e / 4][e % 4];
        r.v[e / 4][e % 4] = first + (sizeof(T) == 2) < left ? v : first < left ? v & 0xffffu : 0u;
    }
}

// The same for transposed loads of kWide columns, whose values past the last column are never used.
template <typename T> __device__ __forceinline__ void settle(uint2_t &v, int early)
{
    for (int i = 0; i < early; ++i) {
        v[0] = sizeof(T) == 4 ? v[1] : v[0] >> 16 | v[1] << 16;
        v[1] = sizeof(T) == 4 ? 0u : v[1] >> 16;
    }
}

// Of fp32 operands as parts, and of the sums of their products.
constexpr float kUp = 0x1p16f, kDown = 0x1p-32f;

// The three parts of eight values.
__device__ __forceinline__ void split8(const float (&x)[8], uint4_t (&part)[3])
{
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        float r0 = x[2 * k], r1 = x[2 * k + 1];
#pragma unroll
        for (int c = 0; c < 3; ++c) {
            const bf2_t b = {(bf16_t)r0, (bf16_t)r1};
            const unsigned bits = __builtin_bit_cast(unsigned, b);
            part[c][k] = bits;
            r0 -= __builtin_bit_cast(float, bits << 16);
            r1 -= __builtin_bit_cast(float, bits & 0xffff0000u);
        }
    }
}

// Adds NaN to `odd` if one of the sums is not finite, else zero.
__device__ __forceinline__ void probe(float &odd, const float16_t &sum)
{
#pragma unroll
    for (int i = 0; i < 16; ++i) odd = fmaf(sum[i], 0.f, odd);
}

// The units of a lane's eight k; of fp32 times sign, 1 or -1.
__device__ __forceinline__ void to_units(const Raw8<bf16_t> &raw, uint4_t (&u)[1], float = 1.f)
{
    u[0] = raw.v[0];
}
__device__ __forceinline__ void to_units(const Raw8<float> &raw, uint4_t (&u)[3], float sign = 1.f)
{
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = sign * kUp * __builtin_bit_cast(float, (unsigned)raw.v[e / 4][e % 4]);
    split8(x, u);
}

// The units of kWide lanes from 8 loads of 8 bytes.
__device__ __forceinline__ void to_units(const uint2_t (&in)[8], uint4_t (&u)[4][1], float = 1.f)
{
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            u[j][0][e] = __builtin_amdgcn_perm(in[2 * e + 1][j >> 1], in[2 * e][j >> 1],
                                               (j & 1) ? 0x07060302u : 0x05040100u);
}

__device__ __forceinline__ void to_units(const uint2_t (&in)[8], uint4_t (&u)[2][3], float sign = 1.f)
{
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = sign * kUp * __builtin_bit_cast(float, (unsigned)in[e][j]);
        split8(x, u[j]);
    }
}

// Writes a lane's units, all parts of k-group kg, to place r of a tile of R.
template <typename T, int R>
__device__ __forceinline__ void put(uint4_t *tile, int groups, int kg, int r, const uint4_t (&u)[kSplit<T>])
{
#pragma unroll
    for (int c = 0; c < kSplit<T>; ++c) tile[(c * groups + kg) * (R + 1) + r] = u[c];
}

// Where a transposed operand's lane r lies in its block of 32.
template <typename T> __device__ __forceinline__ int place(int r)
{
    return sizeof(T) == 2 ? (r & ~31) | (r & 3) << 3 | (r >> 2 & 7) : (r & ~31) | (r & 1) << 4 | (r >> 1 & 15);
}

// The forms for 16-byte loads (rows_outer.hip): the units of kFull lanes, their places, and the columns that a
// lane's sums hold. bf16's eight units go four apart in a block of 32, in odd blocks with the halves of the
// wave exchanged, so that neighbouring threads and blocks write to different banks.
template <typename T> constexpr int kFull = 16 / (int)sizeof(T);

__device__ __forceinline__ void to_units(const uint4_t (&in)[8], uint4_t (&u)[8][1], float = 1.f)
{
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            u[j][0][e] = __builtin_amdgcn_perm(in[2 * e + 1][j >> 1], in[2 * e][j >> 1],
                                               (j & 1) ? 0x07060302u : 0x05040100u);
}

__device__ __forceinline__ void to_units(const uint4_t (&in)[8], uint4_t (&u)[4][3], float sign = 1.f)
{
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = sign * kUp * __builtin_bit_cast(float, (unsigned)in[e][j]);
        split8(x, u[j]);
    }
}

template <typename T> __device__ __forceinline__ int place_full(int r)
{
    if (sizeof(T) == 4) return (r & ~31) | (r & 3) << 3 | (r >> 2 & 7);
    return (r & ~31) | (r & 3) << 3 | ((r >> 2 ^ r >> 5) & 1) << 2 | (r >> 3 & 3);
}
template <typename T> __device__ __forceinline__ int lane_of_full(int p)
{
    if (sizeof(T) == 4) return (p & ~31) | (p & 7) << 2 | (p >> 3 & 3);
    return (p & ~31) | (p & 3) << 3 | ((p >> 2 ^ p >> 5) & 1) << 2 | (p >> 3 & 3);
}

// Four consecutive columns, v = 0..3, of the block of 32 that starts at place p: the first, from p on; the
// values are the sums v, 4 + v, 8 + v, 12 + v.
template <typename T> __device__ __forceinline__ int vec_col_full(int p, int v, int half)
{
    return p + (sizeof(T) == 4 ? 4 * (4 * half + v) : 8 * v + 4 * (half ^ (p >> 5 & 1)));
}

template <typename T> __device__ __forceinline__ void settle(uint4_t &v, int early)
{
    for (int i = 0; i < early; ++i) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const unsigned up = e < 3 ? v[(e + 1) % 4] : 0u;
            v[e] = sizeof(T) == 4 ? up : v[e] >> 16 | up << 16;
        }
    }
}

__device__ __forceinline__ void mfma(float16_t &acc, uint4_t a, uint4_t b)
{
    acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf8_t, a),
                                                  __builtin_bit_cast(bf8_t, b), acc, 0, 0, 0);
}

// acc += A B for one unit of each lane (lanes 0..31 carry k-group 2 s, lanes 32..63 2 s + 1), the smallest
// terms first.
__device__ __forceinline__ void mma(float16_t &acc, const uint4_t (&a)[1], const uint4_t (&b)[1])
{
    mfma(acc, a[0], b[0]);
}
__device__ __forceinline__ void mma(float16_t &acc, const uint4_t (&a)[3], const uint4_t (&b)[3])
{
    mfma(acc, a[0], b[2]);
    mfma(acc, a[2], b[0]);
    mfma(acc, a[1], b[1]);
    mfma(acc, a[0], b[1]);
    mfma(acc, a[1], b[0]);
    mfma(acc, a[0], b[0]);
}

// The products of a step: TC blocks of 32 columns (from unit column c0 of cols) by TR blocks of 32
// rows. acc[c][r][i]: column place 8 (i / 4) + 4 (lane / 32) + i % 4 of block c, row place lane % 32 of
// block r. All k-groups always, zeros past the end: a branch around a matrix instruction costs a copy of
// its sums.
//
// The matrix instruction rounds its sums down, towards minus infinity (measured: results of 896 terms low by
// 4e-8 of their spread on the mean, which a later sum over many rows picks up). fp32 products therefore sum
// a step from zero and add it in fp32, and every other step has its rows negated and is subtracted (sign). bf16
// products keep it: against sums in 64 bits rounded to bf16, results are low by 1e-8 of their magnitude on the mean
// for up to 1,344 terms and for chunks of 16,384 rows, by 1.6e-7 for 20,000 terms of one sign, and 5e-6 to 6e-4 of
// them are another bf16 number (of fp32 sums in another order 1e-3).
template <typename T, int BN, int BM, int TC, int TR, int TX>
__device__ __forceinline__ void step_products(float16_t (&acc)[TX][TR], const uint4_t *cols,
                                              const uint4_t *rws, int c0, int r0, float sign)
{
    constexpr int Q = kSplit<T>, KG = kGroups<T>, S = KG / 2;
    const int lane = threadIdx.x & 63, half = lane >> 5, n = lane & 31;
    if constexpr (Q == 1) {
#pragma unroll
        for (int s = 0; s < S; ++s) {
            uint4_t a[TC][1], b[TR][1];
#pragma unroll
            for (int c = 0; c < TC; ++c) a[c][0] = cols[(2 * s + half) * (BN + 1) + c0 + 32 * c + n];
#pragma unroll
            for (int r = 0; r < TR; ++r) b[r][0] = rws[(2 * s + half) * (BM + 1) + r0 + 32 * r + n];
#pragma unroll
            for (int c = 0; c < TC; ++c)
#pragma unroll
                for (int r = 0; r < TR; ++r) mma(acc[c][r], a[c], b[r]);
        }
    } else {
#pragma unroll
        for (int r = 0; r < TR; ++r) {
            uint4_t b[S][Q];
#pragma unroll
            for (int s = 0; s < S; ++s)
#pragma unroll
                for (int q = 0; q < Q; ++q) b[s][q] = rws[(q * KG + 2 * s + half) * (BM + 1) + r0 + 32 * r + n];
#pragma unroll
            for (int c = 0; c < TC; ++c) {
                float16_t sum;
#pragma unroll
                for (int i = 0; i < 16; ++i) sum[i] = 0.f;
#pragma unroll
                for (int s = 0; s < S; ++s) {
                    uint4_t a[Q];
#pragma unroll
                    for (int q = 0; q < Q; ++q) a[q] = cols[(q * KG + 2 * s + half) * (BN + 1) + c0 + 32 * c + n];
                    mma(sum, a, b[s]);
                }
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[c][r][i] = fmaf(sign * kDown, sum[i], acc[c][r][i]);
            }
        }
    }
}

// Four consecutive columns of a lane's row, v = 0..3: the first of them, and the values. With a
// transposed column operand they come from the places that place() gives them.
template <typename T, bool TRANS> __device__ __forceinline__ int vec_col(int v, int half)
{
    if (!TRANS) return 8 * v + 4 * half;
    return sizeof(T) == 2 ? 4 * (4 * half + v) : 4 * (2 * half + (v & 1) + 4 * (v >> 1));
}

template <typename T, bool TRANS> __device__ __forceinline__ float4_t vec_val(const float16_t &acc, int v)
{
    if (!TRANS) return float4_t{acc[4 * v], acc[4 * v + 1], acc[4 * v + 2], acc[4 * v + 3]};
    if (sizeof(T) == 2) return float4_t{acc[v], acc[4 + v], acc[8 + v], acc[12 + v]};
    const int i = 4 * (v >> 1) + 2 * (v & 1);
    return float4_t{acc[i], acc[i + 8], acc[i + 1], acc[i + 9]};
}

// Stores four consecutive values, of which `left` exist.
template <bool VEC> __device__ __forceinline__ void store_four(float *p, float4_t v, int64_t left)
{
    if (VEC) {
        if (left > 0) *reinterpret_cast<float4_t *>(p) = v;
        return;
    }
    if (left >= 4) {
        *reinterpret_cast<float4_any *>(p) = v;
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
    if (left >= 4) {
        *reinterpret_cast<bf4_any *>(p) = h;
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
// order: fp32 [n][W], or for bf16 three parts [n][3][W], fp32's 24 bits of significand; W is N
// rounded up to a unit, the rest zero.
__host__ __device__ constexpr int narrow_width(int N) { return (N + kU - 1) / kU * kU; }
template <typename T> constexpr int kNarrow = sizeof(T) == 2 ? 3 : 1;

// The three bf16 parts of four values; an infinity or NaN has one.
__device__ __forceinline__ void narrow_parts(float4_t x, bf4_t (&part)[3])
{
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        part[0][e] = (bf16_t)x[e];
        const float r = __builtin_isfinite((float)part[0][e]) ? x[e] - (float)part[0][e] : 0.f;
        part[1][e] = (bf16_t)r;
        part[2][e] = (bf16_t)(r - (float)part[1][e]);
    }
}

// Values 4 half .. 4 half + 3 of k-group g of a narrow result's row of `groups`, as operands in a tile of R rows
// at place r; of bf16 the parts first .. first + count - 1, each behind the one before. k-groups that they do
// not reach come as zeros.
template <typename T, int R>
__device__ __forceinline__ void put_narrow(uint4_t *tile, int g, int r, int half, int groups, int first, int count,
                                           float4_t x)
{
    auto at = [&](int group) { return reinterpret_cast<uint2_t *>(tile + group * (R + 1) + r) + half; };
    if constexpr (sizeof(T) == 2) {
        bf4_t part[3];
        narrow_parts(x, part);
#pragma unroll
        for (int e = 0; e < 3; ++e)
            if (g < groups && e >= first && e < first + count)
                *at((e - first) * groups + g) = __builtin_bit_cast(uint2_t, part[e]);
        for (int z = count * groups; z < kGroups<T>; ++z)
            if (z % 4 == g) *at(z) = uint2_t{0, 0};
    } else {
        x *= kUp;
#pragma unroll
        for (int c = 0; c < 3; ++c) {
            const bf4_t b = {(bf16_t)x[0], (bf16_t)x[1], (bf16_t)x[2], (bf16_t)x[3]};
            *at(c * kGroups<T> + g) = __builtin_bit_cast(uint2_t, b);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] -= (float)b[e];
        }
    }
}

// Where the parts of a narrow result meet the same weights again: k of the parts' row as k of the weights.
template <typename T> __device__ __forceinline__ int narrow_k(int k, int W)
{
    if (kNarrow<T> == 1) return k;
    return k >= 2 * W ? k - 2 * W : k >= W ? k - W : k;
}

template <typename T> __device__ __forceinline__ float narrow_at(const void *h, int64_t pos, int W, int k)
{
    const T *const p = static_cast<const T *>(h) + pos * (kNarrow<T> * W) + k;
    return sizeof(T) == 2 ? (float)p[0] + (float)p[W] + (float)p[2 * W] : (float)p[0];
}

// Waves along the rows of a 128 x 128 tile: fp32 operands, three parts each, are read once a wave where it
// has rows of its own.
template <typename T> constexpr int kWaveRows = sizeof(T) == 2 ? 2 : 4;

// A result that this workgroup has stored, past the caches that other workgroups' stores do not reach.
__device__ __forceinline__ float stored(const float *p)
{
    return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float stored(const bf16_t *p)
{
    const unsigned short bits = __hip_atomic_load(reinterpret_cast<const unsigned short *>(p), __ATOMIC_RELAXED,
                                                  __HIP_MEMORY_SCOPE_AGENT);
    return __builtin_bit_cast(float, (unsigned)bits << 16);
}

// Every wave's stores are done: what follows reads and replaces some of them.
__device__ __forceinline__ void stores_done()
{
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
}

// The results of a workgroup that are not finite, in the columns [c0, c1) of its rows, in plain fp32. h: the
// narrow product's rows in LDS, 32 apart, in place of p.h.
template <typename T, bool WNK>
__device__ void row_plain_sums(const RowOrder &o, const RowProduct &p, int group, int64_t p0, int rows, const int *s_row,
                               const int *s_g, int c0, int c1, const float *h = nullptr)
{
    stores_done();
    const int W = narrow_width(p.r), width = c1 - c0;
    const T *const w = static_cast<const T *>(p.w) + (int64_t)group * p.w_group;
    for (int e = threadIdx.x; e < rows * width; e += kThreads) {
        const int r = e / width, c = c0 + e % width;
        if (s_row[r] < 0) continue;
        float *const narrow_out = static_cast<float *>(p.out) + (p0 + r) * narrow_width(p.N) + c;  // fp32 alone
        T *const out = static_cast<T *>(p.out) + s_row[r] * p.out_stride + c;
        const bool narrow = sizeof(T) == 4 && p.narrow;
        if (__builtin_isfinite(narrow ? stored(narrow_out) : stored(out))) continue;
        const T *const in = static_cast<const T *>(p.in) + s_row[r] * p.in_stride;
        float sum = 0.f;
        auto term = [&](int k) { return (float)in[k] * (float)w[WNK ? (int64_t)c * p.K + k : (int64_t)k * p.N + c]; };
        int k0 = 0;
        for (; k0 + 8 <= p.K && sum == sum; k0 += 8)  // NaN stays
#pragma unroll
            for (int u = 0; u < 8; ++u) sum += term(k0 + u);
        for (; k0 < p.K && sum == sum; ++k0) sum += term(k0);
        if ((p.h || h) && s_g[r] < o.G) {
            const T *const v = static_cast<const T *>(p.v) + (int64_t)s_g[r] * p.r * p.N;
            for (int k = 0; k < p.r; ++k)
                sum += (h ? h[32 * r + k] : narrow_at<T>(p.h, p0 + r, W, k)) *
                       (float)v[WNK ? (int64_t)c * p.r + k : (int64_t)k * p.N + c];
        }
        if (narrow) *narrow_out = p.narrow_scale ? sum * p.narrow_scale[group] : sum;
        else *out = (T)sum;
    }
}

__device__ __forceinline__ void store_narrow(float *p, int W, float4_t v)
{
    *reinterpret_cast<float4_t *>(p) = v;
}

__device__ __forceinline__ void store_narrow(bf16_t *p, int W, float4_t v)
{
    bf4_t part[3];
    narrow_parts(v, part);
#pragma unroll
    for (int e = 0; e < 3; ++e) *reinterpret_cast<bf4_t *>(p + e * W) = part[e];
}

// Whether rows at this stride start on 16-byte boundaries.
template <typename T> bool aligned_rows(const void *p, int64_t stride)
{
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride * (int64_t)sizeof(T) % 16 == 0;
}

}  // namespace rows
}  // namespace cgtp

#endif
