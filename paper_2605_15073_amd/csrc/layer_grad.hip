// The gradients of a narrow layer (up to kWidth inputs and outputs) in one pass over its rows: dz is formed once, from
// dy and z as they are read, and serves both products. Whichever of them are asked for, each has the same bits.
//
// A workgroup owns a chunk of a group's rows and takes them kTileRows at a time. Half of the waves load x, half dy and z,
// 8 rows by 4 columns a thread, a tile ahead; both are staged transposed, units of 8 rows, for dw = x^T dz, whose sums
// stay in registers over the chunk, and dz as it lies, units of 8 columns, for dx = dz W^T. W stays in registers: each
// wave has a 32 x 32 block of either product. Sums of dz's columns are dbias. Chunks of a long group leave their sums in
// slots, which k_row_join adds in order.
//
// dz is held in three bf16 parts in fp32 and in two in bf16, 16 bits of significand: the second product is in the shadow
// of memory, and dx and dw are as exact as their own rounding. What is not finite is formed again (rows_tile.h).
#include "internal.h"
#include "rows_layer.h"

#include <cmath>

namespace cgtp {

namespace {

using namespace rows;

constexpr int kWidth = 64, kTileRows = 64, kLD = kWidth + 1;
constexpr int kCW = 4;             // columns of a thread's block
constexpr int kHalf = kThreads / 2;
static_assert(kTileRows / 8 * (kWidth / kCW) == kHalf, "a block a thread");

template <typename T> struct Block;  // 4 values of a row
template <> struct Block<float> { typedef uint4_t raw; typedef uint4_any any; };
template <> struct Block<bf16_t> { typedef uint2_t raw; typedef uint2_any any; };

__device__ __forceinline__ float4_t unpack(uint4_t v) { return __builtin_bit_cast(float4_t, v); }
__device__ __forceinline__ float4_t unpack(uint2_t v)
{
    return float4_t{__builtin_bit_cast(float, v[0] << 16), __builtin_bit_cast(float, v[0] & 0xffff0000u),
                    __builtin_bit_cast(float, v[1] << 16), __builtin_bit_cast(float, v[1] & 0xffff0000u)};
}

// The transposed units of a block in fp32, of columns j: P parts of eight rows; fp32's of 2^16 times sign.
template <typename T, int P>
__device__ __forceinline__ void parts_of(const float4_t (&in)[8], uint4_t (&u)[kCW][P], float sign)
{
    if constexpr (sizeof(T) == 4) {
        static_assert(P == 3, "fp32");
#pragma unroll
        for (int j = 0; j < kCW; ++j) {
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = sign * kUp * in[e][j];
            split8(x, u[j]);
        }
    } else {
#pragma unroll
        for (int j = 0; j < kCW; ++j)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float a = in[2 * k][j], b = in[2 * k + 1][j];
                if constexpr (P > 1) {
                    unsigned high, low;
                    split_pair(a, b, high, low);
                    u[j][0][k] = high;
                    u[j][1][k] = low;
                } else u[j][0][k] = pack_pair(a, b);
            }
    }
}

// dz of one value, for the sums that are formed again.
template <typename T, bool HAS_Z>
__device__ __forceinline__ float one_dz(const LayerGrad &q, int64_t row, int n)
{
    const float g = (float)static_cast<const T *>(q.dy)[row * q.dy_stride + n];
    return HAS_Z ? g * activate_slope<T>((float)static_cast<const T *>(q.z)[row * q.z_stride + n], q.act) : g;
}

// DW: dw is asked for; else nothing of x is read.
template <typename T, bool HAS_Z, bool DW>
__global__ __launch_bounds__(kThreads, sizeof(T) == 4 ? 2 : 3) void k_layer_grad(RowOrder o, LayerGrad q, ChunkRows R,
                                                                               float *slots)
{
    typedef typename Block<T>::raw Raw;
    typedef typename Block<T>::any Any;
    constexpr int Q = kSplit<T>, P = sizeof(T) == 4 ? 3 : HAS_Z ? 2 : 1;  // parts of x and w, of dz
    constexpr int KG = kGroups<T>, SUB = kTileRows / (8 * KG);            // steps of the products over rows
    __shared__ uint4_t s_zt[SUB][P][KG * kLD], s_xt[SUB][Q][KG * kLD], s_zr[P][kWidth / 8 * kLD];
    __shared__ int64_t s_at[3][2][kTileRows];  // where the rows of x, dy and z of a tile start
    __shared__ int s_row[2][kTileRows];
    const Tile t = find_tile(o, R, tile_at(blockIdx.x, blockIdx.z, gridDim.x));
    if (t.g < 0 || t.p0 >= t.p1) {
        if (t.g < 0 || t.g >= o.G || t.start < t.end) return;  // else a group without rows: zeros
    }
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    auto put_dx = [&](int64_t row, int col, float4_t v) {
        if (q.dx_f32) store_four<false>(static_cast<float *>(q.dx) + row * q.dx_stride + col, v, q.K - col);
        else store_four<false>(static_cast<T *>(q.dx) + row * q.dx_stride + col, v, q.K - col);
    };
    if (t.g == o.G) {  // rows of no group
        if (!q.dx) return;
        const int quads = (q.K + 3) / 4;
        for (int i = tid; i < (int)(t.p1 - t.p0) * quads; i += kThreads) {
            const int row = row_at(o, t.p0 + i / quads);
            if (row >= 0) put_dx(row, 4 * (i % quads), float4_t{0.f, 0.f, 0.f, 0.f});
        }
        return;
    }
    const int wr = wave % 2, wc = wave / 2;
    const bool of_z = wave >= 2;
    const int width = of_z ? q.N : q.K;
    const int kg = tid % kHalf / (kWidth / kCW), first = kCW * (tid % (kWidth / kCW));
    const int start = first + kCW <= width ? first : width - kCW, early = first < width ? first - start : 0;
    const int64_t array = of_z ? 1 : 0;

    // w: columns k of this wave's block of dx, units of n
    uint4_t w[kWidth / 16][Q];
    if (q.dx) {
        const int k = 32 * wc + (lane & 31);
        const T *const row = static_cast<const T *>(q.w) + ((int64_t)t.g * q.K + (k < q.K ? k : 0)) * q.N;
#pragma unroll
        for (int s = 0; s < kWidth / 16; ++s) {
            const int n = (2 * s + half) * kU;
            to_units(load_row8<T, false>(row + n, k < q.K ? q.N - n : 0), w[s]);
        }
    }

    const int steps = (int)((t.p1 - t.p0 + kTileRows - 1) / kTileRows);
    const int32_t *const ids_at = o.order ? o.order : o.offsets;
    int id = -1;
    auto fetch_ids = [&](int s) {
        const int64_t pos = t.p0 + (int64_t)s * kTileRows + tid % kTileRows;
        id = ids_at[o.order && pos < t.p1 ? pos : 0];
    };
    auto put_ids = [&](int s) {
        if (tid >= kTileRows) return;
        const int64_t pos = t.p0 + (int64_t)s * kTileRows + tid;
        const int row = o.order ? id : (int)pos;
        const bool in = pos < t.p1 && (unsigned)row < (unsigned)o.n;
        const int any = in ? row : 0;  // row 0 in place of none: zeroed when staged
        s_row[s & 1][tid] = in ? row : -1;
        s_at[0][s & 1][tid] = (q.per > 1 ? (int)((unsigned)any / (unsigned)q.per) : any) * q.x_stride;
        s_at[1][s & 1][tid] = any * q.dy_stride;
        s_at[2][s & 1][tid] = any * q.z_stride;
    };
    Raw l[8], lz[HAS_Z ? 8 : 1];
    unsigned in = 0;  // bit u: row u of the block exists
    auto fetch = [&](int s) {
        if (!DW && !of_z) return;
        const T *const from = static_cast<const T *>(of_z ? q.dy : q.x) + start;
        in = 0;
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            l[u] = *reinterpret_cast<const Any *>(from + s_at[array][s & 1][8 * kg + u]);
            if (s_row[s & 1][8 * kg + u] >= 0) in |= 1u << u;
        }
        if (HAS_Z && of_z)
#pragma unroll
            for (int u = 0; u < 8; ++u)
                lz[u] = *reinterpret_cast<const Any *>(static_cast<const T *>(q.z) + start + s_at[2][s & 1][8 * kg + u]);
    };
    float column[kCW] = {0.f, 0.f, 0.f, 0.f};
    auto stage = [&]() {
        if (!DW && !of_z) return;
        const int sub = kg / KG, g = kg % KG;
        float4_t f[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            f[u] = unpack(l[u]);
            if (HAS_Z && of_z) {
                const float4_t a = unpack(lz[u]);
#pragma unroll
                for (int e = 0; e < 4; ++e) f[u][e] *= activate_slope<T>(a[e], q.act);
            }
        }
        if (early > 0)
#pragma unroll
            for (int u = 0; u < 8; ++u)
                for (int i = 0; i < early; ++i) f[u] = float4_t{f[u][1], f[u][2], f[u][3], 0.f};
        if (in != 0xffu || first >= width)
#pragma unroll
            for (int u = 0; u < 8; ++u)
                if (!(in >> u & 1) || first >= width) f[u] = float4_t{0.f, 0.f, 0.f, 0.f};
        if (of_z) {
#pragma unroll
            for (int e = 0; e < kCW; ++e) column[e] += sum_of_eight([&](int u) { return f[u][e]; });
            uint4_t u[kCW][P];
            parts_of<T, P>(f, u, 1.f);
#pragma unroll
            for (int c = 0; c < P; ++c)
#pragma unroll
                for (int j = 0; j < kCW; ++j) s_zt[sub][c][g * kLD + place_full<float>(first + j)] = u[j][c];
            // the same parts by rows: half a unit of four columns
#pragma unroll
            for (int c = 0; c < P; ++c)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    uint2_t *const to = reinterpret_cast<uint2_t *>(s_zr[c] + first / 8 * kLD + 8 * kg + 2 * k) + (first / 4 & 1);
                    to[0] = uint2_t{__builtin_amdgcn_perm(u[1][c][k], u[0][c][k], 0x05040100u),
                                    __builtin_amdgcn_perm(u[3][c][k], u[2][c][k], 0x05040100u)};
                    to[2] = uint2_t{__builtin_amdgcn_perm(u[1][c][k], u[0][c][k], 0x07060302u),
                                    __builtin_amdgcn_perm(u[3][c][k], u[2][c][k], 0x07060302u)};
                }
        } else {
            uint4_t u[kCW][Q];
            parts_of<T, Q>(f, u, sub % 2 ? -1.f : 1.f);  // every other step is summed negated (step_products)
#pragma unroll
            for (int c = 0; c < Q; ++c)
#pragma unroll
                for (int j = 0; j < kCW; ++j) s_xt[sub][c][g * kLD + place_full<float>(first + j)] = u[j][c];
        }
    };

    float16_t dw[1][1];
#pragma unroll
    for (int i = 0; i < 16; ++i) dw[0][0][i] = 0.f;
    float odd = 0.f;  // NaN once a result is not finite
    auto product_dx = [&](int s) {
        float16_t sum;
#pragma unroll
        for (int i = 0; i < 16; ++i) sum[i] = 0.f;
        const uint4_t *const z = s_zr[0] + half * kLD + 32 * wr + (lane & 31);
#pragma unroll
        for (int k = 0; k < kWidth / 16; ++k) {
            if constexpr (Q > 1) {
                uint4_t b[Q];
#pragma unroll
                for (int c = 0; c < Q; ++c) b[c] = z[(c * (kWidth / 8) + 2 * k) * kLD];
                mma(sum, w[k], b);
            } else {
#pragma unroll
                for (int c = P - 1; c >= 0; --c) mfma(sum, w[k][0], z[(c * (kWidth / 8) + 2 * k) * kLD]);
            }
        }
        probe(odd, sum);
        const int row = s_row[s & 1][32 * wr + (lane & 31)];
        if (row < 0) return;
#pragma unroll
        for (int v = 0; v < 4; ++v)
            put_dx(row, 32 * wc + vec_col<T, false>(v, half), (Q > 1 ? kDown : 1.f) * vec_val<T, false>(sum, v));
    };
    if (steps > 0) {
        fetch_ids(0);
        put_ids(0);
        fetch_ids(1);
        __syncthreads();
        fetch(0);
        for (int s = 0; s < steps; ++s) {
            __syncthreads();
            stage();
            put_ids(s + 1);
            __syncthreads();
            fetch_ids(s + 2);
            fetch(s + 1);
            if (q.dx) product_dx(s);
#pragma unroll
            for (int i = 0; i < (DW ? SUB : 0); ++i)
                if constexpr (Q > 1) {
                    step_products<T, kWidth, kWidth, 1, 1>(dw, s_zt[i][0], s_xt[i][0], 32 * wc, 32 * wr, i % 2 ? -1.f : 1.f);
                } else {
#pragma unroll
                    for (int c = P - 1; c >= 0; --c)
                        step_products<T, kWidth, kWidth, 1, 1>(dw, s_zt[i][c], s_xt[i][0], 32 * wc, 32 * wr, 1.f);
                }
        }
    }
    const bool whole = t.end - t.start <= R.rows;
    const int64_t of_w = (int64_t)q.K * q.N, cells = DW ? of_w : 0, slot_cells = cells + (q.dbias ? q.N : 0);
    const int64_t slot = 2 * (int64_t)R.of((int)t.start) + R.of((int)(t.p0 - t.start));
    T *const out = static_cast<T *>(q.dw) + t.g * cells;
    float *const part = slots + (whole ? 0 : slot * slot_cells);
    __syncthreads();
    if (q.dbias) {
        float *const of_kg = reinterpret_cast<float *>(s_zr);  // [8][kWidth]
        if (of_z)
#pragma unroll
            for (int j = 0; j < kCW; ++j) of_kg[kg * kWidth + first + j] = column[j];
        __syncthreads();
        if (tid < q.N) {
            float sum = 0.f;
#pragma unroll
            for (int g = 0; g < kTileRows / 8; ++g) sum += of_kg[g * kWidth + tid];
            if (whole) static_cast<T *>(q.dbias)[(int64_t)t.g * q.N + tid] = (T)sum;
            else part[cells + tid] = sum;
        }
    }
    const int i = lane_of_full<float>(32 * wr + (lane & 31));
    if (DW && i < q.K)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const int col = vec_col_full<float>(32 * wc, v, half);
            const float4_t x = {dw[0][0][v], dw[0][0][4 + v], dw[0][0][8 + v], dw[0][0][12 + v]};
            const int64_t at = (int64_t)i * q.N + col;
            if (whole) store_four<false>(out + at, x, q.N - col);
            else store_four<false>(part + at, x, q.N - col);
        }
    if (Q == 1 && P == 1) return;
    if (DW) probe(odd, dw[0][0]);
    if (!__syncthreads_or(odd != odd)) return;
    // the results that are not finite, in plain fp32
    stores_done();
    const T *const wg = static_cast<const T *>(q.w) + (int64_t)t.g * of_w;
    if (q.dx)
        for (int64_t e = tid; e < (t.p1 - t.p0) * q.K; e += kThreads) {
            const int row = row_at(o, t.p0 + e / q.K), k = (int)(e % q.K);
            if (row < 0) continue;
            const int64_t at = row * q.dx_stride + k;
            float *const wide = static_cast<float *>(q.dx) + at;
            T *const to = static_cast<T *>(q.dx) + at;
            if (__builtin_isfinite(q.dx_f32 ? stored(wide) : stored(to))) continue;
            float sum = 0.f;
            for (int n = 0; n < q.N; ++n) sum = fmaf(one_dz<T, HAS_Z>(q, row, n), (float)wg[(int64_t)k * q.N + n], sum);
            if (q.dx_f32) *wide = sum;
            else *to = (T)sum;
        }
    for (int e = tid; e < (int)cells; e += kThreads) {
        if (__builtin_isfinite(whole ? stored(out + e) : stored(part + e))) continue;
        const int k = e / q.N, n = e % q.N;
        float sum = 0.f;
        for (int64_t pos = t.p0; pos < t.p1 && sum == sum; ++pos) {  // NaN stays
            const int row = row_at(o, pos);
            if (row < 0) continue;
            const int64_t from = (int64_t)((unsigned)row / (unsigned)q.per) * q.x_stride + k;
            sum = fmaf((float)static_cast<const T *>(q.x)[from], one_dz<T, HAS_Z>(q, row, n), sum);
        }
        if (whole) out[e] = (T)sum;
        else part[e] = sum;
    }
}

// Rows of a chunk: of sizes about 6% apart that with the least of the rounds that workgroups run in, as many as the GPU
// holds at once, each as long as a chunk, and of the slots' traffic.
int chunk_rows(size_t es, int64_t n, int G, int K, int N)
{
    const double at_once = 256 * (es == 4 ? 2 : 3), groups = (double)(n < G ? n : G), mean = n / groups;
    int best = 256;
    double least = 0;
    for (int r = 256; r <= 16384; r += r / 1024 * 64 + 64) {
        const bool split = mean > r;
        const double blocks = groups * (split ? mean / r + 0.5 : 1);
        const double cost = std::ceil(blocks / at_once) * at_once * (split ? r : mean) * (K + 2 * N) * es +
                            (split ? blocks * K * N * 12 : 0);
        if (r == 256 || cost < least) best = r, least = cost;
        if (!split) break;
    }
    return best;
}

template <typename T> hipError_t launch(const RowOrder &o, const LayerGrad &q, float *slots, hipStream_t s)
{
    const int rows = chunk_rows(sizeof(T), o.n, o.G, q.K, q.N);
    const TileGrid grid = tile_grid(o.n / rows + o.G + 1);
    auto *kernel = q.act == CGTP_ACT_NONE ? (q.dw ? k_layer_grad<T, false, true> : k_layer_grad<T, false, false>)
                                          : (q.dw ? k_layer_grad<T, true, true> : k_layer_grad<T, true, false>);
    hipLaunchKernelGGL(kernel, dim3(grid.x, 1, grid.z), dim3(kThreads), 0, s, o, q, ChunkRows(rows), slots);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || o.n <= rows || (!q.dw && !q.dbias)) return e;
    return launch_row_join(sizeof(T) == 2 ? CGTP_BF16 : CGTP_F32, o, rows, q.dw ? q.K : 0, q.N, slots, q.dw, q.dbias, s);
}

}  // namespace

// Groups of fewer rows than a tile on the mean, or widths below a block, go the general way.
bool layer_grad_takes(int dtype, int64_t n, int G, int K, int N)
{
    return K >= kCW && K <= kWidth && N >= kCW && N <= kWidth && n >= (int64_t)kTileRows * G;
}

size_t layer_grad_slots(int dtype, int64_t n, int G, int K, int N)
{
    const int rows = chunk_rows(dtype == CGTP_BF16 ? 2 : 4, n, G, K, N);
    return n <= rows ? 0 : ((size_t)2 * (n / rows) + 2) * (K + 1) * N * sizeof(float);
}

hipError_t launch_layer_grad(int dtype, const RowOrder &o, const LayerGrad &q, void *slots, hipStream_t s)
{
    float *const f = static_cast<float *>(slots);
    return dtype == CGTP_BF16 ? launch<bf16_t>(o, q, f, s) : launch<float>(o, q, f, s);
}

}  // namespace cgtp
