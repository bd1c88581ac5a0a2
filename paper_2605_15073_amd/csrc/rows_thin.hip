// Products of grouped rows with long inputs and few tiles: a small batch through a wide layer.
//
// A tile of the general product takes its k in steps that wait for memory one after the other, 1.5 to 2 us each; where
// tiles are too few to fill the GPU, that is the call's time. Here a workgroup has 32 rows by 32 columns, and its waves
// share the k: wave w takes the steps w, w + 4, ... with the operands straight from memory, a step ahead, and the four
// sums are added in LDS. Us, in a graph, general product and this form, of a layer (silu) and of the row gradient whose
// product has the same K and N (n rows in G groups):
//
//     n, G          K, N         tiles     bf16                      fp32
//     64, 5         896, 16      7         16 8.0     9.9 5.3        45 13      34 10
//     64, 5         256, 64      14        7.8 4.9    5.1 3.6        16 6.2     11 5.4
//     64, 5         1344, 448    98        18 11      13 7.0         52 19      49 15
//     12000, 10     896, 16      385       17 11      12 9.1         46 22      35 17
//     3000, 20      896, 128     452       15 16      9.3 13         40 23      29 22
//     500, 100      448, 128     460       10 7.6     6.7 5.4        22 13      19 11
//     8000, 20      256, 64      540       8.3 6.8    5.5 5.9        17 11      11 11
//     1000, 10      1344, 448    574       20 23      12 21          58 38      41 38
//     4000, 200     300, 64      650       10 8.5     7.5 6.2        21 12      15 11
//     2000, 300     256, 64      724       9.0 7.2    6.2 5.1        19 9.8     13 9.0
//     6000, 20      896, 128     828       15 19      10 19          41 34      29 35
//     500, 200      448, 128     860       10 8.6     7.4 7.2        16 16      14 14
//     1500, 20      256, 448     924       8.9 10     6.1 6.8        19 15      13 13
//     1500, 300     256, 96      1038      8.6 9.1    6.7 6.0        18 12      15 11
//     16000, 20     256, 64      1040      9.1 11     6.2 8.3        19 18      13 16
//     1000, 500     256, 64      1062      11 9.2     6.8 6.3        9.7 9.9    8.1 8.3
//     3000, 20      1344, 448    1582      24 49      17 44          68 79      49 82
//
// Tiles are those that a call may have, (n / 32 + G) ceil(N / 32). Every one reads its operands from L2 anew, so that of
// groups that fill tiles the general product is ahead from 512 of them or 370,000 tiles times k on in bf16, from 1,024 in
// fp32, row gradients from 640. Groups of fewer rows than a tile leave the general product's larger ones emptier still: there
// bf16 rows of up to 64 columns are ahead to 1,100 tiles, of 32 at any number (4,000 rows of 4,000 groups, 256 -> 32, 36 and
// 22; but the row gradient of 10,007 of 4,005, 37 -> 129, from dz in parts takes 54 and 64).
//
// Sums are split over k: they are other fp32 sums than the general product's, so that only layers and their row
// gradients take this form.
#include "internal.h"
#include "rows_layer.h"

namespace cgtp {

namespace {

using namespace rows;

constexpr int kThin = 32;  // rows and columns of a tile
constexpr int kWaves = kThreads / 64;

// Eight k of column c of [K][N] weights, from k on; zero past their end.
template <typename T> __device__ __forceinline__ Raw8<T> load_column8(const T *w, int c, int k, int K, int N)
{
    Raw8<T> r;
    T v[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) v[u] = w[(int64_t)(k + u < K ? k + u : 0) * N + c];
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int u = 0; u < 8; ++u) r.v[u / 4][u % 4] = k + u < K ? __builtin_bit_cast(unsigned, v[u]) : 0u;
    } else {
#pragma unroll
        for (int u = 0; u < 8; u += 2) {
            const unsigned a = __builtin_bit_cast(unsigned short, v[u]), b = __builtin_bit_cast(unsigned short, v[u + 1]);
            r.v[0][u / 2] = (k + u < K ? a : 0u) | (k + u + 1 < K ? b : 0u) << 16;
        }
    }
    return r;
}

template <typename T, bool WNK, Extra EX>
__global__ __launch_bounds__(kThreads) void k_row_thin(RowOrder o, RowProduct p)
{
    constexpr int Q = kSplit<T>, S = kGroups<T> / 2, KS = kStep<T>, LD = kThin + 4;
    constexpr bool kDz = kForms<EX>;
    static_assert(!kDz || (sizeof(T) == 2 && WNK), "dz in parts: row gradients in bf16");
    __shared__ float4_t s_sum[kWaves][kThin][LD / 4];
    __shared__ int s_row[kThin];
    const Tile t = find_tile(o, TileRows<kThin>{}, tile_at(blockIdx.x, blockIdx.z, gridDim.x));
    if (t.g < 0 || t.p0 >= t.p1) return;
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, n32 = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int rows = (int)(t.p1 - t.p0), c0 = blockIdx.y * kThin, c1 = c0 + kThin < p.N ? c0 + kThin : p.N;
    if (tid < kThin) s_row[tid] = tid < rows ? row_at(o, t.p0 + tid) : -1;
    __syncthreads();
    if (t.g == o.G) {
        if (EX == kBare || EX == kGradZ) store_zeros<T>(p, s_row, rows, c0, c1);
        else store_bare<T>(p, s_row, rows, c0, c1);
        return;
    }
    const int own = s_row[n32], any = own < 0 ? 0 : own;  // row 0 in place of none: never stored
    const T *const in = static_cast<const T *>(p.in) + (EX == kLayer && p.per > 1 ? (int)((unsigned)any / (unsigned)p.per) : any) * p.in_stride;
    const T *const in_z = kDz ? static_cast<const T *>(p.slope_z) + any * p.slope_stride : nullptr;
    const T *const w = static_cast<const T *>(p.w) + (int64_t)t.g * p.w_group;
    const int col = c0 + n32 < p.N ? c0 + n32 : p.N - 1;  // the last one's in place of none
    struct Step { Raw8<T> x[S], z[kDz ? S : 1], w[S]; };
    auto load = [&](int s) {
        Step l;
#pragma unroll
        for (int i = 0; i < S; ++i) {
            const int k = s * KS + (2 * i + half) * kU;
            l.x[i] = load_row8<T, false>(in + k, p.K - k);
            if constexpr (kDz) l.z[i] = load_row8<T, false>(in_z + k, p.K - k);  // past the k that exist 0 act'(0)
            if constexpr (WNK) l.w[i] = load_row8<T, false>(w + (int64_t)col * p.K + k, p.K - k);
            else l.w[i] = load_column8(w, col, k, p.K, p.N);
        }
        return l;
    };
    const int steps = (p.K + KS - 1) / KS;
    float16_t acc;
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[i] = 0.f;
    if (wave < steps) {
        Step next = load(wave);
        float sign = 1.f;
        for (int s = wave; s < steps; s += kWaves) {
            const Step now = next;
            if (s + kWaves < steps) next = load(s + kWaves);
            if constexpr (Q > 1) {
                float16_t sum;
#pragma unroll
                for (int i = 0; i < 16; ++i) sum[i] = 0.f;
#pragma unroll
                for (int i = 0; i < S; ++i) {
                    uint4_t a[Q], b[Q];
                    to_units(now.w[i], a);
                    to_units(now.x[i], b, sign);
                    mma(sum, a, b);
                }
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[i] = fmaf(sign * kDown, sum[i], acc[i]);
                sign = -sign;
            } else if constexpr (kDz) {
#pragma unroll
                for (int i = 0; i < S; ++i) {
                    uint4_t part[2];
                    with_act(p.act, [&](auto act) __attribute__((always_inline)) {
                        dz_parts<decltype(act)::value>(now.x[i].v[0], now.z[i].v[0], part);
                    });
                    mfma(acc, now.w[i].v[0], part[1]);
                    mfma(acc, now.w[i].v[0], part[0]);
                }
            } else {
#pragma unroll
                for (int i = 0; i < S; ++i) mfma(acc, now.w[i].v[0], now.x[i].v[0]);
            }
        }
    }
#pragma unroll
    for (int v = 0; v < 4; ++v) s_sum[wave][n32][vec_col<T, false>(v, half) / 4] = vec_val<T, false>(acc, v);
    __syncthreads();
    const int r = tid / (kThin / 4), quad = tid % (kThin / 4), c = c0 + 4 * quad, row = s_row[r];
    float4_t x = s_sum[0][r][quad];
#pragma unroll
    for (int i = 1; i < kWaves; ++i) x += s_sum[i][r][quad];
    bool odd = false;
    if (row >= 0) {
#pragma unroll
        for (int e = 0; e < 4; ++e) odd |= c + e < p.N && !__builtin_isfinite(x[e]);
        if (EX == kLayer) store_layer<T, (Q > 1)>(p, t.g, true, row, c, x);
        else if (EX == kSums || EX == kSumsZ) store_four<false>(static_cast<float *>(p.out) + row * p.out_stride + c, x, p.N - c);
        else store_four<false>(static_cast<T *>(p.out) + row * p.out_stride + c, x, p.N - c);
    }
    if constexpr (kDz) {
        if (!__syncthreads_or(odd)) return;
        if constexpr (EX == kSumsZ) grad_plain_sums<float>(p, t.g, rows, s_row, c0, c1);
        else grad_plain_sums<T>(p, t.g, rows, s_row, c0, c1);
    }
    if constexpr (Q > 1) {
        if (!__syncthreads_or(odd)) return;
        if constexpr (EX == kLayer) layer_plain_sums<T, WNK>(p, t.g, rows, s_row, c0, c1);
        else row_plain_sums<T, WNK>(o, p, t.g, t.p0, rows, s_row, s_row, c0, c1);
    }
}

template <typename T, bool WNK, Extra EX> hipError_t launch(const RowOrder &o, const RowProduct &p, hipStream_t s)
{
    const TileGrid grid = tile_grid(o.n / kThin + o.G + 1);
    hipLaunchKernelGGL((k_row_thin<T, WNK, EX>), dim3(grid.x, (unsigned)((p.N + kThin - 1) / kThin), grid.z), dim3(kThreads), 0, s,
                       o, p);
    return hipGetLastError();
}

template <typename T> hipError_t pick(const RowOrder &o, const RowProduct &p, hipStream_t s)
{
    if (p.per > 0) return launch<T, false, kLayer>(o, p, s);
    if constexpr (sizeof(T) == 2) {
        if (p.slope_z) return p.out_f32 ? launch<T, true, kSumsZ>(o, p, s) : launch<T, true, kGradZ>(o, p, s);
        if (p.out_f32) return launch<T, true, kSums>(o, p, s);
    }
    return launch<T, true, kBare>(o, p, s);
}

}  // namespace

bool row_thin_takes(int dtype, const RowOrder &o, const RowProduct &p)
{
    const int es = dtype == CGTP_BF16 ? 2 : 4;
    if (!(p.per > 0 || p.split_k) || p.h || p.a || p.narrow || p.K <= 128 * 2 / es) return false;
    const int64_t tiles = (o.n / kThin + o.G) * ((p.N + kThin - 1) / kThin);
    const bool part_tiles = o.n < (int64_t)kThin * o.G;
    if (es == 4) return tiles <= (part_tiles || !p.w_nk ? 1024 : 640);
    if (part_tiles) return tiles <= (p.N <= kThin ? INT64_MAX : p.N <= 2 * kThin ? 1100 : 512);
    return tiles <= 512 && tiles * p.K <= 370000;
}

hipError_t launch_row_thin(int dtype, const RowOrder &o, const RowProduct &p, hipStream_t s)
{
    return dtype == CGTP_BF16 ? pick<bf16_t>(o, p, s) : pick<float>(o, p, s);
}

}  // namespace cgtp
