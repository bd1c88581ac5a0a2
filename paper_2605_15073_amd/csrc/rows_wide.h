// Products of grouped rows with short inputs and wide outputs: a radial network's last layer.
//
// Such a product writes far more than it reads, so what counts is that stores leave in whole lines and
// that many waves have some under way. A wave keeps its 32 input rows in registers, one matrix operand
// per lane as the instruction wants it, straight from memory, and runs over tiles of kCols output columns;
// only the weights of a tile pass through LDS, loaded a tile ahead. The results are turned in a piece of LDS
// that the wave has for itself, and leave as rows of kCols values, four rows a store.
//
// Nothing in the loop over column tiles branches: the wait for the next tile's weights can then leave this
// tile's stores in flight, and the sums stay where they are (a branch around a matrix instruction costs a
// copy of its 32 registers). So the number of k is a template argument, rounded up with zeros; places
// without a row of their own take another place's of the tile (and store the same values to the same
// place), and the last column tile starts early enough to end with the rows.
//
// Stores. LINES: every row starts on half a line, so pieces of 128 bytes go out as they are, past the caches.
// Else a row's results are turned into a ring of two pieces, each value where its address lies in a line, and
// leave line by line: a line is stored once the columns that it takes are there, the ends of a row in vectors that
// overlap. WHOLE: columns come in aligned fours.
// 525,308 rows from 64, us now, and with pieces stored where their columns start, through and past the caches:
// bf16 452 191, 252, 473; 480 146, 201, 148; 900 341, 485, 896; fp32 452 368, 433, 812; 900 644, 815, 1,540; 912
// 544, 659, 544. Rows on lines, past and through the caches: bf16 896 200, 243, fp32 440, 505; with a reader right
// behind, results of 4 to 900 MB, between 9% more (4 MB) and 13% less.
//
// Measured: 525,308 rows, 64 -> 896: 447 to 477 us in fp32 (4.2 to 4.5 TB/s) and 198 us in bf16 (5.1 TB/s), 93% of
// it stores; bound by memory, a large copy reaches 4.8 TB/s. Rows apart from lines: 2.3 to 3.4 TB/s, bound by the
// two broken lines of each row, whose other parts other workgroups write.
//
// Adapters: the narrow product's rows are further k of the same tile, held in registers like the
// inputs, with the adapter's second matrix behind the shared weights in LDS; a tile whose rows have several
// adapters takes them one after the other, with the rows of the others zero. Where adapters have rows enough
// for tiles of their own (FUSED) the narrow product is formed here too: from the inputs in registers and the
// adapter's first matrix through LDS, turned in the wave's piece, and held from then on: 525,308 rows of 32
// adapters, 64 -> 896, bf16, rank 16 212 us (4.8 TB/s), rank 32 250: three and six pairs of k-groups for its parts
// beside the inputs' four; fp32, rank 16, 606.
//
// Layers (EX kLayer): the bias comes with the weights; sums become z, are turned and stored as they are (Z), activated in
// place, and go the way of the results with the residual added (RES), which is read where the sums lie.
#ifndef CGTP_ROWS_WIDE_H
#define CGTP_ROWS_WIDE_H

#include "internal.h"
#include "rows_layer.h"

namespace cgtp {
namespace rows {

constexpr int kRows = 128;    // positions of a workgroup, 32 a wave
constexpr int kCols = kWideCols;  // columns of a tile
template <typename T> constexpr int kPairs = sizeof(T) == 2 ? 8 : 4;  // pairs of k-groups: up to 128 bf16, 64 fp32
template <typename T> constexpr int kExtPairs = sizeof(T) == 2 ? 6 : 2;  // of a narrow product's rows, up to 32 wide

// The results are turned 64 (bf16) or 32 (fp32) columns at a time, 128 bytes a row. Row stride of the turned
// results, in values: a multiple of their vectors, clear of bank conflicts between the rows that the 8
// (fp32, 16 bytes) or 16 (bf16, 8 bytes) lanes of a cycle write. XP: of a narrow product that is turned here too.
template <typename T> constexpr int kPiece = 128 / (int)sizeof(T);
template <typename T, bool LINES, int XP>
constexpr int kTurn = ((LINES ? 1 : 2) * kPiece<T> > 2 * XP * kU ? (LINES ? 1 : 2) * kPiece<T> : 2 * XP * kU) + 4;

template <typename T> struct Out4;
template <> struct Out4<float> { typedef float4_t t; typedef float4_any any; };
template <> struct Out4<bf16_t> { typedef bf4_t t; typedef bf4_any any; };

__device__ __forceinline__ void convert(float4_t v, float4_t &o) { o = v; }
__device__ __forceinline__ void convert(float4_t v, bf4_t &o)
{
    o = bf4_t{(bf16_t)v[0], (bf16_t)v[1], (bf16_t)v[2], (bf16_t)v[3]};
}

// NP, XP: pairs of k-groups of the inputs and of the narrow product's rows (0: no adapters). All parts of those
// rows, XP / P pairs each, meet the same weights, which lie in LDS once.
template <typename T, bool WNK, int NP, int XP, bool FUSED, bool WHOLE, bool LINES, Extra EX, bool Z, bool RES>
__global__ __launch_bounds__(kThreads) void k_row_wide(RowOrder o, RowProduct p, int splits)
{
    constexpr int U = kU, P = kNarrow<T>, Q = kSplit<T>, XE = XP > 0 ? XP / P : 1, KG = 2 * (NP + XP / P), LD = kCols + 1, CW = kWide<T>;
    constexpr bool EXT = XP > 0;
    // fp32: the matrix instruction rounds down, so the second half of the k is summed negated (step_products)
    constexpr int kPlus = Q > 1 && NP > 1 ? NP / 2 : NP;
    constexpr float kSign = kPlus < NP ? -1.f : 1.f;  // of the adapters' products and of the result
    constexpr float kOut = Q > 1 ? kSign * kDown : kSign;
    static_assert(NP <= kPairs<T> && !(EXT && WNK), "adapters: [K][N] weights");
    constexpr bool kDz = kForms<EX>;
    constexpr int kParts = kDz ? 2 : Q;  // operands of a row's k
    static_assert(EX == kBare || (EX == kLayer && !EXT && !WNK) || (EX == kGradZ && !EXT && WNK && sizeof(T) == 2),
                  "layers: [K][N] weights, no adapters; their row gradients from dz in parts: bf16");
    typedef typename Out4<T>::t O;
    typedef typename Out4<T>::any O_any;
    __shared__ uint4_t s_w[Q * KG * LD];
    constexpr int TURN = kTurn<T, LINES, FUSED ? XP : 0>, RING = 2 * kPiece<T>;
    __shared__ O s_turn[4 * 32 * TURN / 4];
    constexpr int ZTURN = LINES ? kCols + 4 : TURN;  // z of all columns at once, or a ring like that of the results
    __shared__ O s_z_turn[Z ? 4 * 32 * ZTURN / 4 : 1];
    __shared__ float4_t s_bias[EX == kLayer ? kCols / 4 : 1];
    __shared__ int s_row[kRows], s_place[kRows], s_any;
    __shared__ int s_g[EXT ? kRows : 1], s_seg_g[EXT ? kRows : 1], s_seg_at[EXT ? kRows + 1 : 1], s_nseg;

    int64_t index = tile_at(blockIdx.x, blockIdx.z, gridDim.x);
    if (EX != kBare) {
        if (p.xcd_tiles > 0) index = xcd_tile(index, p.xcd_tiles);
        if (index < 0) return;
    }
    Tile t;
    if (EXT && !FUSED) {
        t.p0 = index * kRows;
        if (t.p0 >= o.n) return;
        t.p1 = t.p0 + kRows < o.n ? t.p0 + kRows : o.n;
        t.g = 0;
    } else {
        t = find_tile(o, TileRows<kRows>{}, index);
        if (t.g < 0 || t.p0 >= t.p1) return;
    }
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int rows = (int)(t.p1 - t.p0);
    const int ctiles = (p.N + kCols - 1) / kCols;
    // this workgroup's column tiles: the last two, which overlap, go together
    const int whole = p.N / kCols;
    const int ct0 = (int)((int64_t)whole * blockIdx.y / splits);
    const int ct1 = blockIdx.y + 1 == gridDim.y ? ctiles : (int)((int64_t)whole * (blockIdx.y + 1) / splits);
    if (ct0 >= ct1) return;
    const int my_row = tid < rows ? row_at(o, t.p0 + tid) : -1;
    if (tid < kRows) s_row[tid] = my_row;
    if (tid == 0) s_any = -1;
    __syncthreads();
    if (my_row >= 0) s_any = tid;  // any place that has a row
    if (EX == kLayer && t.g == o.G) {
        store_bare<T>(p, s_row, rows, ct0 * kCols, ct1 * kCols < p.N ? ct1 * kCols : p.N);
        return;
    }
    if (!EXT && t.g == o.G) {
        store_zeros<T>(p, s_row, rows, ct0 * kCols, ct1 * kCols < p.N ? ct1 * kCols : p.N);
        return;
    }
    int nseg = 0;
    if (FUSED) {
        nseg = t.g < o.G;
        if (tid == 0) {
            s_seg_g[0] = nseg ? t.g : 0;
            s_seg_at[0] = 0;
            s_seg_at[1] = kRows;
        }
        __syncthreads();
    } else if (EXT) nseg = find_segments<kRows>(o, t.p0, rows, s_g, s_seg_g, s_seg_at, &s_nseg);
    else __syncthreads();
    if (s_any < 0) return;
    if (tid < kRows) s_place[tid] = my_row >= 0 ? tid : s_any;
    __syncthreads();

    // inputs: row 32 wave + lane % 32, k-groups 2 s + half
    const int pl = s_place[32 * wave + (lane & 31)];
    const T *const in = static_cast<const T *>(p.in) +
                        (EX == kLayer && p.per > 1 ? (int)((unsigned)s_row[pl] / (unsigned)p.per) : s_row[pl]) * p.in_stride;
    const int W = EXT ? narrow_width(p.r) : 0;
    uint4_t x[NP][kParts], h[EXT ? XP : 1][Q];
    float odd = 0.f;  // NaN once a result is not finite
    if constexpr (kDz) {
        const T *const in_z = static_cast<const T *>(p.slope_z) + s_row[pl] * p.slope_stride;
        Raw8<T> dy[NP], z[NP];
#pragma unroll
        for (int s = 0; s < NP; ++s) {
            const int k = (2 * s + half) * U;
            dy[s] = load_row8<T, false>(in + k, p.K - k);
            z[s] = load_row8<T, false>(in_z + k, p.K - k);  // past the k that exist 0 act'(0)
        }
#pragma unroll
        for (int s = 0; s < NP; ++s)
            with_act(p.act, [&](auto act) __attribute__((always_inline)) {
                dz_parts<decltype(act)::value>(dy[s].v[0], z[s].v[0], x[s]);
            });
    } else {
#pragma unroll
        for (int s = 0; s < NP; ++s) {
            const int k = (2 * s + half) * U;
            to_units(load_row8<T, false>(in + k, p.K - k), x[s], s < kPlus ? 1.f : -1.f);
        }
    }
    O *const turn = s_turn + wave * (32 * TURN / 4), *const z_turn = s_z_turn + (Z ? wave * (32 * ZTURN / 4) : 0);
    if constexpr (FUSED) {
        // the adapter's first matrix, [K][r], as a tile of 32 columns
        constexpr int kQuads = 32 / CW;
        for (int task = tid; task < kQuads * 2 * NP; task += kThreads) {
            const int g = task / kQuads, c = CW * (task % kQuads);
            const T *const q = static_cast<const T *>(p.a) + ((int64_t)(nseg ? t.g : 0) * p.K + g * U) * p.r + c;
            uint2_t in[8];
#pragma unroll
            for (int u = 0; u < U; ++u)
                in[u] = load_8<T, false>(q + (int64_t)u * p.r, nseg && g * U + u < p.K ? p.r - c : 0);
            uint4_t unit[CW][Q];
            to_units(in, unit);
#pragma unroll
            for (int j = 0; j < CW; ++j) put<T, kCols>(s_w, KG, g, place<T>(c + j), unit[j]);
        }
        __syncthreads();
        float16_t sum;
#pragma unroll
        for (int i = 0; i < 16; ++i) sum[i] = 0.f;
#pragma unroll
        for (int s = 0; s < NP; ++s) {
            uint4_t c[Q];
#pragma unroll
            for (int q = 0; q < Q; ++q) c[q] = s_w[(q * KG + 2 * s + half) * LD + (lane & 31)];
            if (s == kPlus)
#pragma unroll
                for (int i = 0; i < 16; ++i) sum[i] = -sum[i];
            mma(sum, c, x[s]);
        }
        const float scale = p.narrow_scale && nseg ? p.narrow_scale[t.g] : 1.f;
        T *const mine = reinterpret_cast<T *>(turn) + (lane & 31) * TURN;
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const int col = vec_col<T, true>(v, half);
            float4_t f = vec_val<T, true>(sum, v);
#pragma unroll
            for (int e = 0; e < 4; ++e) f[e] = col + e < p.r ? f[e] * kOut * scale : 0.f;  // an infinite input times nothing is NaN
            if (col < W) store_narrow(mine + col, W, f);
        }
        wave_sync();
#pragma unroll
        for (int s = 0; s < XP; ++s) {
            const int k = (2 * (s % XE) + half) * U;
            to_units(load_row8<T, false>(mine + s / XE * W + k, W - k), h[s], kSign);
        }
        wave_sync();
    } else if (EXT) {
        const bool grouped = s_g[pl] < o.G;
#pragma unroll
        for (int s = 0; s < XP; ++s) {
            const int k = (2 * (s % XE) + half) * U;
            const T *const q = static_cast<const T *>(p.h) + (grouped ? (t.p0 + pl) * (P * W) + s / XE * W : 0) + k;
            to_units(load_row8<T, true>(q, grouped ? W - k : 0), h[s], kSign);
        }
    }
    // outputs: of a piece of 128 bytes this lane stores vector lane % kVecs of rows 64 / kVecs i + lane / kVecs
    constexpr int kVecs = kPiece<T> / 4, kStores = 32 * kVecs / 64;
    T *out[kStores], *z_out[Z ? kStores : 1];
#pragma unroll
    for (int i = 0; i < kStores; ++i) {
        const int64_t row = s_row[s_place[32 * wave + (64 / kVecs) * i + lane / kVecs]];
        out[i] = static_cast<T *>(p.out) + row * p.out_stride;
        if (Z) z_out[i] = static_cast<T *>(p.z) + row * p.z_stride;
    }
    const T *const res = RES ? static_cast<const T *>(p.residual) + s_row[pl] * p.residual_stride : nullptr;

    // what this lane's row of results is off the start of a line by, in values
    const int my_at = (int)(reinterpret_cast<uintptr_t>(static_cast<T *>(p.out) + s_row[pl] * p.out_stride) % 128 / sizeof(T));

    // Weights. Round 0 of a column tile: the shared ones, with the first adapter's behind them; then the
    // other adapters' of the tile.
    constexpr int kTasks = (WNK ? kCols : kCols / CW) * KG;  // units, or units of CW columns
    constexpr int NT = wide_rounds(kTasks);
    static_assert(kThreads == kWideThreads, "units of the threads");
    const T *const w = static_cast<const T *>(p.w) + (FUSED ? 0 : (int64_t)t.g * p.w_group);
    Raw8<T> wn[WNK ? NT : 1];
    uint2_t wt[WNK ? 1 : NT][8];
    int early[WNK ? NT : 1];  // what the loads started early
    int have[NT];  // k of the k-groups in flight that the weights have
    auto first_col = [&](int ct) { return wide_first_col(ct, p.N); };
    T bias;  // of column tid % kCols of the tile whose weights are in flight
    const T *const bias_at = EX == kLayer && p.bias ? static_cast<const T *>(p.bias) + (int64_t)t.g * p.N : w;
    auto fetch = [&](int ct, int seg) {
        const int c0 = first_col(ct);
        if (EX == kLayer) bias = bias_at[c0 + tid % kCols];
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            const int task = wide_unit(tid, i, kTasks);
            const int g = WNK ? task % KG : task / (kCols / CW);
            int k = g * U, K = p.K;
            const T *wb = w;
            if (EXT && g >= 2 * NP) {
                k = (g - 2 * NP) * U;
                K = nseg > 0 ? p.r : 0;
                wb = static_cast<const T *>(p.v) + (int64_t)(nseg > 0 ? s_seg_g[seg] : 0) * p.r * p.N;
            }
            have[i] = K - k;
            if (have[i] <= 0) k = 0;
            if constexpr (WNK) {
                const T *const q = wb + (int64_t)(c0 + task / KG) * p.K;
                const int at = start8(k, p.K);
                early[i] = k - at;
                wn[i] = load_any8(q + at);
            } else {
                const int c = c0 + CW * (task % (kCols / CW));
#pragma unroll
                for (int u = 0; u < U; ++u)
                    wt[i][u] = *reinterpret_cast<const uint2_any *>(wb + (int64_t)(u < have[i] ? k + u : 0) * p.N + c);
            }
        }
    };
    auto stage = [&]() {
        if (EX == kLayer && tid < kCols) reinterpret_cast<float *>(s_bias)[tid] = p.bias ? (float)bias : 0.f;
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            const int task = tid + kThreads * i;
            if (kTasks % kThreads != 0 && task >= kTasks) continue;
            if constexpr (WNK) {
                uint4_t unit[Q];
                Raw8<T> raw = wn[i];
                if (have[i] < kU) settle(raw, early[i], have[i]);
                to_units(raw, unit);
                put<T, kCols>(s_w, KG, task % KG, task / KG, unit);
            } else {
                uint2_t in[8];
#pragma unroll
                for (int u = 0; u < U; ++u) in[u] = u < have[i] ? wt[i][u] : uint2_t{0, 0};
                uint4_t unit[CW][Q];
                to_units(in, unit);
#pragma unroll
                for (int j = 0; j < CW; ++j)
                    put<T, kCols>(s_w, KG, task / (kCols / CW), place<T>(CW * (task % (kCols / CW)) + j), unit[j]);
            }
        }
    };

    const uint4_t *const a = s_w + half * LD + (lane & 31);
    fetch(ct0, 0);
    for (int ct = ct0; ct < ct1; ++ct) {
        float16_t acc[2];
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[c][i] = 0.f;
        __syncthreads();
        stage();
        __syncthreads();
        if (EX == kLayer && Q == 1)  // bf16 sums start at the bias; fp32's, of scaled parts, get it behind
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int v = 0; v < 4; ++v) set_vec<T, !WNK>(acc[c], v, s_bias[(32 * c + vec_col<T, !WNK>(v, half)) / 4]);
        fetch(nseg > 1 || ct + 1 == ct1 ? ct : ct + 1, nseg > 1 ? 1 : 0);
        auto product = [&](int pair, const uint4_t (&b)[kParts]) {
            uint4_t c0[Q], c1[Q];
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                c0[q] = a[(q * KG + 2 * pair) * LD];
                c1[q] = a[(q * KG + 2 * pair) * LD + 32];
            }
            if constexpr (kDz) {
#pragma unroll
                for (int e = kParts - 1; e >= 0; --e) {
                    mfma(acc[0], c0[0], b[e]);
                    mfma(acc[1], c1[0], b[e]);
                }
            } else {
                mma(acc[0], c0, b);
                mma(acc[1], c1, b);
            }
        };
#pragma unroll
        for (int s = 0; s < NP; ++s) {
            if (s == kPlus)
#pragma unroll
                for (int c = 0; c < 2; ++c)
#pragma unroll
                    for (int i = 0; i < 16; ++i) acc[c][i] = -acc[c][i];
            product(s, x[s]);
        }
        if (EXT) {
            for (int seg = 0;;) {
                const bool in_seg = nseg > 0 && pl >= s_seg_at[seg] && pl < s_seg_at[seg + 1];
#pragma unroll
                for (int s = 0; s < XP; ++s) {
                    uint4_t b[kParts];
#pragma unroll
                    for (int q = 0; q < Q; ++q)
#pragma unroll
                        for (int e = 0; e < 4; ++e) b[q][e] = in_seg ? h[s][q][e] : 0u;
                    product(NP + s % XE, b);
                }
                if (++seg >= nseg) break;
                __syncthreads();
                stage();
                __syncthreads();
                if (seg + 1 < nseg) fetch(ct, seg + 1);
                else fetch(ct + 1 < ct1 ? ct + 1 : ct, 0);
            }
        }
        if (kDz || (EX == kBare && (Q > 1 || EXT)))
#pragma unroll
            for (int c = 0; c < 2; ++c) probe(odd, acc[c]);
        if constexpr (EX == kLayer) {
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    float4_t f = vec_val<T, !WNK>(acc[c], v);
                    if (Q > 1) {
                        f = kOut * f + s_bias[(32 * c + vec_col<T, !WNK>(v, half)) / 4];
                        set_vec<T, !WNK>(acc[c], v, f);
                    }
                    if (Z && LINES) convert(f, z_turn[((lane & 31) * ZTURN + 32 * c + vec_col<T, !WNK>(v, half)) / 4]);
                }
            // fp32: NaN where z, an infinite bias with it, is not finite, for layer_plain_sums to find
            if (Q > 1)
#pragma unroll
                for (int c = 0; c < 2; ++c) probe(odd, acc[c]);
            if (!Z || LINES)
#pragma unroll
                for (int c = 0; c < 2; ++c) activate_all<T, (Q > 1)>(acc[c], p.act);
        }
        constexpr float kLast = EX == kLayer ? 1.f : kOut;
        // rows of 128 bytes, several a store
#pragma unroll
        for (int piece = 0; piece < kCols; piece += kPiece<T>) {
            const int first = first_col(ct) + piece, end = first + kPiece<T>;
            if constexpr (Z && !LINES) {  // z of the piece to its ring, whose lines are where the results' are
#pragma unroll
                for (int c = 0; c < kPiece<T> / 32; ++c) {
#pragma unroll
                    for (int v = 0; v < 4; ++v) {
                        const float4_t f = vec_val<T, !WNK>(acc[piece / 32 + c], v);
                        const int at = my_at + first + 32 * c + vec_col<T, !WNK>(v, half);
                        if (WHOLE) convert(f, z_turn[((lane & 31) * TURN + at % RING) / 4]);
                        else {
#pragma unroll
                            for (int e = 0; e < 4; ++e) reinterpret_cast<T *>(z_turn)[(lane & 31) * TURN + (at + e) % RING] = (T)f[e];
                        }
                    }
                    activate_all<T, (Q > 1)>(acc[piece / 32 + c], p.act);
                }
            }
#pragma unroll
            for (int c = 0; c < kPiece<T> / 32; ++c)
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    float4_t f = kLast * vec_val<T, !WNK>(acc[piece / 32 + c], v);
                    const int col = 32 * c + vec_col<T, !WNK>(v, half);
                    if (RES) f += load_four(res + first + col, 4);
                    if (LINES) convert(f, turn[((lane & 31) * TURN + col) / 4]);
                    else if (WHOLE) convert(f, turn[((lane & 31) * TURN + (my_at + first + col) % RING) / 4]);
                    else {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            reinterpret_cast<T *>(turn)[(lane & 31) * TURN + (my_at + first + col + e) % RING] = (T)f[e];
                    }
                }
            wave_sync();
            const int in_piece = 4 * (lane % kVecs);
            if (LINES) {
#pragma unroll
                for (int i = 0; i < kStores; ++i) {
                    const T *const from = reinterpret_cast<const T *>(turn) +
                                          ((64 / kVecs) * i + lane / kVecs) * TURN + in_piece;
                    __builtin_nontemporal_store(*reinterpret_cast<const O *>(from), reinterpret_cast<O *>(out[i] + first + in_piece));
                    if (Z) {
                        const T *const z_from = reinterpret_cast<const T *>(z_turn) +
                                                ((64 / kVecs) * i + lane / kVecs) * ZTURN + piece + in_piece;
                        __builtin_nontemporal_store(*reinterpret_cast<const O *>(z_from), reinterpret_cast<O *>(z_out[i] + first + in_piece));
                    }
                }
            } else {
                const int from_col = ct0 * kCols > end - RING ? ct0 * kCols : end - RING;
                // line `line` of each row, as far as its columns are there: places past them take the last or the first
                auto store_line = [&](int line) {
#pragma unroll
                    for (int i = 0; i < kStores; ++i) {
                        const int at = (int)(reinterpret_cast<uintptr_t>(out[i]) % 128 / sizeof(T));
                        int c = line * kPiece<T> - at + in_piece;
                        c = c < from_col ? from_col : c > end - 4 ? end - 4 : c;
                        auto store = [&](const O *ring, T *to) {
                            const T *const from = reinterpret_cast<const T *>(ring) + ((64 / kVecs) * i + lane / kVecs) * TURN;
                            O v;
                            if (WHOLE) v = *reinterpret_cast<const O *>(from + (at + c) % RING);
                            else {
#pragma unroll
                                for (int e = 0; e < 4; ++e) v[e] = from[(at + c + e) % RING];
                            }
                            *reinterpret_cast<O_any *>(to + c) = v;
                        };
                        store(turn, out[i]);
                        if constexpr (Z) store(z_turn, z_out[i]);
                    }
                };
                // a line more for each piece; at the end all that is left
                const bool early_tile = first_col(ct) < ct * kCols;
                int line = ct * kCols / kPiece<T> + (early_tile ? 0 : piece / kPiece<T>);
                if (ct + 1 < ct1 || piece + kPiece<T> < kCols) {
                    store_line(line);
                } else {
                    for (; (line - 1) * kPiece<T> + 1 < end; ++line) store_line(line);
                }
            }
            wave_sync();
        }
    }
    if constexpr (kDz) {
        if (__syncthreads_or(odd != odd)) grad_plain_sums<T>(p, t.g, rows, s_row, ct0 * kCols, ct1 * kCols < p.N ? ct1 * kCols : p.N);
    }
    if constexpr (Q > 1 || EXT) {
        const int end = ct1 * kCols < p.N ? ct1 * kCols : p.N;
        if constexpr (EX == kLayer) {
            if (__syncthreads_or(odd != odd)) layer_plain_sums<T, WNK>(p, t.g, rows, s_row, ct0 * kCols, end);
        } else if (__syncthreads_or(odd != odd)) {
            float *const plain_h = FUSED ? reinterpret_cast<float *>(s_turn) : nullptr;
            if constexpr (FUSED) {
                static_assert(sizeof(s_turn) >= sizeof(float) * kRows * 32, "rows of up to 32 values");
                for (int e = tid; e < rows * p.r; e += kThreads) {
                    const int r = e / p.r, c = e % p.r;
                    const T *const ac = static_cast<const T *>(p.a) + (int64_t)(nseg ? t.g : 0) * p.K * p.r + c;
                    float sum = 0.f;
                    if (nseg && s_row[r] >= 0)
                        for (int k = 0; k < p.K; ++k)
                            sum += (float)static_cast<const T *>(p.in)[s_row[r] * p.in_stride + k] * (float)ac[(int64_t)k * p.r];
                    plain_h[32 * r + c] = p.narrow_scale && nseg ? sum * p.narrow_scale[t.g] : sum;
                }
                if (tid < rows) s_g[tid] = t.g;
            }
            row_plain_sums<T, WNK>(o, p, p.w_group ? t.g : 0, t.p0, rows, s_row, s_g, ct0 * kCols, end, plain_h);
        }
    }
}

// Rows of an output: all on half a line, or in aligned fours.
template <typename T> bool by_lines(const void *out, int64_t stride, int N)
{
    constexpr int half = kPiece<T> / 2;
    return N % half == 0 && stride % half == 0 && reinterpret_cast<uintptr_t>(out) % 64 == 0;
}
template <typename T> bool by_fours(const void *out, int64_t stride, int N)
{
    return N % 4 == 0 && stride % 4 == 0 && reinterpret_cast<uintptr_t>(out) % (4 * sizeof(T)) == 0;
}

// Workgroups: tiles of rows, and column tiles shared among some where rows are few.
struct WideGrid {
    dim3 grid;
    int splits;
};
inline WideGrid wide_grid(int64_t tiles, int N)
{
    const int whole = N / kCols;
    // few rows: column tiles go to workgroups of their own (60,000 rows, 64 -> 1344, with 512, 2,048 and 8,192
    // workgroups bf16 37, 39 and 54 us, fp32 95, 94 and 124; 20,000 rows, 64 -> 896 bf16 12, 16 and 16)
    int splits = (int)(2048 / tiles);
    splits = splits < 1 ? 1 : splits > whole ? whole : splits;
    const TileGrid grid = tile_grid(tiles);
    return {dim3(grid.x, (unsigned)splits, grid.z), splits};
}

}  // namespace rows
}  // namespace cgtp

#endif
