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
#include "internal.h"
#include "rows_tile.h"

namespace cgtp {

namespace {

using namespace rows;

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

// Orders a wave's LDS writes before its other lanes' reads.
__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// NP, XP: pairs of k-groups of the inputs and of the narrow product's rows (0: no adapters). All parts of those
// rows, XP / P pairs each, meet the same weights, which lie in LDS once.
template <typename T, bool WNK, int NP, int XP, bool FUSED, bool WHOLE, bool LINES>
__global__ __launch_bounds__(kThreads) void k_row_wide(RowOrder o, RowProduct p, int splits)
{
    constexpr int U = kU, P = kNarrow<T>, Q = kSplit<T>, XE = XP > 0 ? XP / P : 1, KG = 2 * (NP + XP / P), LD = kCols + 1, CW = kWide<T>;
    constexpr bool EXT = XP > 0;
    // fp32: the matrix instruction rounds down, so the second half of the k is summed negated (step_products)
    constexpr int kPlus = Q > 1 && NP > 1 ? NP / 2 : NP;
    constexpr float kSign = kPlus < NP ? -1.f : 1.f;  // of the adapters' products and of the result
    constexpr float kOut = Q > 1 ? kSign * kDown : kSign;
    static_assert(NP <= kPairs<T> && !(EXT && WNK), "adapters: [K][N] weights");
    typedef typename Out4<T>::t O;
    typedef typename Out4<T>::any O_any;
    __shared__ uint4_t s_w[Q * KG * LD];
    constexpr int TURN = kTurn<T, LINES, FUSED ? XP : 0>, RING = 2 * kPiece<T>;
    __shared__ O s_turn[4 * 32 * TURN / 4];
    __shared__ int s_row[kRows], s_place[kRows], s_any;
    __shared__ int s_g[EXT ? kRows : 1], s_seg_g[EXT ? kRows : 1], s_seg_at[EXT ? kRows + 1 : 1], s_nseg;

    const int64_t index = tile_at(blockIdx.x, blockIdx.z, gridDim.x);
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
    const T *const in = static_cast<const T *>(p.in) + s_row[pl] * p.in_stride;
    const int W = EXT ? narrow_width(p.r) : 0;
    uint4_t x[NP][Q], h[EXT ? XP : 1][Q];
    float odd = 0.f;  // NaN once a result is not finite
#pragma unroll
    for (int s = 0; s < NP; ++s) {
        const int k = (2 * s + half) * U;
        to_units(load_row8<T, false>(in + k, p.K - k), x[s], s < kPlus ? 1.f : -1.f);
    }
    O *const turn = s_turn + wave * (32 * TURN / 4);
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
    T *out[kStores];
#pragma unroll
    for (int i = 0; i < kStores; ++i)
        out[i] = static_cast<T *>(p.out) + s_row[s_place[32 * wave + (64 / kVecs) * i + lane / kVecs]] * p.out_stride;

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
    auto fetch = [&](int ct, int seg) {
        const int c0 = first_col(ct);
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
        fetch(nseg > 1 || ct + 1 == ct1 ? ct : ct + 1, nseg > 1 ? 1 : 0);
        auto product = [&](int pair, const uint4_t (&b)[Q]) {
            uint4_t c0[Q], c1[Q];
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                c0[q] = a[(q * KG + 2 * pair) * LD];
                c1[q] = a[(q * KG + 2 * pair) * LD + 32];
            }
            mma(acc[0], c0, b);
            mma(acc[1], c1, b);
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
                    uint4_t b[Q];
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
        if (Q > 1 || EXT)
#pragma unroll
            for (int c = 0; c < 2; ++c) probe(odd, acc[c]);
        // rows of 128 bytes, several a store
#pragma unroll
        for (int piece = 0; piece < kCols; piece += kPiece<T>) {
            const int first = first_col(ct) + piece, end = first + kPiece<T>;
#pragma unroll
            for (int c = 0; c < kPiece<T> / 32; ++c)
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    const float4_t f = kOut * vec_val<T, !WNK>(acc[piece / 32 + c], v);
                    const int col = 32 * c + vec_col<T, !WNK>(v, half);
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
                        const T *const from = reinterpret_cast<const T *>(turn) + ((64 / kVecs) * i + lane / kVecs) * TURN;
                        O v;
                        if (WHOLE) v = *reinterpret_cast<const O *>(from + (at + c) % RING);
                        else {
#pragma unroll
                            for (int e = 0; e < 4; ++e) v[e] = from[(at + c + e) % RING];
                        }
                        *reinterpret_cast<O_any *>(out[i] + c) = v;
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
    if constexpr (Q > 1 || EXT) {
        const int end = ct1 * kCols < p.N ? ct1 * kCols : p.N;
        if (__syncthreads_or(odd != odd)) {
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

template <typename T, bool WNK, int NP, int XP, bool FUSED, bool WHOLE, bool LINES>
hipError_t launch(const RowOrder &o, const RowProduct &p, hipStream_t s)
{
    const int64_t tiles = XP > 0 && !FUSED ? (o.n + kRows - 1) / kRows : o.n / kRows + o.G + 1;
    const int whole = p.N / kCols;
    // few rows: column tiles go to workgroups of their own (60,000 rows, 64 -> 1344, with 512, 2,048 and 8,192
    // workgroups bf16 37, 39 and 54 us, fp32 95, 94 and 124; 20,000 rows, 64 -> 896 bf16 12, 16 and 16)
    int splits = (int)(2048 / tiles);
    splits = splits < 1 ? 1 : splits > whole ? whole : splits;
    const TileGrid grid = tile_grid(tiles);
    hipLaunchKernelGGL((k_row_wide<T, WNK, NP, XP, FUSED, WHOLE, LINES>), dim3(grid.x, (unsigned)splits, grid.z), dim3(kThreads),
                       0, s, o, p, splits);
    return hipGetLastError();
}

template <typename T, int NP, bool WHOLE, bool LINES>
hipError_t with_pairs(const RowOrder &o, const RowProduct &p, hipStream_t s)
{
    if (!p.h && !p.a)
        return p.w_nk ? launch<T, true, NP, 0, false, WHOLE, LINES>(o, p, s)
                      : launch<T, false, NP, 0, false, WHOLE, LINES>(o, p, s);
    constexpr int X = kExtPairs<T>;
    const bool half = kNarrow<T> * narrow_width(p.r) <= X * kU;
    if (p.a)
        return half ? launch<T, false, NP, X / 2, true, WHOLE, LINES>(o, p, s)
                    : launch<T, false, NP, X, true, WHOLE, LINES>(o, p, s);
    return half ? launch<T, false, NP, X / 2, false, WHOLE, LINES>(o, p, s)
                : launch<T, false, NP, X, false, WHOLE, LINES>(o, p, s);
}

template <typename T, bool WHOLE, bool LINES>
hipError_t with_rows(const RowOrder &o, const RowProduct &p, hipStream_t s)
{
    constexpr int M = kPairs<T>;
    if (p.K <= M / 4 * 2 * kU) return with_pairs<T, M / 4, WHOLE, LINES>(o, p, s);
    if (p.K <= M / 2 * 2 * kU) return with_pairs<T, M / 2, WHOLE, LINES>(o, p, s);
    return with_pairs<T, M, WHOLE, LINES>(o, p, s);
}

template <typename T> hipError_t pick(const RowOrder &o, const RowProduct &p, hipStream_t s)
{
    const uintptr_t out = reinterpret_cast<uintptr_t>(p.out);
    constexpr int kHalf = kPiece<T> / 2;
    if (p.N % kHalf == 0 && p.out_stride % kHalf == 0 && out % 64 == 0) return with_rows<T, true, true>(o, p, s);
    if (p.N % 4 == 0 && p.out_stride % 4 == 0 && out % (4 * sizeof(T)) == 0) return with_rows<T, true, false>(o, p, s);
    return with_rows<T, false, false>(o, p, s);
}

template <typename T> bool takes(const RowProduct &p)
{
    if (p.narrow || p.N <= kCols || p.K > 2 * kPairs<T> * kU) return false;
    if (!p.h && !p.a) return p.w_group != 0 && (!p.w_nk || p.K >= kU);
    return !p.w_nk && kNarrow<T> * narrow_width(p.r) <= 2 * kExtPairs<T> * kU;
}

}  // namespace

bool row_wide_takes(int dtype, const RowProduct &p)
{
    return dtype == CGTP_BF16 ? takes<bf16_t>(p) : takes<float>(p);
}

// Tiles of one adapter each.
bool adapter_wide_takes(int dtype, const RowOrder &o, const RowProduct &p)
{
    return p.a && !p.h_out && own_tiles(o) && row_wide_takes(dtype, p);
}

hipError_t launch_row_wide(int dtype, const RowOrder &o, const RowProduct &p, hipStream_t s)
{
    return dtype == CGTP_BF16 ? pick<bf16_t>(o, p, s) : pick<float>(o, p, s);
}

}  // namespace cgtp
