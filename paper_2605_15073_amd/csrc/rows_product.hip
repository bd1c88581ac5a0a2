// Products of grouped rows, out_i = in_i W_g, on the matrix cores (cgtp_grouped_linear, the row
// gradients, the narrow products of adapters and the shared projection with them).
//
// A workgroup owns up to BM rows of one group (of any groups where W is shared) and runs over tiles
// of BN columns of its share of the output, so that its input rows come from HBM once and from the
// L2 for every further column tile; the weights of a group stay in the L2s. The loads of the next
// step (rows and weights, kStep deep) are in flight while a step is multiplied. None of them is under a
// condition (adapters' gradients 500 us, with one 530): a vector that would pass the end of its row starts
// early, one without values points to some that exist, and both are put right when they are staged. Only
// widths below a vector (WIDE false) load value by value.
//
// Measured: row gradients of 261,766 rows, 1344 -> 128 bf16, 197 us (3.9 TB/s; bound by the reads and the
// latency of a step's loads); 60,000 rows, 896 x 896: 174 us in bf16 (550 TFLOP/s), 658 us in fp32
// (146 TFLOP/s, six instructions a product: bound by the matrix cores and the splitting of the operands).
//
// Adapters: after the steps over the shared W, a tile's sums go on over the adapters of its rows, one
// segment of rows at a time, with the narrow product's result as input rows (zero outside the
// segment) and the adapter's second matrix as weights: the epilogue is fused, and rows of many
// adapters share the tile.
//
// FUSED: tiles of one adapter each, whose narrow product is formed here too. Its matrix, [r][K] like the
// shared weights, gives 32 more columns of the tile (so the input is read once for both); the result goes
// through LDS as the input rows of one more step (bf16 ranks above 16: two, as its parts fill them), over the
// adapter's second matrix: 131,327 rows of 8 adapters, 896 -> 128, rank 16, fp32 290 us, bf16 86; 100,000 rows of 100,
// fp32 265 where the two products apart take 298, bf16 71 and 105.
#include "internal.h"
#include "rows_tile.h"

namespace cgtp {

namespace {

using namespace rows;

template <typename T, bool WNK, int BM, int BN, int WR, bool WIDE, bool FUSED>
__global__ __launch_bounds__(kThreads, sizeof(T) == 4 ? 2 : 1) void k_row_product(RowOrder o, RowProduct p, int splits)
{
    constexpr int KG = kGroups<T>, BK = kStep<T>, P = kNarrow<T>, Q = kSplit<T>, CW = kWide<T>;
    constexpr int WC = 4 / WR, TR = BM / WR / 32, TC = BN / WC / 32;
    constexpr int BX = BN + (FUSED ? 32 : 0), TX = TC + (FUSED ? 1 : 0);  // with the narrow product's columns
    static_assert(!FUSED || (WNK && WR == 4 && WIDE), "fused: a wave has whole rows, weights are [N][K]");
    static_assert(TR >= 1 && TC >= 1, "tile");
    constexpr int kLanes = kThreads / KG;              // rows staged at once
    constexpr int NR = BM / kLanes > 0 ? BM / kLanes : 1;
    constexpr int NC = (BX + kLanes - 1) / kLanes;
    __shared__ uint4_t s_tiles[kTile<T, BX> + kTile<T, BM>];
    uint4_t *const s_cols = s_tiles, *const s_rows = s_tiles + kTile<T, BX>;
    __shared__ int s_row[BM], s_g[BM], s_seg_g[BM], s_seg_at[BM + 1], s_nseg, s_any;

    const bool shared_w = !FUSED && p.w_group == 0;
    const int64_t index = tile_at(blockIdx.x, blockIdx.z, gridDim.x);
    Tile t;
    if (shared_w) {
        t.p0 = index * BM;
        if (t.p0 >= o.n) return;
        t.p1 = t.p0 + BM < o.n ? t.p0 + BM : o.n;
        t.g = 0;
    } else {
        t = find_tile(o, TileRows<BM>{}, index);
        if (t.g < 0 || t.p0 >= t.p1) return;
    }
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int rows = (int)(t.p1 - t.p0);
    // this workgroup's column tiles
    const int ctiles = (p.N + BN - 1) / BN;
    const int ct0 = (int)((int64_t)ctiles * blockIdx.y / splits);
    const int ct1 = (int)((int64_t)ctiles * (blockIdx.y + 1) / splits);
    if (ct0 >= ct1) return;
    const int col_end = ct1 * BN < p.N ? ct1 * BN : p.N;

    const int my_row = tid < rows ? row_at(o, t.p0 + tid) : -1;
    if (tid < BM) s_row[tid] = my_row;
    if (tid == 0) s_any = -1;
    if (!FUSED && !shared_w && t.g == o.G) {  // rows of no group
        if (p.narrow) return;
        __syncthreads();
        store_zeros<T>(p, s_row, rows, ct0 * BN, col_end);
        return;
    }
    const bool grouped = t.g < o.G;
    int nseg = 0;
    __syncthreads();
    if (my_row >= 0) s_any = my_row;  // any row of the tile
    if (shared_w && p.h) nseg = find_segments<BM>(o, t.p0, rows, s_g, s_seg_g, s_seg_at, &s_nseg);
    else __syncthreads();
    if (s_any < 0) return;

    // rows of the input, and of [N][K] weights: k-group tid % KG of lanes tid / KG + kLanes i
    const int kg = tid % KG, rr = tid / KG;
    const T *in[NR];
#pragma unroll
    for (int i = 0; i < NR; ++i) {
        const int r = rr + kLanes * i, row = r < BM ? s_row[r] : -1;
        in[i] = static_cast<const T *>(p.in) + (row < 0 ? s_any : row) * p.in_stride;  // any: never stored
    }
    const T *const w = static_cast<const T *>(p.w) + (FUSED ? 0 : (int64_t)t.g * p.w_group);
    const T *const narrow_w = FUSED && grouped ? static_cast<const T *>(p.a) + (int64_t)t.g * p.r * p.K : w;
    const int W = narrow_width(p.r);  // of a part of the narrow input
    // transposed weights: columns CW tc .. CW tc + CW - 1, k-group tg
    constexpr bool kIdle = BN / CW * KG < kThreads;  // some threads have none to stage
    const int tc = tid % (BN / CW), tg = kIdle ? tid / (BN / CW) % KG : tid / (BN / CW);
    const bool has_w = !kIdle || tid < BN / CW * KG;

    // The steps: of the shared or the group's weights (seg < 0), then of each adapter.
    struct Cursor { int ct, seg, k; } next = {ct0, -1, 0}, now = next;  // the step to load, to multiply
    auto advance = [&](Cursor &c) {
        c.k += BK;
        if (c.k >= (c.seg < 0 ? p.K : P * W)) {
            c.k = 0;
            if (++c.seg >= nseg) {
                c.seg = -1;
                ++c.ct;
            }
        }
    };
    struct {
        Raw8<T> x[NR], wn[WNK ? NC : 1];
        uint2_t wt[WNK ? 1 : 8];
        int xk, wk;  // values that exist of this thread's k-group of rows and weights
        int xe, we;  // what their loads started early
        unsigned rows;  // bit i: x[i] is of a row that takes part
    } l;
    float odd = 0.f;  // NaN once a result is not finite
    float sign = 1.f;  // of the step's rows
    auto fetch = [&]() {
        if (!WIDE && next.ct >= ct1) return;  // else past the last step the last tile's first loads again
        const bool ext = next.seg >= 0;
        const int seg = ext ? next.seg : 0, c0 = (next.ct < ct1 ? next.ct : ct1 - 1) * BN, k = next.k;
        const int K = ext ? P * W : p.K;   // of the rows
        const int ld = ext ? p.r : p.K;    // of the weights
        const T *wb = w;
        int at = 0, end = BM;
        if (nseg > 0) {
            wb = ext ? static_cast<const T *>(p.v) + (int64_t)s_seg_g[seg] * p.r * p.N : w;
            at = ext ? s_seg_at[seg] : 0;
            end = ext ? s_seg_at[seg + 1] : BM;
        }
        const int kx = k + kg * kU;
        l.xk = K - kx;
        const int xs = l.xk > 0 ? start8(kx, K) : 0;
        l.xe = l.xk > 0 ? kx - xs : 0;
        l.rows = 0;
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            const int r = rr + kLanes * i;
            if (r >= at && r < end) l.rows |= 1u << i;
            const T *q = ext ? static_cast<const T *>(p.h) + (t.p0 + (r < rows ? r : 0)) * K : in[i];
            if constexpr (WIDE) l.x[i] = load_any8(q + xs);
            else l.x[i] = load_row8<T, false>(q + kx, l.xk);
        }
        int kw = WNK ? kx : k + tg * kU;
        const bool in_k = kw < K;
        if (ext) kw = narrow_k<T>(kw, W);
        l.wk = in_k ? ld - kw : 0;
        if constexpr (WNK) {
            const int ws = l.wk > 0 ? start8(kw, ld) : 0;
            l.we = l.wk > 0 ? kw - ws : 0;
#pragma unroll
            for (int i = 0; i < NC; ++i) {
                const int cl = rr + kLanes * i, c = c0 + cl;
                const T *q = wb + (int64_t)(c < p.N ? c : p.N - 1) * ld;
                if (FUSED && cl >= BN) q = narrow_w + (int64_t)(grouped && cl - BN < p.r ? cl - BN : 0) * ld;
                if constexpr (WIDE) l.wn[i] = load_any8(q + ws);
                else l.wn[i] = load_row8<T, false>(q + kw, l.wk);
            }
        } else {
            const int c = c0 + CW * tc;
            l.we = c + CW <= p.N || c >= p.N ? 0 : c + CW - p.N;
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const T *q = wb + (int64_t)(u < l.wk ? kw + u : 0) * p.N;
                if constexpr (WIDE) l.wt[u] = *reinterpret_cast<const uint2_any *>(q + (c + CW <= p.N ? c : p.N - CW));
                else l.wt[u] = load_8<T, false>(q + c, u < l.wk ? p.N - c : 0);
            }
        }
        if (next.ct < ct1) advance(next);
    };
    auto stage = [&]() {
        uint4_t u[Q];
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            if (BM < kLanes && rr >= BM) break;
            if (l.xk < kU || !(l.rows >> i & 1)) settle(l.x[i], WIDE ? l.xe : 0, l.rows >> i & 1 ? l.xk : 0);
            to_units(l.x[i], u, sign);
            put<T, BM>(s_rows, KG, kg, rr + kLanes * i, u);
        }
        if constexpr (WNK) {
#pragma unroll
            for (int i = 0; i < NC; ++i) {
                if (BX % kLanes != 0 && rr + kLanes * i >= BX) break;
                if (l.wk < kU) settle(l.wn[i], WIDE ? l.we : 0, l.wk);
                to_units(l.wn[i], u);
                put<T, BX>(s_cols, KG, kg, rr + kLanes * i, u);
            }
        } else if (has_w) {
            if (l.wk < kU) {
#pragma unroll
                for (int e = 0; e < 8; ++e) l.wt[e] = e < l.wk ? l.wt[e] : uint2_t{0, 0};
            }
            if (WIDE && l.we > 0) {
#pragma unroll
                for (int e = 0; e < 8; ++e) settle<T>(l.wt[e], l.we);
            }
            uint4_t c[CW][Q];
            to_units(l.wt, c);
#pragma unroll
            for (int j = 0; j < CW; ++j) put<T, BX>(s_cols, KG, tg, place<T>(CW * tc + j), c[j]);
        }
    };

    const int wr = wave % WR, wc = wave / WR;
    const int r0 = wr * (BM / WR), c0w = wc * (BN / WC);
    float16_t acc[TX][TR];
    auto clear = [&]() {
#pragma unroll
        for (int c = 0; c < TX; ++c)
#pragma unroll
            for (int r = 0; r < TR; ++r)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[c][r][i] = 0.f;
    };
    auto store = [&](int ct) {
        const int c0 = ct * BN + c0w;
        if (p.narrow) {
            const float scale = p.narrow_scale ? p.narrow_scale[t.g] : 1.f;
            const int No = narrow_width(p.N);
#pragma unroll
            for (int r = 0; r < TR; ++r) {
                const int pl = r0 + 32 * r + (lane & 31);
                if (pl >= rows) continue;
                T *const q = static_cast<T *>(p.out) + (t.p0 + pl) * (P * No);
#pragma unroll
                for (int c = 0; c < TC; ++c)
#pragma unroll
                    for (int v = 0; v < 4; ++v) {
                        const int col = c0 + 32 * c + vec_col<T, !WNK>(v, half);
                        float4_t x = vec_val<T, !WNK>(acc[c][r], v);
#pragma unroll
                        for (int e = 0; e < 4; ++e) x[e] = col + e < p.N ? x[e] * scale : 0.f;
                        if (col < No) store_narrow(q + col, No, x);
                    }
            }
        } else {
#pragma unroll
            for (int r = 0; r < TR; ++r) {
                const int row = s_row[r0 + 32 * r + (lane & 31)];
                if (row < 0) continue;
                T *const q = static_cast<T *>(p.out) + row * p.out_stride;
#pragma unroll
                for (int c = 0; c < TC; ++c)
#pragma unroll
                    for (int v = 0; v < 4; ++v) {
                        const int col = c0 + 32 * c + vec_col<T, !WNK>(v, half);
                        store_four<false>(q + col, vec_val<T, !WNK>(acc[c][r], v), p.N - col);
                    }
            }
        }
    };
    // FUSED: the narrow sums, scaled, are written out and become the rows of a step over v
    auto narrow_step = [&]() {
        const float scale = p.narrow_scale && grouped ? p.narrow_scale[t.g] : grouped ? 1.f : 0.f;
        const int place = r0 + (lane & 31);
        T *const out = static_cast<T *>(p.h_out) + (t.p0 + place) * (P * W);
        float4_t x[4];
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const int col = vec_col<T, false>(v, half);
            x[v] = vec_val<T, false>(acc[TX - 1][0], v);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[v][e] = grouped && col + e < p.r ? x[v][e] * scale : 0.f;
            if (p.h_out && grouped && place < rows && col < W) store_narrow(out + col, W, x[v]);
        }
        const int most = KG * kU / W;  // parts that a step has room for: all, or two of bf16's three
        for (int first = 0; first < P; first += most) {
            const int count = P - first < most ? P - first : most;
            __syncthreads();  // the last step's tiles are consumed
#pragma unroll
            for (int v = 0; v < 4; ++v) put_narrow<T, BM>(s_rows, v, place, half, W / kU, first, count, x[v]);
            uint4_t u[Q];
            for (int task = tid; task < BN * KG; task += kThreads) {
                const int g = task % KG, c = task / KG;
                const bool in_k = g * kU < count * W && c < p.N && grouped;
                const int k = narrow_k<T>(g * kU, W);
                const T *const q = static_cast<const T *>(p.v) + ((int64_t)(grouped ? t.g : 0) * p.N + c) * p.r + k;
                to_units(load_row8<T, false>(q, in_k ? p.r - k : 0), u);
                put<T, BX>(s_cols, KG, g, c, u);
            }
            __syncthreads();
            step_products<T, BX, BM, TC, TR>(acc, s_cols, s_rows, c0w, r0, 1.f);
        }
    };
    auto step = [&]() {
        __syncthreads();
        stage();
        __syncthreads();
        fetch();
        step_products<T, BX, BM, TX, TR>(acc, s_cols, s_rows, c0w, r0, sign);
        sign = -sign;
        const int ct = now.ct;
        advance(now);
        if (now.ct != ct) {
            if constexpr (FUSED) narrow_step();
            store(ct);
            if (Q > 1 || FUSED || nseg > 0)
#pragma unroll
                for (int c = 0; c < TC; ++c)
#pragma unroll
                    for (int r = 0; r < TR; ++r) probe(odd, acc[c][r]);
            clear();
        }
    };
    clear();
    fetch();
    while (now.ct < ct1) step();
    if ((Q > 1 || FUSED || nseg > 0) && __syncthreads_or(odd != odd)) {
        float *const h = FUSED ? reinterpret_cast<float *>(s_tiles) : nullptr;
        if constexpr (FUSED) {
            stores_done();
            static_assert(sizeof(s_tiles) >= sizeof(float) * BM * 32, "rows of up to 32 values");
            for (int e = tid; e < rows * p.r; e += kThreads) {
                const int r = e / p.r, c = e % p.r;
                float sum = 0.f;
                if (grouped && s_row[r] >= 0)
                    for (int k = 0; k < p.K; ++k)
                        sum += (float)static_cast<const T *>(p.in)[s_row[r] * p.in_stride + k] *
                               (float)narrow_w[(int64_t)c * p.K + k];
                if (p.narrow_scale && grouped) sum *= p.narrow_scale[t.g];
                h[32 * r + c] = sum;
                if constexpr (Q > 1) {  // sums of bf16 products are right as they are
                    float *const out = static_cast<float *>(p.h_out) + (t.p0 + r) * W + c;
                    if (p.h_out && grouped && !__builtin_isfinite(stored(out))) *out = sum;
                }
            }
            if (tid < rows) s_g[tid] = t.g;
        }
        row_plain_sums<T, WNK>(o, p, FUSED ? 0 : t.g, t.p0, rows, s_row, s_g, ct0 * BN, col_end, h);
    }
}

template <typename T, bool WNK, int BM, int BN, int WR, bool FUSED = false>
hipError_t launch(const RowOrder &o, const RowProduct &p, hipStream_t s)
{
    // rows of eight values or more, of columns or k as they are loaded
    const bool wide = p.K >= kU && (WNK ? !p.h || p.r >= kU : p.N >= kWide<T>);
    const int64_t tiles = p.w_group || FUSED ? o.n / BM + o.G + 1 : (o.n + BM - 1) / BM;
    const int ctiles = (p.N + BN - 1) / BN;
    // few rows: column tiles go to workgroups of their own (20,000 rows, 300 -> 896 fp32, with 512, 2,048 and 8,192
    // workgroups 119, 113 and 113 us; 60,000 rows, 300 -> 1344 443, 439 and 455, bf16 160, 155 and 156)
    int splits = (int)(2048 / tiles);
    splits = splits < 1 ? 1 : splits > ctiles ? ctiles : splits;
    auto *kernel = FUSED || wide ? k_row_product<T, WNK, BM, BN, WR, true, FUSED>
                                 : k_row_product<T, WNK, BM, BN, WR, FUSED, FUSED>;
    const TileGrid grid = tile_grid(tiles);
    hipLaunchKernelGGL(kernel, dim3(grid.x, (unsigned)splits, grid.z), dim3(kThreads), 0, s, o, p, splits);
    return hipGetLastError();
}

template <typename T, bool WNK>
hipError_t pick(const RowOrder &o, const RowProduct &p, hipStream_t s)
{
    const int dtype = sizeof(T) == 2 ? CGTP_BF16 : CGTP_F32;
    if constexpr (WNK)
        // 100,000 rows, 896 -> 64, us with tiles of 64 and 128 columns: bf16 51 and 62, fp32 169 and 234
        if (p.a) return p.N <= 64 ? launch<T, true, 128, 64, 4, true>(o, p, s) : launch<T, true, 128, 128, 4, true>(o, p, s);
    if (p.a) return launch_row_wide(dtype, o, p, s);
    if (row_few_takes(dtype, o, p)) return launch_row_few(o, p, s);
    const int64_t groups = p.w_group ? o.G : 1;
    // Rows of a tile, by those of a group. Us with tiles of 32 and of 128 rows (or the wide form), 500 groups of 24, 32,
    // 40, 48 and 64 rows: 256 -> 256 bf16 22 27 33 34 41 and 27 27 28 29 31, fp32 41 51 66 70 79 and 74 74 74 76 78;
    // 64 -> 448 bf16 15 19 24 24 28 and 18 18 18 17 18, fp32 29 34 43 44 49 and 37 37 38 38 40.
    const bool few = o.n < 40 * groups;
    // Columns of a tile: 200,000 rows, us with 32, 64 and 128: bf16 256 -> 32 29 33 38, -> 64 49 36 38, -> 72 70 60 42;
    // fp32 1344 -> 32 283 433 542, -> 64 563 444 555, -> 72 865 842 557.
    if (!few && row_wide_takes(dtype, p)) return launch_row_wide(dtype, o, p, s);
    if (p.N <= 32) return launch<T, WNK, 128, 32, 4>(o, p, s);
    if (few && p.N > 64) return launch<T, WNK, 32, 128, 1>(o, p, s);
    if (few || p.N <= 64) return launch<T, WNK, 64, 64, 2>(o, p, s);
    return launch<T, WNK, 128, 128, kWaveRows<T>>(o, p, s);
}

}  // namespace

size_t narrow_bytes(int dtype, int64_t n_rows, int N)
{
    return (size_t)n_rows * narrow_width(N) * (dtype == CGTP_BF16 ? kNarrow<bf16_t> * 2 : 4);
}

// Adapters with tiles of their own, one column tile of [N][K] weights.
bool adapter_product_takes(int dtype, const RowOrder &o, const RowProduct &p)
{
    return p.a && p.w_nk && p.N <= 128 && p.r <= 32 && p.K >= kU && own_tiles(o);
}

hipError_t launch_row_product(int dtype, const RowOrder &o, const RowProduct &p, hipStream_t s)
{
    if (dtype == CGTP_BF16) return p.w_nk ? pick<bf16_t, true>(o, p, s) : pick<bf16_t, false>(o, p, s);
    return p.w_nk ? pick<float, true>(o, p, s) : pick<float, false>(o, p, s);
}

}  // namespace cgtp
