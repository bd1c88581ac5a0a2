// Products of grouped rows, out_i = in_i W_g, on the matrix cores (cgtp_grouped_linear, the row
// gradients, the narrow products of adapters and the shared projection with them).
//
// A workgroup owns up to BM rows of one group (of any groups where W is shared) and runs over tiles
// of BN columns of its share of the output, so that its input rows come from HBM once and from the
// L2 for every further column tile; the weights of a group stay in the L2s. The loads of a step
// (rows and weights, kStep deep) are in flight while the step before is multiplied.
//
// Adapters: after the steps over the shared W, a tile's sums go on over the adapters of its rows, one
// segment of rows at a time, with the narrow product's result as input rows (zero outside the
// segment) and the adapter's second matrix as weights: the epilogue is fused, and rows of many
// adapters share the tile.
#include "internal.h"
#include "rows_tile.h"

namespace cgtp {

namespace {

using namespace rows;

template <typename T, bool WNK, int BM, int BN, int WR, bool VEC>
__global__ __launch_bounds__(kThreads) void k_row_product(RowOrder o, RowProduct p, int splits, bool v_vec)
{
    constexpr int KG = kGroups<T>, BK = kStep<T>, P = kNarrow<T>, Q = kSplit<T>, CW = kWide<T>;
    constexpr int WC = 4 / WR, TR = BM / WR / 32, TC = BN / WC / 32;
    constexpr int kShift = BM == 128 ? 7 : BM == 64 ? 6 : 5;
    static_assert(BM == 1 << kShift && TR >= 1 && TC >= 1, "tile");
    constexpr int kLanes = kThreads / KG;              // rows staged at once
    constexpr int NR = BM / kLanes > 0 ? BM / kLanes : 1;
    constexpr int NC = BN / kLanes > 0 ? BN / kLanes : 1;
    __shared__ uint4_t s_cols[kTile<T, BN>], s_rows[kTile<T, BM>];
    __shared__ int s_row[BM], s_g[BM], s_seg_g[BM], s_seg_at[BM + 1], s_nseg;

    const bool shared_w = p.w_group == 0;
    Tile t;
    if (shared_w) {
        t.p0 = (int64_t)blockIdx.x * BM;
        t.p1 = t.p0 + BM < o.n ? t.p0 + BM : o.n;
        t.g = 0;
    } else {
        t = find_tile(o, kShift, blockIdx.x);
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

    if (tid < BM) s_row[tid] = tid < rows ? row_at(o, t.p0 + tid) : -1;
    if (!shared_w && t.g == o.G) {  // rows of no group
        if (p.narrow) return;
        __syncthreads();
        store_zeros<T>(p, s_row, rows, ct0 * BN, col_end);
        return;
    }
    int nseg = 0;
    if (shared_w && p.h) nseg = find_segments<BM>(o, t.p0, rows, s_g, s_seg_g, s_seg_at, &s_nseg);
    __syncthreads();

    // rows of the input, and of [N][K] weights: k-group tid % KG of lanes tid / KG + kLanes i
    const int kg = tid % KG, rr = tid / KG;
    const T *in[NR];
#pragma unroll
    for (int i = 0; i < NR; ++i) {
        const int r = rr + kLanes * i, row = r < BM ? s_row[r] : -1;
        in[i] = row >= 0 ? static_cast<const T *>(p.in) + row * p.in_stride + kg * kU : nullptr;
    }
    const T *const w = static_cast<const T *>(p.w) + (int64_t)t.g * p.w_group;
    const int W = narrow_width(p.r);  // of a part of the narrow input
    // transposed weights: columns CW tc .. CW tc + CW - 1, k-group tg
    const int tc = tid % (BN / CW), tg = tid / (BN / CW);

    Raw8<T> xr[NR], wn[WNK ? NC : 1];
    uint2_t wt[8];
    bool lose = false;
    // the loads of step k of column tile ct; seg < 0: the shared weights, else an adapter
    auto fetch = [&](int ct, int seg, int k) {
        const int c0 = ct * BN;
        int K = p.K;
        const T *wb = w;
        int wk = p.K;  // k of the weights from which on there are none
        if (seg >= 0) {
            K = P * W;
            wb = static_cast<const T *>(p.v) + (int64_t)s_seg_g[seg] * p.r * p.N;
            wk = p.r;
            const int at = s_seg_at[seg], end = s_seg_at[seg + 1];
#pragma unroll
            for (int i = 0; i < NR; ++i) {
                const int r = rr + kLanes * i;
                const int left = r >= at && r < end && in[i] ? K - k - kg * kU : 0;
                xr[i] = load_row8<T, true>(static_cast<const T *>(p.h) + (t.p0 + r) * K + k + kg * kU, left);
            }
        } else {
#pragma unroll
            for (int i = 0; i < NR; ++i) xr[i] = load_row8<T, VEC>(in[i] + k, in[i] ? K - k - kg * kU : 0);
        }
        if constexpr (WNK) {
#pragma unroll
            for (int i = 0; i < NC; ++i) {
                const int c = c0 + rr + kLanes * i;
                int kk = k + kg * kU;
                const bool in_k = kk < K && rr + kLanes * i < BN;
                if (seg >= 0 && P == 2 && kk >= W) kk -= W;  // the second part meets the same weights
                const T *const q = wb + (int64_t)c * wk + kk;
                const int left = c < p.N && in_k ? wk - kk : 0;
                if (seg >= 0 && !v_vec) wn[i] = load_row8<T, false>(q, left);
                else wn[i] = load_row8<T, VEC>(q, left);
            }
        } else if (tg < KG) {
            const int c = c0 + CW * tc;
            int kk = k + tg * kU;
            const bool in_k = kk < K;
            if (seg >= 0 && P == 2 && kk >= W) kk -= W;
#pragma unroll
            for (int u = 0; u < 8; ++u)
                wt[u] = load_8<T, VEC>(wb + (int64_t)(kk + u) * p.N + c, in_k && kk + u < wk ? p.N - c : 0);
        }
    };
    auto stage = [&]() {
        uint4_t u[Q];
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            if (BM < kLanes && rr >= BM) break;
            to_units(xr[i], u, lose);
            put<T, BM>(s_rows, KG, kg, rr + kLanes * i, u);
        }
        if constexpr (WNK) {
#pragma unroll
            for (int i = 0; i < NC; ++i) {
                if (BN < kLanes && rr >= BN) break;
                to_units(wn[i], u, lose);
                put<T, BN>(s_cols, KG, kg, rr + kLanes * i, u);
            }
        } else if (tg < KG) {
            uint4_t c[CW][Q];
            to_units(wt, c, lose);
#pragma unroll
            for (int j = 0; j < CW; ++j) put<T, BN>(s_cols, KG, tg, place<T>(CW * tc + j), c[j]);
        }
    };

    const int wr = wave % WR, wc = wave / WR;
    const int r0 = wr * (BM / WR), c0w = wc * (BN / WC);
    float16_t acc[TC][TR];
    int ct = ct0, seg = -1, k = 0;
    fetch(ct, seg, k);
    while (ct < ct1) {
#pragma unroll
        for (int c = 0; c < TC; ++c)
#pragma unroll
            for (int r = 0; r < TR; ++r)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[c][r][i] = 0.f;
        const int now = ct;
        while (ct == now) {
            __syncthreads();
            stage();
            __syncthreads();
            k += BK;
            if (k >= (seg < 0 ? p.K : P * W)) {
                k = 0;
                if (++seg >= nseg) {
                    seg = -1;
                    ++ct;
                }
            }
            if (ct < ct1) fetch(ct, seg, k);
            step_products<T, BN, BM, TC, TR>(acc, s_cols, s_rows, c0w, r0);
        }
        const int c0 = now * BN + c0w;
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
                        store_four<VEC>(q + col, vec_val<T, !WNK>(acc[c][r], v), p.N - col);
                    }
            }
        }
    }
    if constexpr (Q > 1) {
        __threadfence_block();
        if (__syncthreads_or(lose)) row_plain_sums<WNK>(o, p, t.g, t.p0, rows, s_row, s_g, ct0 * BN, col_end);
    }
}

template <typename T, bool WNK, int BM, int BN, int WR>
hipError_t launch(const RowOrder &o, const RowProduct &p, hipStream_t s)
{
    constexpr int V = 16 / (int)sizeof(T);
    const bool vec = aligned_rows<T>(p.in, p.in_stride) && p.K % V == 0 && p.N % V == 0 &&
                     aligned_rows<T>(p.w, 0) && (p.narrow || aligned_rows<T>(p.out, p.out_stride)) &&
                     (!p.h || aligned_rows<T>(p.v, 0));
    const bool v_vec = vec && p.r % V == 0;  // rows of r adapter weights
    const int64_t tiles = p.w_group ? o.n / BM + o.G + 1 : (o.n + BM - 1) / BM;
    const int ctiles = (p.N + BN - 1) / BN;
    // few rows: column tiles go to workgroups of their own
    int splits = (int)(2048 / tiles);
    splits = splits < 1 ? 1 : splits > ctiles ? ctiles : splits;
    auto *kernel = vec ? k_row_product<T, WNK, BM, BN, WR, true> : k_row_product<T, WNK, BM, BN, WR, false>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)tiles, (unsigned)splits), dim3(kThreads), 0, s, o, p, splits, v_vec);
    return hipGetLastError();
}

template <typename T, bool WNK>
hipError_t pick(const RowOrder &o, const RowProduct &p, hipStream_t s)
{
    const bool few = o.n < 64 * (p.w_group ? (int64_t)o.G : 1);  // rows per group
    const int dtype = sizeof(T) == 2 ? CGTP_BF16 : CGTP_F32;
    if (!few && row_wide_takes(dtype, p)) return launch_row_wide(dtype, o, p, s);
    if (p.N <= 32) return launch<T, WNK, 128, 32, 4>(o, p, s);
    if (few && p.N > 64) return launch<T, WNK, 32, 128, 1>(o, p, s);
    if (few || p.N <= 64) return launch<T, WNK, 64, 64, 2>(o, p, s);
    return launch<T, WNK, 128, 128, 2>(o, p, s);
}

}  // namespace

size_t narrow_bytes(int dtype, int64_t n_rows, int N)
{
    return (size_t)n_rows * narrow_width(N) * 4;  // one fp32 or two bf16
}

hipError_t launch_row_product(int dtype, const RowOrder &o, const RowProduct &p, hipStream_t s)
{
    if (dtype == CGTP_BF16) return p.w_nk ? pick<bf16_t, true>(o, p, s) : pick<bf16_t, false>(o, p, s);
    return p.w_nk ? pick<float, true>(o, p, s) : pick<float, false>(o, p, s);
}

}  // namespace cgtp
