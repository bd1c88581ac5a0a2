// Weight gradients of grouped rows, out_g = sum over the group's rows of a_i b_i^T, on the matrix
// cores: the products' k is the row, so both operands are transposed while they are staged.
//
// A workgroup owns one tile of the output and one chunk of a group's rows, R at most. A group
// of one chunk is written at once; the sums of a larger one go to the workspace, a slot per chunk,
// and a second kernel adds the slots in their order, so that the result does not depend on which
// workgroup came first. Slots: 2 (start / R) + j. A group of more than one chunk covers at least
// one multiple of the chunk size beyond its start, and 2 floor((s + m) / R) - 2 floor(s / R) >=
// ceil(m / R) for m > R, so slots of different groups never meet and 2 (n / R) + 2 suffice.
//
// With a narrow product's result as b, bf16 multiplies all of its parts into the same sums.
//
// Half of the waves stage a, half b, 16 bytes of eight rows a thread: 226 us for 261,766 rows, 128 x 1344 bf16
// (0.77 GB read, 0.09 GB of slots written; the join, 22 us, with it), where every wave staging both in 8 bytes took 28
// more. Bound by the latency of the loads of a step, of which three workgroups on a compute unit hide a part. dA of
// 131,327 rows, 128 x 16 bf16, with the narrow product 78 us.
#include "internal.h"
#include "rows_tile.h"

#include <cmath>

namespace cgtp {

namespace {

using namespace rows;

template <typename T, int BM, int BN, int WR, bool WIDE, bool NARROW>
__global__ __launch_bounds__(kThreads) void k_row_outer(RowOrder o, RowOuter q, ChunkRows R, bool big,
                                                        float *slots)
{
    constexpr int KG = kGroups<T>, BK = kStep<T>, P = NARROW ? kNarrow<T> : 1, Q = kSplit<T>, CW = kFull<T>;
    constexpr int WC = 4 / WR, TR = BM / WR / 32, TC = BN / WC / 32;
    __shared__ uint4_t s_cols[P][kTile<T, BN>], s_rows[kTile<T, BM>];
    __shared__ int64_t s_at[2][2][BK];  // where the rows of a and b of a step start
    __shared__ unsigned s_rows_in[2][BK / 32];  // bit per row of a step: it exists

    // Block b runs on XCD b % 8: the tiles of a chunk, which share its rows, follow each other on one.
    const int B = NARROW ? q.r : q.B;
    const int btiles = (B + BN - 1) / BN, tiles = btiles * ((q.A + BM - 1) / BM);
    const int on_xcd = blockIdx.x / 8, tile = on_xcd % tiles;
    const int64_t chunk = (int64_t)(on_xcd / tiles) * 8 + blockIdx.x % 8;
    const Tile t = big ? find_big(o, R.rows, chunk) : find_tile(o, R, chunk);
    if (t.g < 0 || t.g >= o.G) return;
    const int W = narrow_width(B);
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int a0 = tile / btiles * BM, b0 = tile % btiles * BN;
    const int wr = wave % WR, wc = wave / WR;
    const int r0 = wr * (BM / WR), c0w = wc * (BN / WC);

    // waves 0 and 1 stage a, waves 2 and 3 b: lanes first .. first + CW - 1 of k-group kg, of b of one of its parts.
    // b's parts are spread over the threads (narrow tiles leave most without work in one part alone).
    constexpr int kHalf = kThreads / 2, kPart = KG * (BN / CW), NL = (P * kPart + kHalf - 1) / kHalf;
    static_assert(KG * (BM / CW) <= kHalf, "a: one task a thread");
    const bool of_b = wave >= 2;
    const int width = !of_b ? q.A : NARROW ? W : B;
    struct Task {
        bool has;
        int part, kg, first, early;
        const T *from;
    } tasks[NL];
#pragma unroll
    for (int i = 0; i < NL; ++i) {
        const int all = tid % kHalf + kHalf * i, lanes = of_b ? BN : BM, task = of_b ? all % kPart : all;
        Task &k = tasks[i];
        k.part = of_b ? all / kPart : 0;
        k.kg = task / (lanes / CW);
        k.first = CW * (task % (lanes / CW));
        k.has = k.kg < KG && k.part < P && (of_b || i == 0);
        const int col = (of_b ? b0 : a0) + k.first;
        k.early = WIDE && col < width && col + CW > width ? col + CW - width : 0;
        k.from = static_cast<const T *>(!of_b ? q.a : NARROW ? q.h : q.b) +
                 ((k.has ? k.part : 0) * (NARROW ? W : 0) + (WIDE && col + CW > width ? width - CW : col));
    }
    uint4_t l[NL][8];
    unsigned in[NL];  // bit u: row u of the k-group exists
    float sign = 1.f;  // of the step's a
    const int steps = (int)((t.p1 - t.p0 + BK - 1) / BK);
    // ids of the rows of step s, -1 past the chunk; loads without a condition, as the operands'
    const int32_t *const ids_at = o.order ? o.order : o.offsets;
    int id = -1;
    auto fetch_ids = [&](int s) {
        const int64_t pos = t.p0 + (int64_t)s * BK + tid % BK;
        id = ids_at[o.order && pos < t.p1 ? pos : 0];
    };
    auto put_ids = [&](int s) {
        const int64_t pos = t.p0 + (int64_t)s * BK + tid;
        const int row = o.order ? id : (int)pos;
        const bool in = pos < t.p1 && (unsigned)row < (unsigned)o.n;
        if (tid < BK) {
            s_at[0][s & 1][tid] = in ? row * q.a_stride : 0;  // row 0 in place of none: zeroed when staged
            s_at[1][s & 1][tid] = !in ? 0 : NARROW ? pos * (P * W) : row * q.b_stride;
            const unsigned long long m = __ballot(in);
            if (tid % 32 == 0) s_rows_in[s & 1][tid / 32] = (unsigned)(m >> (tid & 32));
        }
    };
    auto fetch = [&](int s) {
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            const Task &k = tasks[i];
            if (!k.has) continue;
            const int64_t *const at = s_at[of_b][s & 1] + k.kg * kU;
            in[i] = s_rows_in[s & 1][k.kg / 4] >> 8 * (k.kg % 4) & 0xffu;
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                if (WIDE) l[i][u] = *reinterpret_cast<const uint4_any *>(k.from + at[u]);
                else l[i][u] = load_16<T, false>(k.from + at[u], width - ((of_b ? b0 : a0) + k.first));
            }
        }
    };
    auto stage = [&]() {
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            const Task &k = tasks[i];
            if (!k.has) continue;
            if (k.early > 0) {
#pragma unroll
                for (int r = 0; r < 8; ++r) settle<T>(l[i][r], k.early);
            }
            if (in[i] != 0xffu) {
#pragma unroll
                for (int r = 0; r < 8; ++r) l[i][r] = in[i] >> r & 1 ? l[i][r] : uint4_t{0, 0, 0, 0};
            }
            uint4_t u[CW][Q];
            to_units(l[i], u, of_b ? 1.f : sign);
#pragma unroll
            for (int j = 0; j < CW; ++j) {
                if (of_b) put<T, BN>(s_cols[k.part], KG, k.kg, place_full<T>(k.first + j), u[j]);
                else put<T, BM>(s_rows, KG, k.kg, place_full<T>(k.first + j), u[j]);
            }
        }
    };

    float16_t acc[TC][TR];
#pragma unroll
    for (int c = 0; c < TC; ++c)
#pragma unroll
        for (int r = 0; r < TR; ++r)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[c][r][i] = 0.f;
    if (steps > 0) {
        // operands a step ahead of the products, row ids two
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
            fetch_ids(s + 2);  // before the operands, whose loads then stay in flight when it is written
            fetch(s + 1);
#pragma unroll
            for (int e = 0; e < P; ++e) step_products<T, BN, BM, TC, TR>(acc, s_cols[e], s_rows, c0w, r0, sign);
            sign = -sign;
        }
    }
    const bool whole = t.end - t.start <= R.rows;
    const int64_t cells = (int64_t)q.A * B;
    const int64_t slot = 2 * (int64_t)R.of((int)t.start) + R.of((int)(t.p0 - t.start));
    T *const out = static_cast<T *>(q.out) + t.g * cells;
    float *const part = slots + (whole ? 0 : slot * cells);
#pragma unroll
    for (int r = 0; r < TR; ++r) {
        const int i = a0 + lane_of_full<T>(r0 + 32 * r + (lane & 31));
        if (i >= q.A) continue;
#pragma unroll
        for (int c = 0; c < TC; ++c)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const int col = b0 + vec_col_full<T>(c0w + 32 * c, v, half);
                const float4_t x = {acc[c][r][v], acc[c][r][4 + v], acc[c][r][8 + v], acc[c][r][12 + v]};
                if (q.transposed) {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (col + e < B) {
                            const int64_t at = (int64_t)(col + e) * q.A + i;
                            if (whole) out[at] = (T)x[e];
                            else part[at] = x[e];
                        }
                } else {
                    const int64_t at = (int64_t)i * B + col;
                    if (whole) store_four<false>(out + at, x, B - col);
                    else store_four<false>(part + at, x, B - col);
                }
            }
    }
    if constexpr (Q > 1 || NARROW) {
        float odd = 0.f;
#pragma unroll
        for (int c = 0; c < TC; ++c)
#pragma unroll
            for (int r = 0; r < TR; ++r) probe(odd, acc[c][r]);
        if (!__syncthreads_or(odd != odd)) return;
        // the sums that are not finite, in plain fp32 (bf16: an infinity times the parts of a narrow result may be NaN)
        stores_done();
        const int na = q.A - a0 < BM ? q.A - a0 : BM, nb = B - b0 < BN ? B - b0 : BN;
        for (int e = tid; e < na * nb; e += kThreads) {
            const int i = a0 + e / nb, c = b0 + e % nb;
            const int64_t at = q.transposed ? (int64_t)c * q.A + i : (int64_t)i * B + c;
            if (__builtin_isfinite(whole ? stored(out + at) : stored(part + at))) continue;
            float sum = 0.f;
            auto add = [&](int64_t pos) {  // no load waits for a branch
                const int row = row_at(o, pos), any = row < 0 ? 0 : row;
                const float y = NARROW ? narrow_at<T>(q.h, pos, W, c)
                                       : (float)static_cast<const T *>(q.b)[any * q.b_stride + c];
                const float x = (float)static_cast<const T *>(q.a)[any * q.a_stride + i];
                sum = row < 0 ? sum : fmaf(x, y, sum);
            };
            int64_t pos = t.p0;
            for (; pos + 8 <= t.p1 && sum == sum; pos += 8)  // NaN stays
#pragma unroll
                for (int u = 0; u < 8; ++u) add(pos + u);
            for (; pos < t.p1 && sum == sum; ++pos) add(pos);
            if (whole) out[at] = (T)sum;
            else part[at] = sum;
        }
    }
}

constexpr int kJoinCells = 128, kJoinLanes = 8;

// out_g = its slots' sum, for the groups of more than one chunk: a workgroup takes 128 cells, each thread
// four of them of every eighth slot, and the eight sums are then added in order. Where there are fewer
// groups than chunk sizes in the sequence, block x is for group x; else for the group whose first multiple
// of the chunk size beyond its start is x + 1 (each such group has one).
template <typename T, bool VEC>
__global__ __launch_bounds__(kThreads) void k_row_join(RowOrder o, ChunkRows R, bool by_group, int64_t cells,
                                                       const float *__restrict__ slots, T *__restrict__ out)
{
    __shared__ float4_t s_sum[kJoinLanes][kJoinCells / 4];
    const int64_t pos = ((int64_t)blockIdx.x + 1) * R.rows;
    int lo = 0, hi = o.G;
    if (by_group) lo = blockIdx.x;
    else
        while (lo < hi) {  // the group that holds pos
            const int mid = (lo + hi + 1) / 2;
            if (clamp_offset(o.offsets[mid], o.n) <= pos) lo = mid;
            else hi = mid - 1;
        }
    if (lo >= o.G) return;
    const int64_t start = clamp_offset(o.offsets[lo], o.n), end = clamp_offset(o.offsets[lo + 1], o.n);
    if (end - start <= R.rows) return;
    const int64_t chunks = R.of((int)(end - start - 1)) + 1, first = R.of((int)start);
    if (!by_group && first != blockIdx.x) return;
    const float *const src = slots + 2 * first * cells;
    const int quad = threadIdx.x % (kJoinCells / 4), lane = threadIdx.x / (kJoinCells / 4);
    for (int64_t c0 = (int64_t)blockIdx.y * kJoinCells; c0 < cells; c0 += (int64_t)gridDim.y * kJoinCells) {
        const int64_t i = c0 + 4 * quad, left = cells - i;
        auto slot = [&](int64_t c) {
            return __builtin_bit_cast(float4_t, load_16<float, VEC>(src + c * cells + i, left));
        };
        float4_t sum = {0.f, 0.f, 0.f, 0.f};
        int64_t c = lane;
        for (; c + 3 * kJoinLanes < chunks; c += 4 * kJoinLanes) {
            const float4_t v0 = slot(c), v1 = slot(c + kJoinLanes);
            const float4_t v2 = slot(c + 2 * kJoinLanes), v3 = slot(c + 3 * kJoinLanes);
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[e] += (v0[e] + v1[e]) + (v2[e] + v3[e]);
        }
        for (; c < chunks; c += kJoinLanes) {
            const float4_t v = slot(c);
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[e] += v[e];
        }
        __syncthreads();
        s_sum[lane][quad] = sum;
        __syncthreads();
        if (lane == 0) {
#pragma unroll
            for (int j = 1; j < kJoinLanes; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) sum[e] += s_sum[j][quad][e];
            store_four<VEC>(out + lo * cells + i, sum, left);
        }
    }
}

constexpr int kMinRows = 256, kMaxRows = 16384;  // of a chunk

struct Shape {
    int bm, bn, rows;  // of a chunk
    int64_t tiles;
};

// Rows of a chunk. Workgroups run in rounds of as many as the GPU holds at once, each as long as a chunk; the slots
// cost another 8 bytes a cell, half as much again as they have nothing beside them. Of sizes about 6% apart, the
// one with the least of both. An XCD is given whole chunks, and may have one more than the mean. Of all sizes,
// measured for twelve shapes (20,000 to 525,308 rows, 1 to 55 groups), this picks one within 4% of the best on the
// mean, 14% at worst; powers of two that leave two rounds were 13% off, 25% at worst.
int chunk_rows(size_t es, int64_t n, int G, const Shape &s)
{
    const int per_cu = es == 4 ? (s.bm == 128 && s.bn >= 64 ? 2 : 3) : s.bn == 128 ? 3 : 4;
    const double at_once = 256 * per_cu, groups = (double)(n < G ? n : G), mean = n / groups;
    int best = kMinRows;
    double least = 0;
    for (int r = kMinRows; r <= kMaxRows; r += r / 1024 * 64 + 64) {
        const bool split = mean > r;
        const double blocks = s.tiles * groups * (split ? mean / r + 0.5 : 1);
        const double cost = std::ceil((blocks + 8. * s.tiles) / at_once) * at_once * (split ? r : mean) * (s.bm + s.bn) * es +
                            (split ? blocks * s.bm * s.bn * 12 : 0);
        if (r == kMinRows || cost < least) best = r, least = cost;
        if (!split) break;
    }
    // whole groups: indices without a chunk, n / r of them, no more than a quarter as many as groups
    const int wide = mean < kMaxRows / 4 ? ((int)mean + 15) / 16 * 64 : kMaxRows;
    return best >= mean && wide > best ? wide : best;
}

Shape shape(size_t es, int64_t n, int G, int A, int B)
{
    Shape s;
    s.bm = A > 64 ? 128 : 64;
    s.bn = B > 64 ? 128 : B > 32 ? 64 : 32;
    if (s.bm == 64) s.bn = 64;
    s.tiles = (int64_t)((A + s.bm - 1) / s.bm) * ((B + s.bn - 1) / s.bn);
    s.rows = n > 0 ? chunk_rows(es, n, G, s) : kMinRows;
    return s;
}

template <typename T, int BM, int BN, int WR>
hipError_t launch(const RowOrder &o, const RowOuter &q, const Shape &sh, bool big, float *slots, hipStream_t s)
{
    const int B = q.r > 0 ? q.r : q.B;
    const bool wide = q.A >= kFull<T> && (q.r > 0 || B >= kFull<T>);  // 16 bytes of a row and more
    const int64_t chunks = ((big ? o.n / kFewRows : o.n / sh.rows + o.G) + 7) / 8 * 8;
    if (chunks * sh.tiles > 0x7fffffffLL) return hipErrorInvalidConfiguration;
    auto *kernel = wide ? k_row_outer<T, BM, BN, WR, true, false> : k_row_outer<T, BM, BN, WR, false, false>;
    if constexpr (BN <= CGTP_MAX_ADAPTER_RANK)
        if (q.r > 0) kernel = wide ? k_row_outer<T, BM, BN, WR, true, true> : k_row_outer<T, BM, BN, WR, false, true>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(chunks * sh.tiles)), dim3(kThreads), 0, s, o, q, ChunkRows(sh.rows), big,
                       slots);
    return hipGetLastError();
}

template <typename T> hipError_t run(const RowOrder &o, const RowOuter &q, float *slots, hipStream_t s)
{
    const int B = q.r > 0 ? q.r : q.B;
    const Shape sh = shape(sizeof(T), o.n, o.G, q.A, B);
    const bool big = o.n <= kFewMean * (int64_t)o.G;  // the groups of few rows go their own way
    hipError_t e;
    if (big) {
        e = launch_row_outer_few(sizeof(T) == 2 ? CGTP_BF16 : CGTP_F32, o, q, s);
        if (e != hipSuccess || o.n <= kFewRows) return e;
    }
    if (sh.bm == 64) e = launch<T, 64, 64, 2>(o, q, sh, big, slots, s);
    else if (sh.bn == 32) e = launch<T, 128, 32, 4>(o, q, sh, big, slots, s);
    else if (sh.bn == 64) e = launch<T, 128, 64, 4>(o, q, sh, big, slots, s);
    else e = launch<T, 128, 128, kWaveRows<T>>(o, q, sh, big, slots, s);
    if (e != hipSuccess || o.n <= sh.rows) return e;
    const int64_t cells = (int64_t)q.A * B, by = (cells + kJoinCells - 1) / kJoinCells;
    const int64_t spans = o.n / sh.rows, bx = o.G < spans ? o.G : spans;
    const int64_t y = 8192 / bx < 1 ? 1 : 8192 / bx;
    const bool vec = cells % 4 == 0 && aligned_rows<T>(q.out, 0);
    auto *kernel = vec ? k_row_join<T, true> : k_row_join<T, false>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)bx, (unsigned)(by < y ? by : y)), dim3(kThreads), 0, s, o, ChunkRows(sh.rows),
                       o.G < spans, cells, slots, static_cast<T *>(q.out));
    return hipGetLastError();
}

}  // namespace

size_t row_outer_bytes(int dtype, int64_t n, int G, int A, int B)
{
    const Shape sh = shape(dtype == CGTP_BF16 ? 2 : 4, n, G, A, B);
    return n <= sh.rows ? 0 : ((size_t)2 * (n / sh.rows) + 2) * A * B * sizeof(float);
}

hipError_t launch_row_outer(int dtype, const RowOrder &o, const RowOuter &q, void *ws, hipStream_t s)
{
    float *const slots = static_cast<float *>(ws);
    return dtype == CGTP_BF16 ? run<bf16_t>(o, q, slots, s) : run<float>(o, q, slots, s);
}

}  // namespace cgtp
