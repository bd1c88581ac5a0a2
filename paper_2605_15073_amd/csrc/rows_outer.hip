// Weight gradients of grouped rows, out_g = sum over the group's rows of a_i b_i^T, on the matrix
// cores: the products' k is the row, so both operands are transposed while they are staged.
//
// A workgroup owns one tile of the output and one chunk of a group's rows, 2^shift at most. A group
// of one chunk is written at once; the sums of a larger one go to the workspace, a slot per chunk,
// and a second kernel adds the slots in their order, so that the result does not depend on which
// workgroup came first. Slots: 2 (start >> shift) + j. A group of more than one chunk covers at least
// one multiple of the chunk size beyond its start, and 2 floor((s + m) / R) - 2 floor(s / R) >=
// ceil(m / R) for m > R, so slots of different groups never meet and 2 (n >> shift) + 2 suffice.
//
// With a narrow product's result as b, bf16 multiplies both of its parts into the same sums.
#include "internal.h"
#include "rows_tile.h"

namespace cgtp {

namespace {

using namespace rows;

template <typename T, int BM, int BN, int WR, bool VEC, bool NARROW>
__global__ __launch_bounds__(kThreads) void k_row_outer(RowOrder o, RowOuter q, int shift, float *slots)
{
    constexpr int KG = kGroups<T>, BK = kStep<T>, P = NARROW ? kNarrow<T> : 1, Q = kSplit<T>, CW = kWide<T>;
    constexpr int WC = 4 / WR, TR = BM / WR / 32, TC = BN / WC / 32;
    __shared__ uint4_t s_cols[P][kTile<T, BN>], s_rows[kTile<T, BM>];
    __shared__ int s_id[2][BK];

    // Block b runs on XCD b % 8: the tiles of a chunk, which share its rows, follow each other on one.
    const int B = NARROW ? q.r : q.B;
    const int btiles = (B + BN - 1) / BN, tiles = btiles * ((q.A + BM - 1) / BM);
    const int on_xcd = blockIdx.x / 8, tile = on_xcd % tiles;
    const int64_t chunk = (int64_t)(on_xcd / tiles) * 8 + blockIdx.x % 8;
    const Tile t = find_tile(o, shift, chunk);
    if (t.g < 0 || t.g >= o.G) return;
    const int W = narrow_width(B);
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int a0 = tile / btiles * BM, b0 = tile % btiles * BN;
    const int wr = wave % WR, wc = wave / WR;
    const int r0 = wr * (BM / WR), c0w = wc * (BN / WC);

    // lanes CW l .. CW l + CW - 1 of an operand, k-group g
    const int al = tid % (BM / CW), ag = tid / (BM / CW);
    const int bl = tid % (BN / CW), bg = tid / (BN / CW);
    uint2_t ar[8], br[P][8];
    bool lose = false;
    int id = -1;
    const int steps = (int)((t.p1 - t.p0 + BK - 1) / BK);
    auto fetch_ids = [&](int s) {
        const int64_t pos = t.p0 + (int64_t)s * BK + tid;
        id = tid < BK && pos < t.p1 ? row_at(o, pos) : -1;
    };
    auto fetch = [&](int s) {
        const int *const ids = s_id[s & 1];
        if (ag < KG) {
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const int row = ids[ag * kU + u];
                const int c = a0 + CW * al;
                ar[u] = load_8<T, VEC>(static_cast<const T *>(q.a) + (row < 0 ? 0 : row * q.a_stride) + c,
                                       row < 0 ? 0 : q.A - c);
            }
        }
        if (bg < KG) {
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const int row = ids[bg * kU + u];
                const int c = b0 + CW * bl;
                if (NARROW) {
                    const int64_t pos = t.p0 + (int64_t)s * BK + bg * kU + u;
#pragma unroll
                    for (int e = 0; e < P; ++e)
                        br[e][u] = load_8<T, true>(static_cast<const T *>(q.h) + (pos * P + e) * W + c,
                                                   row < 0 ? 0 : W - c);
                } else {
                    br[0][u] = load_8<T, VEC>(static_cast<const T *>(q.b) + (row < 0 ? 0 : row * q.b_stride) + c,
                                              row < 0 ? 0 : B - c);
                }
            }
        }
    };
    auto stage = [&]() {
        uint4_t u[CW][Q];
        if (ag < KG) {
            to_units(ar, u, lose);
#pragma unroll
            for (int j = 0; j < CW; ++j) put<T, BM>(s_rows, KG, ag, place<T>(CW * al + j), u[j]);
        }
        if (bg < KG) {
#pragma unroll
            for (int e = 0; e < P; ++e) {
                to_units(br[e], u, lose);
#pragma unroll
                for (int j = 0; j < CW; ++j) put<T, BN>(s_cols[e], KG, bg, place<T>(CW * bl + j), u[j]);
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
        // row ids two steps ahead of the products, operands one
        fetch_ids(0);
        if (tid < BK) s_id[0][tid] = id;
        fetch_ids(1);
        __syncthreads();
        fetch(0);
        for (int s = 0; s < steps; ++s) {
            __syncthreads();
            stage();
            if (tid < BK) s_id[(s + 1) & 1][tid] = id;
            __syncthreads();
            if (s + 1 < steps) {
                fetch(s + 1);
                fetch_ids(s + 2);
            }
#pragma unroll
            for (int e = 0; e < P; ++e) step_products<T, BN, BM, TC, TR>(acc, s_cols[e], s_rows, c0w, r0);
        }
    }
    const bool whole = t.end - t.start <= ((int64_t)1 << shift);
    const int64_t cells = (int64_t)q.A * B;
    const int64_t slot = 2 * (t.start >> shift) + ((t.p0 - t.start) >> shift);
    T *const out = static_cast<T *>(q.out) + t.g * cells;
    float *const part = slots + (whole ? 0 : slot * cells);
    if constexpr (Q > 1) {
        if (__syncthreads_or(lose)) {  // values outside the range of parts: plain fp32 sums
            const int na = q.A - a0 < BM ? q.A - a0 : BM, nb = B - b0 < BN ? B - b0 : BN;
            for (int e = tid; e < na * nb; e += kThreads) {
                const int i = a0 + e / nb, c = b0 + e % nb;
                float sum = 0.f;
                for (int64_t pos = t.p0; pos < t.p1; ++pos) {
                    const int row = row_at(o, pos);
                    if (row < 0) continue;
                    const float y = NARROW ? narrow_at<float>(q.h, pos, W, c)
                                           : static_cast<const float *>(q.b)[row * q.b_stride + c];
                    sum += static_cast<const float *>(q.a)[row * q.a_stride + i] * y;
                }
                const int64_t at = q.transposed ? (int64_t)c * q.A + i : (int64_t)i * B + c;
                if (whole) out[at] = (T)sum;
                else part[at] = sum;
            }
            return;
        }
    }
#pragma unroll
    for (int r = 0; r < TR; ++r) {
        const int i = a0 + lane_of<T>(r0 + 32 * r + (lane & 31));
        if (i >= q.A) continue;
#pragma unroll
        for (int c = 0; c < TC; ++c)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const int col = b0 + c0w + 32 * c + vec_col<T, true>(v, half);
                const float4_t x = vec_val<T, true>(acc[c][r], v);
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
                    if (whole) store_four<VEC>(out + at, x, B - col);
                    else store_four<VEC>(part + at, x, B - col);
                }
            }
    }
}

constexpr int kJoinCells = 32, kJoinLanes = kThreads / kJoinCells;

// out_g = its slots' sum, for the groups of more than one chunk: a workgroup takes 32 cells, 8 threads
// each with every eighth slot, whose sums are then added in order. Where there are fewer groups than
// chunk sizes in the sequence, block x is for group x; else for the group whose first multiple of the
// chunk size beyond its start is x + 1 (each such group has one).
template <typename T>
__global__ __launch_bounds__(kThreads) void k_row_join(RowOrder o, int shift, bool by_group, int64_t cells,
                                                       const float *__restrict__ slots, T *__restrict__ out)
{
    __shared__ float s_sum[kJoinLanes][kJoinCells];
    const int64_t pos = ((int64_t)blockIdx.x + 1) << shift;
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
    const int64_t chunks = (end - start + ((int64_t)1 << shift) - 1) >> shift;
    if (chunks < 2 || (!by_group && (start >> shift) + 1 != pos >> shift)) return;
    const float *const src = slots + 2 * (start >> shift) * cells;
    const int cell = threadIdx.x % kJoinCells, lane = threadIdx.x / kJoinCells;
    for (int64_t c0 = (int64_t)blockIdx.y * kJoinCells; c0 < cells; c0 += (int64_t)gridDim.y * kJoinCells) {
        const int64_t i = c0 + cell;
        float sum = 0.f;
        if (i < cells) {
            int64_t c = lane;
            for (; c + 3 * kJoinLanes < chunks; c += 4 * kJoinLanes) {
                const float v0 = src[c * cells + i], v1 = src[(c + kJoinLanes) * cells + i];
                const float v2 = src[(c + 2 * kJoinLanes) * cells + i], v3 = src[(c + 3 * kJoinLanes) * cells + i];
                sum += (v0 + v1) + (v2 + v3);
            }
            for (; c < chunks; c += kJoinLanes) sum += src[c * cells + i];
        }
        __syncthreads();
        s_sum[lane][cell] = sum;
        __syncthreads();
        if (lane == 0 && i < cells) {
#pragma unroll
            for (int j = 1; j < kJoinLanes; ++j) sum += s_sum[j][cell];
            out[lo * cells + i] = (T)sum;
        }
    }
}

constexpr int64_t kBlocks = 1536;  // workgroups that fill the GPU
constexpr int kMinShift = 8, kMaxShift = 14;

// Rows of a chunk: as many as leave kBlocks workgroups, but no fewer than keep the traffic of the
// slots (8 bytes a cell and chunk) at a quarter of the operands'.
int chunk_shift(size_t es, int64_t n, int A, int B, int64_t tiles)
{
    const int64_t fill = n * tiles / kBlocks;
    const int64_t least = (int64_t)(32.0 * A * B / ((double)(A + B) * es));
    int shift = kMinShift;
    while (shift < kMaxShift && (((int64_t)2 << shift) <= fill || ((int64_t)1 << shift) < least)) ++shift;
    return shift;
}

struct Shape {
    int bm, bn, shift;
    int64_t tiles;
};

Shape shape(size_t es, int64_t n, int A, int B)
{
    Shape s;
    s.bm = A > 64 ? 128 : 64;
    s.bn = B > 64 ? 128 : B > 32 ? 64 : 32;
    if (s.bm == 64) s.bn = 64;
    s.tiles = (int64_t)((A + s.bm - 1) / s.bm) * ((B + s.bn - 1) / s.bn);
    s.shift = chunk_shift(es, n, A, B, s.tiles);
    return s;
}

template <typename T, int BM, int BN, int WR>
hipError_t launch(const RowOrder &o, const RowOuter &q, const Shape &sh, float *slots, hipStream_t s)
{
    const int B = q.r > 0 ? q.r : q.B;
    constexpr int V = 16 / (int)sizeof(T);
    const bool vec = aligned_rows<T>(q.a, q.a_stride) && q.A % V == 0 && B % V == 0 &&
                     aligned_rows<T>(q.out, 0) && (q.r > 0 || aligned_rows<T>(q.b, q.b_stride));
    const int64_t chunks = ((o.n >> sh.shift) + o.G + 7) / 8 * 8;
    if (chunks * sh.tiles > 0x7fffffffLL) return hipErrorInvalidConfiguration;
    auto *kernel = q.r > 0 ? (vec ? k_row_outer<T, BM, BN, WR, true, true> : k_row_outer<T, BM, BN, WR, false, true>)
                           : (vec ? k_row_outer<T, BM, BN, WR, true, false> : k_row_outer<T, BM, BN, WR, false, false>);
    hipLaunchKernelGGL(kernel, dim3((unsigned)(chunks * sh.tiles)), dim3(kThreads), 0, s, o, q, sh.shift, slots);
    return hipGetLastError();
}

template <typename T> hipError_t run(const RowOrder &o, const RowOuter &q, float *slots, hipStream_t s)
{
    const int B = q.r > 0 ? q.r : q.B;
    const Shape sh = shape(sizeof(T), o.n, q.A, B);
    hipError_t e;
    if (sh.bm == 64) e = launch<T, 64, 64, 2>(o, q, sh, slots, s);
    else if (sh.bn == 32) e = launch<T, 128, 32, 4>(o, q, sh, slots, s);
    else if (sh.bn == 64) e = launch<T, 128, 64, 4>(o, q, sh, slots, s);
    else e = launch<T, 128, 128, 2>(o, q, sh, slots, s);
    if (e != hipSuccess || o.n >> sh.shift == 0) return e;
    const int64_t cells = (int64_t)q.A * B, by = (cells + kJoinCells - 1) / kJoinCells;
    const int64_t spans = o.n >> sh.shift, bx = o.G < spans ? o.G : spans;
    const int64_t y = 8192 / bx < 1 ? 1 : 8192 / bx;
    hipLaunchKernelGGL(k_row_join<T>, dim3((unsigned)bx, (unsigned)(by < y ? by : y)), dim3(kThreads), 0, s, o,
                       sh.shift, o.G < spans, cells, slots, static_cast<T *>(q.out));
    return hipGetLastError();
}

}  // namespace

size_t row_outer_bytes(int dtype, int64_t n, int G, int A, int B)
{
    const Shape sh = shape(dtype == CGTP_BF16 ? 2 : 4, n, A, B);
    return n >> sh.shift == 0 ? 0 : ((size_t)2 * (n >> sh.shift) + 2) * A * B * sizeof(float);
}

hipError_t launch_row_outer(int dtype, const RowOrder &o, const RowOuter &q, void *ws, hipStream_t s)
{
    float *const slots = static_cast<float *>(ws);
    return dtype == CGTP_BF16 ? run<bf16_t>(o, q, slots, s) : run<float>(o, q, slots, s);
}

}  // namespace cgtp
