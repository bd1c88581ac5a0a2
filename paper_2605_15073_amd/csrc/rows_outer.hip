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
#include "rows_layer.h"

#include <cmath>

namespace cgtp {

namespace {

using namespace rows;

// Sums of b's columns, from the loads of its values: of the tiles that hold the first columns of a. The eight rows of a
// load are added first, so that a long sum takes an eighth of the additions.
__device__ __forceinline__ void add_columns(float (&sum)[8], const uint4_t (&in)[8], bf16_t)
{
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        sum[2 * e] += sum_of_eight([&](int r) { return __builtin_bit_cast(float, in[r][e] << 16); });
        sum[2 * e + 1] += sum_of_eight([&](int r) { return __builtin_bit_cast(float, in[r][e] & 0xffff0000u); });
    }
}
__device__ __forceinline__ void add_columns(float (&sum)[4], const uint4_t (&in)[8], float)
{
#pragma unroll
    for (int e = 0; e < 4; ++e) sum[e] += sum_of_eight([&](int r) { return __builtin_bit_cast(float, (unsigned)in[r][e]); });
}

enum Dz { kNoDz, kFormDz, kHeldDz };

// LAYER: rows of a are shared (per), and the columns of b are summed beside the products (sums). b's rows may be layers' dz
// in two bf16 parts (rows_layer.h), which meet the same a: kHeldDz, as they lie, like a narrow product's; kFormDz, from dy
// and z as they are loaded. That takes registers for both and for their parts, so that there all waves stage both
// operands, 8 bytes of eight rows a thread, a row's slopes at a time: 261,764 rows, 128 x 448, 200 us and the join's 17. Waves
// wait three fifths of their time: for loads (470 MB of dy and z) and each other; the vector ALU is busy for half of it, the
// matrix cores for a seventh. Columns summed from the parts behind the slopes, not between them: 262,144 rows, 64 x 448, 145 and 200.
template <typename T, int BM, int BN, int WR, bool WIDE, bool NARROW, bool LAYER, Dz DZ_>
__global__ __launch_bounds__(kThreads, DZ_ == kNoDz ? 1 : DZ_ == kFormDz ? 3 : 4) void k_row_outer(RowOrder o, RowOuter q, ChunkRows R, bool big,
                                                        float *slots)
{
    constexpr bool DZ = DZ_ == kFormDz, HELD = DZ_ == kHeldDz;
    constexpr int KG = kGroups<T>, BK = kStep<T>, P = NARROW ? kNarrow<T> : DZ || HELD ? 2 : 1, Q = kSplit<T>, CW = DZ ? 4 : kFull<T>;
    constexpr int WC = 4 / WR, TR = BM / WR / 32, TC = BN / WC / 32;
    static_assert(DZ_ == kNoDz || (LAYER && !NARROW && sizeof(T) == 2), "dz in parts: layers in bf16");
    typedef typename std::conditional<DZ, float, T>::type Places;  // of loads of CW lanes: fp32's for four
    __shared__ uint4_t s_cols[P][kTile<T, BN>], s_rows[kTile<T, BM>];
    __shared__ int64_t s_at[DZ ? 3 : 2][2][BK];  // where the rows of a, b and slope_z of a step start
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
    constexpr int kHalf = kThreads / 2, kPart = KG * (BN / CW), NL = DZ ? 1 : (P * kPart + kHalf - 1) / kHalf;
    static_assert(KG * (BM / CW) <= (DZ ? kThreads : kHalf) && (!DZ || kPart <= kThreads), "a, and b of DZ: one task a thread");
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
                 ((k.has ? k.part : 0) * (NARROW ? W : HELD ? B : 0) + (WIDE && col + CW > width ? width - CW : col));
    }
    // DZ: a task of a for the first threads, one of b for the last, without a branch inside a wave
    const int task_a = tid, task_b = tid - (kThreads - kPart);
    const bool has_a = DZ && task_a < KG * (BM / CW), has_b = DZ && task_b >= 0;
    const int kg_a = task_a / (BM / CW) % KG, first_a = CW * (task_a % (BM / CW));
    const int kg_b = has_b ? task_b / (BN / CW) : 0, first_b = has_b ? CW * (task_b % (BN / CW)) : 0;
    auto start4 = [&](int col, int width) { return WIDE && col + CW > width ? width - CW : col; };
    auto early4 = [&](int col, int width) { return WIDE && col < width && col + CW > width ? col + CW - width : 0; };
    uint2_t la[DZ ? 8 : 1], lb[DZ ? 8 : 1], lz[DZ ? 8 : 1];
    unsigned in_a = 0, in_b = 0;
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
            const int of_a = LAYER && q.per > 1 ? (int)((unsigned)row / (unsigned)q.per) : row;
            s_at[0][s & 1][tid] = in ? of_a * q.a_stride : 0;  // row 0 in place of none: zeroed when staged
            s_at[1][s & 1][tid] = !in ? 0 : NARROW ? pos * (P * W) : row * q.b_stride;
            if constexpr (DZ) s_at[2][s & 1][tid] = in ? row * q.slope_stride : 0;
            const unsigned long long m = __ballot(in);
            if (tid % 32 == 0) s_rows_in[s & 1][tid / 32] = (unsigned)(m >> (tid & 32));
        }
    };
    auto load4 = [&](uint2_t (&to)[DZ ? 8 : 1], const void *from, const int64_t *at, int col, int width) __attribute__((always_inline)) {
        const T *const p = static_cast<const T *>(from) + start4(col, width);
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            if (WIDE) to[u] = *reinterpret_cast<const uint2_any *>(p + at[u]);
            else to[u] = load_8<T, false>(p + at[u], width - col);
        }
    };
    auto fetch = [&](int s) {
        if constexpr (DZ) {
            if (has_a) {
                in_a = s_rows_in[s & 1][kg_a / 4] >> 8 * (kg_a % 4) & 0xffu;
                load4(la, q.a, s_at[0][s & 1] + kg_a * kU, a0 + first_a, q.A);
            }
            if (has_b) {
                in_b = s_rows_in[s & 1][kg_b / 4] >> 8 * (kg_b % 4) & 0xffu;
                load4(lb, q.b, s_at[1][s & 1] + kg_b * kU, b0 + first_b, B);
                load4(lz, q.slope_z, s_at[2][s & 1] + kg_b * kU, b0 + first_b, B);
            }
            return;
        }
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
    const bool sums = LAYER && q.sums && (DZ || of_b) && a0 == 0;
    float column[LAYER ? CW : 1];
#pragma unroll
    for (int j = 0; j < (LAYER ? CW : 1); ++j) column[j] = 0.f;
    auto stage = [&]() {
        if constexpr (DZ) {
            uint4_t u[CW][Q];
            if (has_a) {
                const int early = early4(a0 + first_a, q.A);
                if (early > 0) {
#pragma unroll
                    for (int r = 0; r < 8; ++r) settle<T>(la[r], early);
                }
                if (in_a != 0xffu) {
#pragma unroll
                    for (int r = 0; r < 8; ++r) la[r] = in_a >> r & 1 ? la[r] : uint2_t{0, 0};
                }
                to_units(la, u);
#pragma unroll
                for (int j = 0; j < CW; ++j) put<T, BM>(s_rows, KG, kg_a, place_full<Places>(first_a + j), u[j]);
            }
            if (has_b) {
                const int early = early4(b0 + first_b, B);
                if (early > 0) {
#pragma unroll
                    for (int r = 0; r < 8; ++r) {
                        settle<T>(lb[r], early);
                        settle<T>(lz[r], early);
                    }
                }
                if (in_b != 0xffu) {  // 0 act'(0)
#pragma unroll
                    for (int r = 0; r < 8; ++r) {
                        lb[r] = in_b >> r & 1 ? lb[r] : uint2_t{0, 0};
                        lz[r] = in_b >> r & 1 ? lz[r] : uint2_t{0, 0};
                    }
                }
                // the parts in place of what they are formed from, a row at a time: its registers are free for the next
#pragma unroll
                for (int r = 0; r < 8; ++r)
                    with_act(q.act, [&](auto act) __attribute__((always_inline)) {
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            unsigned high, low;
                            dz_pair<decltype(act)::value>(lb[r][k], lz[r][k], high, low);
                            lb[r][k] = high;
                            lz[r][k] = low;
                        }
                    });
                if (sums) {  // of the parts; an infinity or NaN is the first alone
                    auto value = [](unsigned high, unsigned low) {
                        const float h = __builtin_bit_cast(float, high);
                        return __builtin_isfinite(h) ? h + __builtin_bit_cast(float, low) : h;
                    };
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        column[2 * k] += sum_of_eight([&](int r) { return value(lb[r][k] << 16, lz[r][k] << 16); });
                        column[2 * k + 1] +=
                            sum_of_eight([&](int r) { return value(lb[r][k] & 0xffff0000u, lz[r][k] & 0xffff0000u); });
                    }
                }
                to_units(lb, u);
#pragma unroll
                for (int j = 0; j < CW; ++j) put<T, BN>(s_cols[0], KG, kg_b, place_full<Places>(first_b + j), u[j]);
                to_units(lz, u);
#pragma unroll
                for (int j = 0; j < CW; ++j) put<T, BN>(s_cols[P - 1], KG, kg_b, place_full<Places>(first_b + j), u[j]);
            }
            return;
        }
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
            if constexpr (LAYER && !DZ)
                if (sums) add_columns(column, l[i], T());
            uint4_t u[CW][Q];
            if constexpr (!DZ) to_units(l[i], u, of_b ? 1.f : sign);  // DZ is staged above
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
    const int64_t cells = (int64_t)q.A * B, slot_cells = cells + (LAYER && q.sums ? B : 0);
    const int64_t slot = 2 * (int64_t)R.of((int)t.start) + R.of((int)(t.p0 - t.start));
    T *const out = static_cast<T *>(q.out) + t.g * cells;
    float *const part = slots + (whole ? 0 : slot * slot_cells);
    if constexpr (LAYER) {
        // parts of b that threads of their own load, each with sums of its own
        constexpr int SP = NL == 1 ? P : 1, sp = DZ ? 1 : SP;
        static_assert(NL <= 2 && sizeof(s_rows) >= sizeof(float) * sp * KG * BN, "one task a thread, or both parts of it");
        if (q.sums && a0 == 0) {
            float *const of_kg = reinterpret_cast<float *>(s_rows);  // [sp][KG][BN]
            __syncthreads();
            if (DZ ? has_b : of_b && tasks[0].has)
#pragma unroll
                for (int j = 0; j < CW; ++j) of_kg[DZ ? kg_b * BN + first_b + j : (tasks[0].part * KG + tasks[0].kg) * BN + tasks[0].first + j] = column[j];
            __syncthreads();
            if (tid < BN && b0 + tid < B) {
                float sum = 0.f;
#pragma unroll
                for (int g = 0; g < sp * KG; ++g) sum += of_kg[g * BN + tid];
                if (whole) static_cast<T *>(q.sums)[(int64_t)t.g * B + b0 + tid] = (T)sum;
                else part[cells + b0 + tid] = sum;
            }
        }
    }
    if (LAYER && !q.out) return;  // the sums alone
#pragma unroll
    for (int r = 0; r < TR; ++r) {
        const int i = a0 + lane_of_full<Places>(r0 + 32 * r + (lane & 31));
        if (i >= q.A) continue;
#pragma unroll
        for (int c = 0; c < TC; ++c)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const int col = b0 + vec_col_full<Places>(c0w + 32 * c, v, half);
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
    if constexpr (Q > 1 || NARROW || DZ_ != kNoDz) {
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
                float y;
                if constexpr (NARROW) y = narrow_at<T>(q.h, pos, W, c);
                else y = (float)static_cast<const T *>(q.b)[any * q.b_stride + c];
                if constexpr (DZ_ != kNoDz)
                    y = dz_value(y, (float)static_cast<const T *>(q.slope_z)[any * q.slope_stride + c], q.act);
                const int of_a = LAYER && q.per > 1 ? (int)((unsigned)any / (unsigned)q.per) : any;
                const float x = (float)static_cast<const T *>(q.a)[of_a * q.a_stride + i];
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
// Cells from `split` on are those of a second output.
template <typename T, bool VEC>
__global__ __launch_bounds__(kThreads) void k_row_join(RowOrder o, ChunkRows R, bool by_group, int64_t cells, int64_t split,
                                                       const float *__restrict__ slots, T *__restrict__ out,
                                                       T *__restrict__ rest)
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
            if (!out) {
                for (int e = 0; e < 4 && e < left; ++e)
                    if (i + e >= split) rest[lo * (cells - split) + (i + e - split)] = (T)sum[e];
            } else if (i + 4 <= split || split == cells) store_four<VEC>(out + lo * split + i, sum, split - i);
            else if (i >= split) store_four<VEC>(rest + lo * (cells - split) + (i - split), sum, left);
            else
                for (int e = 0; e < 4 && e < left; ++e) {
                    if (i + e < split) out[lo * split + i + e] = (T)sum[e];
                    else rest[lo * (cells - split) + (i + e - split)] = (T)sum[e];
                }
        }
    }
}

constexpr int kMinRows = 256, kMaxRows = 16384;  // of a chunk

struct Shape {
    int bm, bn, rows;  // of a chunk
    int per_cu;        // workgroups on a compute unit
    int64_t tiles;
};

// Rows of a chunk. Workgroups run in rounds of as many as the GPU holds at once, each as long as a chunk; the slots
// cost another 8 bytes a cell, half as much again as they have nothing beside them. Of sizes about 6% apart, the
// one with the least of both. An XCD is given whole chunks, and may have one more than the mean. Of all sizes,
// measured for twelve shapes (20,000 to 525,308 rows, 1 to 55 groups), this picks one within 4% of the best on the
// mean, 14% at worst; powers of two that leave two rounds were 13% off, 25% at worst.
int chunk_rows(size_t es, int64_t n, int G, const Shape &s)
{
    const double at_once = 256 * s.per_cu, groups = (double)(n < G ? n : G), mean = n / groups;
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

// dz in parts: 64 columns, whose sums leave registers for both. Us with 128 of them and 64: formed, 261,764 rows, 128 x 448,
// 230 (two workgroups on a compute unit) and 229, 20,000 of 100 groups, 128 x 128, 25 and 22; held, 60,000, 1344 x 448, 304
// and 302, 6,000 of 20 groups 64 and 56. With three and four workgroups on a compute unit: the first 217 and 247, the third
// 300 and 286.
Shape shape(size_t es, int64_t n, int G, int A, int B, bool parts)
{
    Shape s;
    s.bm = A > 64 ? 128 : 64;
    s.bn = B > 64 ? (parts ? 64 : 128) : B > 32 ? 64 : 32;
    if (s.bm == 64) s.bn = 64;
    const bool large = s.bm == 128 && s.bn >= 64;
    s.per_cu = es == 4 ? (large ? 2 : 3) : large && (s.bn == 128 || (parts && A <= 128)) ? 3 : 4;  // formed up to 128
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
    auto *kernel = wide ? k_row_outer<T, BM, BN, WR, true, false, false, kNoDz>
                        : k_row_outer<T, BM, BN, WR, false, false, false, kNoDz>;
    if (q.per > 0)
        kernel = wide ? k_row_outer<T, BM, BN, WR, true, false, true, kNoDz> : k_row_outer<T, BM, BN, WR, false, false, true, kNoDz>;
    if constexpr (sizeof(T) == 2 && BN <= 64)
        if (q.slope_z)
            kernel = q.act == kDzHeld
                         ? (wide ? k_row_outer<T, BM, BN, WR, true, false, true, kHeldDz> : k_row_outer<T, BM, BN, WR, false, false, true, kHeldDz>)
                         : (wide ? k_row_outer<T, BM, BN, WR, true, false, true, kFormDz> : k_row_outer<T, BM, BN, WR, false, false, true, kFormDz>);
    if constexpr (BN <= CGTP_MAX_ADAPTER_RANK)
        if (q.r > 0)
            kernel = wide ? k_row_outer<T, BM, BN, WR, true, true, false, kNoDz> : k_row_outer<T, BM, BN, WR, false, true, false, kNoDz>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(chunks * sh.tiles)), dim3(kThreads), 0, s, o, q, ChunkRows(sh.rows), big,
                       slots);
    return hipGetLastError();
}

template <typename T>
hipError_t join(const RowOrder &o, int chunk, int A, int B, const float *slots, void *out, void *sums, hipStream_t s)
{
    const int64_t split = (int64_t)A * B, cells = split + (sums ? B : 0), by = (cells + kJoinCells - 1) / kJoinCells;
    const int64_t spans = o.n / chunk, bx = o.G < spans ? o.G : spans;
    const int64_t y = 8192 / bx < 1 ? 1 : 8192 / bx;
    const bool vec = split % 4 == 0 && aligned_rows<T>(out, 0) && (!sums || (B % 4 == 0 && aligned_rows<T>(sums, 0)));
    auto *kernel = vec ? k_row_join<T, true> : k_row_join<T, false>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)bx, (unsigned)(by < y ? by : y)), dim3(kThreads), 0, s, o, ChunkRows(chunk),
                       o.G < spans, cells, split, slots, static_cast<T *>(out), static_cast<T *>(sums));
    return hipGetLastError();
}

template <typename T> hipError_t run(const RowOrder &o, const RowOuter &q, float *slots, hipStream_t s)
{
    const int B = q.r > 0 ? q.r : q.B;
    const Shape sh = shape(sizeof(T), o.n, o.G, q.A, B, q.slope_z != nullptr);
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
    return join<T>(o, sh.rows, q.A, B, slots, q.out, q.sums, s);
}

}  // namespace

size_t row_outer_bytes(int dtype, int64_t n, int G, int A, int B, bool sums, bool parts)
{
    const Shape sh = shape(dtype == CGTP_BF16 ? 2 : 4, n, G, A, B, parts);
    return n <= sh.rows ? 0 : ((size_t)2 * (n / sh.rows) + 2) * (A + sums) * B * sizeof(float);
}

hipError_t launch_row_join(int dtype, const RowOrder &o, int chunk_rows, int A, int B, const float *slots, void *out,
                           void *sums, hipStream_t s)
{
    return dtype == CGTP_BF16 ? join<bf16_t>(o, chunk_rows, A, B, slots, out, sums, s)
                              : join<float>(o, chunk_rows, A, B, slots, out, sums, s);
}

hipError_t launch_row_outer(int dtype, const RowOrder &o, const RowOuter &q, void *ws, hipStream_t s)
{
    float *const slots = static_cast<float *>(ws);
    return dtype == CGTP_BF16 ? run<bf16_t>(o, q, slots, s) : run<float>(o, q, slots, s);
}

}  // namespace cgtp
