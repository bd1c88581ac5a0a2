// Row order by group (cgtp_group_rows): a stable counting sort of the group ids.
//
// Chunks of consecutive rows count their ids, a scan over the chunks turns the counts into the
// position of each chunk's first row of each group, and the chunks then place their rows. Within
// a workgroup every wave owns consecutive rows; a row's rank among the 64 that the wave handles
// together comes from ballots over the bits of the id, so no atomic decides an order. Rows whose
// id is outside [0, G) form a group G of their own, placed last.
//
// Up to kSmall rows one workgroup does all of it in one launch.
#include "internal.h"
#include "rows.h"

namespace cgtp {

namespace {

constexpr int kThreads = 512;
constexpr int kWaves = kThreads / 64;
constexpr int kSmall = 4096;   // rows of the one-launch form
constexpr int kChunks = 64;    // chunks at most: a wave scans one lane per chunk
constexpr int kMinChunk = 2048;

struct Shape {
    int chunks, rows;  // rows per chunk, a multiple of 64 * kWaves
};

Shape shape(int64_t n)
{
    int64_t rows = (n + kChunks - 1) / kChunks;
    if (rows < kMinChunk) rows = kMinChunk;
    rows = (rows + kThreads - 1) / kThreads * kThreads;
    return {(int)((n + rows - 1) / rows), (int)rows};
}

__device__ __forceinline__ int key_of(int id, int G) { return (unsigned)id < (unsigned)G ? id : G; }

// counts[key][chunk]
__global__ __launch_bounds__(kThreads) void k_group_count(int64_t n, int G, int rows, int chunks,
                                                          const int32_t *__restrict__ ids,
                                                          int32_t *__restrict__ counts)
{
    extern __shared__ int sh[];
    for (int g = threadIdx.x; g <= G; g += kThreads) sh[g] = 0;
    __syncthreads();
    const int64_t r0 = (int64_t)blockIdx.x * rows, r1 = r0 + rows < n ? r0 + rows : n;
    for (int64_t r = r0 + threadIdx.x; r < r1; r += kThreads) atomicAdd(&sh[key_of(ids[r], G)], 1);
    __syncthreads();
    for (int g = threadIdx.x; g <= G; g += kThreads)
        counts[(int64_t)g * chunks + blockIdx.x] = sh[g];
}

// In place: the rows of the key in the chunks before; totals[key].
__global__ __launch_bounds__(256) void k_group_scan(int G, int chunks, int32_t *__restrict__ counts,
                                                    int32_t *__restrict__ totals)
{
    const int g = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (g > G) return;
    const int c = lane < chunks ? counts[(int64_t)g * chunks + lane] : 0;
    int sum = c;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int up = __shfl_up(sum, d);
        if (lane >= d) sum += up;
    }
    if (lane < chunks) counts[(int64_t)g * chunks + lane] = sum - c;
    if (lane == 63) totals[g] = sum;
}

// LDS: base[G + 1] (int), the position of the chunk's first row of each key, then
// run[kWaves][G + 1], the rows of each key that the waves before, then this one, have placed.
__global__ __launch_bounds__(kThreads) void k_group_place(
    int64_t n, int G, int rows, int chunks, const int32_t *__restrict__ ids,
    const int32_t *__restrict__ counts, const int32_t *__restrict__ totals,
    int32_t *__restrict__ offsets, int32_t *__restrict__ order)
{
    extern __shared__ int sh[];
    __shared__ int wave_sum[kWaves];
    int *const base = sh;
    int *const run = sh + G + 1;  // [kWaves][G + 1]
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t r0 = (int64_t)blockIdx.x * rows, r1 = r0 + rows < n ? r0 + rows : n;
    const int per = rows / kWaves;  // rows of a wave, consecutive, a multiple of 64
    const int64_t w0 = r0 + (int64_t)wave * per;
    const int64_t w1 = w0 + per < r1 ? w0 + per : r1;
    for (int i = tid; i < kWaves * (G + 1); i += kThreads) run[i] = 0;
    __syncthreads();
    int *const mine = run + wave * (G + 1);
    for (int64_t r = w0 + lane; r < w1; r += 64) atomicAdd(&mine[key_of(ids[r], G)], 1);
    __syncthreads();
    // totals of the keys (of this workgroup where there is one chunk), then their exclusive scan
    for (int g = tid; g <= G; g += kThreads) {
        int t = 0;
        for (int w = 0; w < kWaves; ++w) {
            const int c = run[w * (G + 1) + g];
            run[w * (G + 1) + g] = t;
            t += c;
        }
        base[g] = totals ? totals[g] : t;
    }
    __syncthreads();
    const int span = (G + 1 + kThreads - 1) / kThreads;
    int first = tid * span, last = first + span;
    if (first > G + 1) first = G + 1;
    if (last > G + 1) last = G + 1;
    int sum = 0;
    for (int g = first; g < last; ++g) sum += base[g];
    int scan = sum;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int up = __shfl_up(scan, d);
        if (lane >= d) scan += up;
    }
    if (lane == 63) wave_sum[wave] = scan;
    __syncthreads();
    int at = scan - sum;
    for (int w = 0; w < wave; ++w) at += wave_sum[w];
    for (int g = first; g < last; ++g) {
        const int t = base[g];
        base[g] = at + (counts ? counts[(int64_t)g * chunks + blockIdx.x] : 0);
        if (blockIdx.x == 0) offsets[g] = at;
        at += t;
    }
    __syncthreads();
    if (n == 0) return;
    int bits = 1;
    while ((G >> bits) != 0) ++bits;
    for (int64_t b = w0; b < w1; b += 64) {
        const int64_t r = b + lane;
        const bool in = r < w1;
        const int key = in ? key_of(ids[r], G) : 0;
        unsigned long long same = __ballot(in);
        for (int k = 0; k < bits; ++k) {
            const unsigned long long set = __ballot((key >> k) & 1);
            same &= ((key >> k) & 1) ? set : ~set;
        }
        if (in) {
            const unsigned long long below = same & ((1ull << lane) - 1);
            const int rank = __popcll(below);
            const int before = mine[key];
            order[base[key] + before + rank] = (int)r;
            // the first of the rows that share a key moves its count on, once all have read it
            __builtin_amdgcn_wave_barrier();
            if (below == 0) mine[key] = before + __popcll(same);
        }
        __builtin_amdgcn_wave_barrier();
    }
}

}  // namespace

size_t group_rows_bytes(int64_t n, int G)
{
    if (n <= kSmall) return 0;
    return 4 * ((size_t)(G + 1) * shape(n).chunks + (size_t)(G + 1));
}

hipError_t launch_group_rows(int64_t n, int G, const int32_t *ids, int32_t *offsets, int32_t *order,
                             void *ws, hipStream_t s)
{
    const size_t place_lds = 4 * (size_t)(kWaves + 1) * (G + 1);
    static_assert(4 * (kWaves + 1) * (CGTP_MAX_GROUPS + 1) + 1024 <= 160 * 1024, "LDS");
    if (n <= kSmall) {
        hipLaunchKernelGGL(k_group_place, dim3(1), dim3(kThreads), place_lds, s, n, G, kSmall, 1,
                           ids, nullptr, nullptr, offsets, order);
        return hipGetLastError();
    }
    const Shape sh = shape(n);
    int32_t *const counts = static_cast<int32_t *>(ws);
    int32_t *const totals = counts + (size_t)(G + 1) * sh.chunks;
    hipLaunchKernelGGL(k_group_count, dim3(sh.chunks), dim3(kThreads), 4 * (size_t)(G + 1), s, n, G,
                       sh.rows, sh.chunks, ids, counts);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(k_group_scan, dim3((G + 1 + 3) / 4), dim3(256), 0, s, G, sh.chunks, counts,
                       totals);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(k_group_place, dim3(sh.chunks), dim3(kThreads), place_lds, s, n, G, sh.rows,
                       sh.chunks, ids, counts, totals, offsets, order);
    return hipGetLastError();
}

}  // namespace cgtp
