// Row order by group (cgtp_group_rows): a stable counting sort of the group ids.
//
// Chunks of consecutive rows count their ids, a scan over the chunks turns the counts into the
// position of each chunk's first row of each group, and the chunks then place their rows. A workgroup
// takes its chunk in rounds of kRound rows, whose ids it holds in registers, four to a thread, so that
// counting and placing wait for memory once; every wave owns consecutive rows of a round. A row's rank among
// the 64 that a wave handles together comes from ballots over the bits of the id: no atomic decides an
// order. Rows whose id is outside [0, G) form a group G of their own, placed last.
//
// Up to kRound rows one workgroup does all of it in one launch. Bound by latency: the chains of three
// launches, and in each of memory, LDS and barriers. Measured: 525,308 rows of 4,005 groups 26 us (counting
// 6.3, scan 4.5, placing 15.7; 1.5 of it for stores to scattered places), of 5 groups 17, 64 rows 9 us (the kernel 4.9).
// 512 threads of eight ids took 27 us; ranks from atomic adds, with ballots only where keys meet, 27.
#include "internal.h"
#include "rows.h"

namespace cgtp {

namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / 64;
constexpr int kPer = 4;                       // ids of a thread
constexpr int kRound = kThreads * kPer;       // rows of a round
constexpr int kChunks = 256;                  // chunks at most
constexpr int kScanKeys = 64, kScanSlices = 16;
constexpr int kWordsEach = ((CGTP_MAX_GROUPS + 2) / 2 + kThreads - 1) / kThreads;  // words of two keys of a thread

// Words of two of the G + 1 keys, in whole 16 bytes.
__host__ __device__ constexpr int word_stride(int G) { return ((G + 2) / 2 + 3) / 4 * 4; }

struct Shape {
    int chunks, rounds;  // rounds of a chunk
};

Shape shape(int64_t n)
{
    const int64_t all = (n + kRound - 1) / kRound, rounds = (all + kChunks - 1) / kChunks;
    return {(int)((all + rounds - 1) / rounds), (int)rounds};
}

__device__ __forceinline__ int key_of(int id, int G) { return (unsigned)id < (unsigned)G ? id : G; }

// The keys of this thread's rows of the round that starts at r0: rows r0 + wave kPer 64 + 64 i + lane; -1 past n.
__device__ __forceinline__ void load_keys(int (&key)[kPer], int64_t r0, int64_t n, int G, const int32_t *ids)
{
    const int64_t r = r0 + (threadIdx.x >> 6) * (kPer * 64) + (threadIdx.x & 63);
#pragma unroll
    for (int i = 0; i < kPer; ++i) key[i] = ids[r + 64 * i < n ? r + 64 * i : 0];
#pragma unroll
    for (int i = 0; i < kPer; ++i) key[i] = r + 64 * i < n ? key_of(key[i], G) : -1;
}

// counts[chunk][key]
__global__ __launch_bounds__(kThreads) void k_group_count(int64_t n, int G, int rounds,
                                                          const int32_t *__restrict__ ids,
                                                          int32_t *__restrict__ counts)
{
    extern __shared__ int sh[];
    int key[kPer];
    const int64_t r0 = (int64_t)blockIdx.x * rounds * kRound;
    load_keys(key, r0, n, G, ids);
    for (int g = threadIdx.x; g <= G; g += kThreads) sh[g] = 0;
    __syncthreads();
    for (int round = 0;;) {
#pragma unroll
        for (int i = 0; i < kPer; ++i)
            if (key[i] >= 0) atomicAdd(&sh[key[i]], 1);
        if (++round == rounds) break;
        load_keys(key, r0 + (int64_t)round * kRound, n, G, ids);
    }
    __syncthreads();
    for (int g = threadIdx.x; g <= G; g += kThreads) counts[(int64_t)blockIdx.x * (G + 1) + g] = sh[g];
}

// In place: the rows of the key in the chunks before; totals[key]. A workgroup takes 64 keys, a wave of it a slice
// of the chunks, whose counts it holds in registers: one trip to memory.
__global__ __launch_bounds__(kScanKeys *kScanSlices) void k_group_scan(int G, int chunks,
                                                                       int32_t *__restrict__ counts,
                                                                       int32_t *__restrict__ totals)
{
    constexpr int kMost = kChunks / kScanSlices;
    __shared__ int s_sum[kScanSlices][kScanKeys];
    const int k = threadIdx.x % kScanKeys, slice = threadIdx.x / kScanKeys;
    const int g = blockIdx.x * kScanKeys + k;
    const int per = (chunks + kScanSlices - 1) / kScanSlices;
    const int c0 = slice * per, own = chunks - c0 < per ? chunks - c0 : per;
    int v[kMost], sum = 0;
#pragma unroll
    for (int i = 0; i < kMost; ++i) v[i] = g <= G ? counts[(int64_t)(i < own ? c0 + i : 0) * (G + 1) + g] : 0;
#pragma unroll
    for (int i = 0; i < kMost; ++i) sum += i < own ? v[i] : 0;
    s_sum[slice][k] = sum;
    __syncthreads();
    if (g > G) return;
    int before = 0;
    for (int s = 0; s < slice; ++s) before += s_sum[s][k];
    if (slice == kScanSlices - 1) totals[g] = before + sum;
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
        if (i >= own) break;
        counts[(int64_t)(c0 + i) * (G + 1) + g] = before;
        before += v[i];
    }
}

// Counts of a wave fit 16 bits (a round's are kRound at most), so a word holds those of two keys: it is scanned
// over the waves as one. Word w = tid + kThreads j, keys 2 w and 2 w + 1, is this thread's throughout; its loads
// of totals and counts are on their way while the round is counted.
//
// LDS: base[2 words], the position of the round's first row of each key, then run[kWaves][words], the rows of
// each key that the waves before, then this one, have placed in the round.
__global__ __launch_bounds__(kThreads) void k_group_place(
    int64_t n, int G, int rounds, const int32_t *__restrict__ ids, const int32_t *__restrict__ counts,
    const int32_t *__restrict__ totals, int32_t *__restrict__ offsets, int32_t *__restrict__ order)
{
    extern __shared__ __align__(16) int sh[];
    __shared__ int wave_sum[64];
    static_assert(kWordsEach * kWaves <= 64, "one wave scans the sums");
    const int words = (G + 2) / 2, stride = word_stride(G);
    int *const base = sh;
    unsigned *const run = reinterpret_cast<unsigned *>(sh + 2 * stride);
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t r0 = (int64_t)blockIdx.x * rounds * kRound;
    unsigned *const mine = run + wave * stride;
    int key[kPer];
    if (n > 0) load_keys(key, r0, n, G, ids);
    int total[kWordsEach][2], count[kWordsEach][2];
#pragma unroll
    for (int j = 0; j < kWordsEach; ++j)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int g = 2 * (tid + kThreads * j) + h;
            total[j][h] = totals && g <= G ? totals[g] : 0;
            count[j][h] = counts && g <= G ? counts[(int64_t)blockIdx.x * (G + 1) + g] : 0;
        }
    int bits = 1;
    while ((G >> bits) != 0) ++bits;
    for (int round = 0; round < rounds; ++round) {
        for (int i = tid; i < kWaves * stride / 4; i += kThreads) reinterpret_cast<uint4 *>(run)[i] = uint4{0, 0, 0, 0};
        __syncthreads();
        if (n > 0) {
#pragma unroll
            for (int i = 0; i < kPer; ++i)
                if (key[i] >= 0) atomicAdd(&mine[key[i] >> 1], 1u << (16 * (key[i] & 1)));
        }
        __syncthreads();
        // each wave's first place among the round's rows of a key
        unsigned in_round[kWordsEach];
#pragma unroll
        for (int j = 0; j < kWordsEach; ++j) {
            const int w = tid + kThreads * j;
            unsigned t = 0;
            if (w < words) {
#pragma unroll
                for (int v = 0; v < kWaves; ++v) {
                    const unsigned c = run[v * stride + w];
                    run[v * stride + w] = t;
                    t += c;
                }
            }
            in_round[j] = t;
        }
        if (round == 0) {
            // the keys' first positions: the exclusive scan of their totals (the round's own where there is
            // one chunk), j by j, in each over the threads
            int sum[kWordsEach], scan[kWordsEach];
#pragma unroll
            for (int j = 0; j < kWordsEach; ++j) {
                if (!totals) total[j][0] = in_round[j] & 0xffff, total[j][1] = in_round[j] >> 16;
                scan[j] = sum[j] = total[j][0] + total[j][1];
#pragma unroll
                for (int d = 1; d < 64; d *= 2) {
                    const int up = __shfl_up(scan[j], d);
                    if (lane >= d) scan[j] += up;
                }
                if (lane == 63) wave_sum[j * kWaves + wave] = scan[j];
            }
            __syncthreads();
            if (wave == 0) {
                const int own = lane < kWordsEach * kWaves ? wave_sum[lane] : 0;
                int at = own;
#pragma unroll
                for (int d = 1; d < 64; d *= 2) {
                    const int up = __shfl_up(at, d);
                    if (lane >= d) at += up;
                }
                wave_sum[lane] = at - own;
            }
            __syncthreads();
#pragma unroll
            for (int j = 0; j < kWordsEach; ++j) {
                const int w = tid + kThreads * j;
                if (w >= words) break;
                int at = wave_sum[j * kWaves + wave] + scan[j] - sum[j];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    if (blockIdx.x == 0 && 2 * w + h <= G) offsets[2 * w + h] = at;
                    base[2 * w + h] = at + count[j][h];
                    at += total[j][h];
                }
            }
        }
        __syncthreads();
        if (n == 0) return;
        const int64_t r = r0 + (int64_t)round * kRound + wave * (kPer * 64) + lane;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const bool in = key[i] >= 0;
            const int k = in ? key[i] : 0;
            unsigned long long same = __ballot(in);
            for (int b = 0; b < bits; ++b) {
                const unsigned long long set = __ballot((k >> b) & 1);
                same &= ((k >> b) & 1) ? set : ~set;
            }
            const unsigned long long below = same & ((1ull << lane) - 1);
            if (in) order[base[k] + (int)(mine[k >> 1] >> (16 * (k & 1)) & 0xffff) + __popcll(below)] = (int)(r + 64 * i);
            // the first of the rows that share a key moves its count on, once all have read it
            __builtin_amdgcn_wave_barrier();
            if (in && below == 0) atomicAdd(&mine[k >> 1], (unsigned)__popcll(same) << (16 * (k & 1)));
            __builtin_amdgcn_wave_barrier();
        }
        if (round + 1 == rounds) break;
        load_keys(key, r0 + (int64_t)(round + 1) * kRound, n, G, ids);
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kWordsEach; ++j) {
            const int w = tid + kThreads * j;
            if (w >= words) break;
            base[2 * w] += in_round[j] & 0xffff;
            base[2 * w + 1] += in_round[j] >> 16;
        }
    }
}

}  // namespace

size_t group_rows_bytes(int64_t n, int G)
{
    if (n <= kRound) return 0;
    return 4 * ((size_t)(G + 1) * shape(n).chunks + (size_t)(G + 1));
}

hipError_t launch_group_rows(int64_t n, int G, const int32_t *ids, int32_t *offsets, int32_t *order,
                             void *ws, hipStream_t s)
{
    const size_t place_lds = 4 * (size_t)(kWaves + 2) * word_stride(G);
    static_assert(4 * (kWaves + 2) * word_stride(CGTP_MAX_GROUPS) + 1024 <= 160 * 1024, "LDS");
    if (n <= kRound) {
        hipLaunchKernelGGL(k_group_place, dim3(1), dim3(kThreads), place_lds, s, n, G, 1, ids, nullptr,
                           nullptr, offsets, order);
        return hipGetLastError();
    }
    const Shape sh = shape(n);
    int32_t *const counts = static_cast<int32_t *>(ws);
    int32_t *const totals = counts + (size_t)(G + 1) * sh.chunks;
    hipLaunchKernelGGL(k_group_count, dim3(sh.chunks), dim3(kThreads), 4 * (size_t)(G + 1), s, n, G,
                       sh.rounds, ids, counts);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(k_group_scan, dim3((G + kScanKeys) / kScanKeys), dim3(kScanKeys * kScanSlices), 0, s,
                       G, sh.chunks, counts, totals);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(k_group_place, dim3(sh.chunks), dim3(kThreads), place_lds, s, n, G, sh.rounds, ids,
                       counts, totals, offsets, order);
    return hipGetLastError();
}

}  // namespace cgtp
