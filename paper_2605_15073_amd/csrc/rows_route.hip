// Rows to experts (cgtp_route_rows): scores, the choice of the largest keys, and the weights; and its gradient.
//
// L lanes of a wave share a row; lane l has the experts l + L j, j < PER, in registers. Keys that are sums or blocks'
// scores are formed in 64 bits: two that differ by less than fp32's rounding are still told apart, so that the choice
// is the formula's. Without a bias and blocks the logits themselves are compared. The choice takes the largest key k
// times: each lane its own, then the lanes of the row, the lowest expert among equals.
#include <type_traits>

#include "internal.h"
#include "rows_layer.h"

namespace cgtp {

namespace {

using namespace rows;

constexpr int kWaves = kThreads / 64;

// Orders a wave's LDS writes before its other lanes' reads.
__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

template <int L> __device__ __forceinline__ float row_max(float v)
{
#pragma unroll
    for (int d = 1; d < L; d *= 2) v = fmaxf(v, __shfl_xor(v, d));
    return v;
}
template <int L, typename F> __device__ __forceinline__ F row_sum(F v)
{
#pragma unroll
    for (int d = 1; d < L; d *= 2) v += __shfl_xor(v, d);
    return v;
}

// A logit of -inf, or NaN, is of an expert that the row may not have.
__device__ __forceinline__ bool there(float l) { return l > -__builtin_inff(); }

// KEYS: keys are scores with a bias or of blocks, in 64 bits; else the logits.
template <typename T, int L, int PER, bool KEYS>
__global__ __launch_bounds__(kThreads) void k_route(RowRoute p)
{
    typedef typename std::conditional<KEYS, double, float>::type Key;
    constexpr int R = 64 / L;  // rows of a wave
    constexpr float kNone = -__builtin_inff();
    extern __shared__ __align__(16) char sh[];
    __shared__ int s_ids[kWaves][R][CGTP_MAX_TOP_K];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l = lane % L, r = lane / L;
    int64_t row = (tile_at(blockIdx.x, blockIdx.z, gridDim.x) * kWaves + wave) * R + r;
    const bool stores = row < p.n;
    if (!stores) row = p.n - 1;
    const T *const from = static_cast<const T *>(p.logits) + row * p.stride;
    float x[PER];
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        const int e = l + L * j;
        x[j] = e < p.E ? (float)from[e] : kNone;
    }
    float top = kNone;
    bool odd = false;  // NaN or +inf among the logits
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        top = fmaxf(top, there(x[j]) ? x[j] : kNone);
        odd |= !(x[j] < __builtin_inff());
    }
    top = row_max<L>(top);
    Key key[PER];
    if constexpr (KEYS) {
        if (p.score == CGTP_SCORE_SOFTMAX) {
            double sum = 0;
#pragma unroll
            for (int j = 0; j < PER; ++j) {
                key[j] = there(x[j]) ? exp((double)x[j] - (double)top) : 0.0;
                sum += key[j];
            }
            sum = row_sum<L>(sum);
#pragma unroll
            for (int j = 0; j < PER; ++j) key[j] /= sum;
        } else {
#pragma unroll
            for (int j = 0; j < PER; ++j) key[j] = 1.0 / (1.0 + exp(-(double)x[j]));
        }
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            const int e = l + L * j;
            if (p.bias && e < p.E) key[j] += (double)p.bias[e];
            if (!there(x[j]) || !(key[j] > (double)kNone)) key[j] = (double)kNone;
        }
        if (p.blocks > 1) {
            // keys of the row, then scores of its blocks
            const int size = p.E / p.blocks;
            double *const keys = reinterpret_cast<double *>(sh) + (int64_t)(wave * R + r) * (p.E + p.blocks);
            double *const scores = keys + p.E;
#pragma unroll
            for (int j = 0; j < PER; ++j)
                if (l + L * j < p.E) keys[l + L * j] = key[j];
            wave_sync();
            for (int b = l; b < p.blocks; b += L) {
                double first = (double)kNone, second = first;
                for (int i = 0; i < size; ++i) {
                    const double v = keys[b * size + i];
                    second = v > first ? first : v > second ? v : second;
                    first = v > first ? v : first;
                }
                scores[b] = second > (double)kNone ? first + second : first;
            }
            wave_sync();
#pragma unroll
            for (int j = 0; j < PER; ++j) {
                const int e = l + L * j;
                if (e >= p.E) continue;
                const int b = e / size;
                const double own = scores[b];
                int ahead = 0;
                for (int i = 0; i < p.blocks; ++i) ahead += scores[i] > own || (scores[i] == own && i < b);
                if (ahead >= p.keep) key[j] = (double)kNone;
            }
        }
    } else {
#pragma unroll
        for (int j = 0; j < PER; ++j) key[j] = there(x[j]) ? x[j] : kNone;
    }
    for (int i = 0; i < p.k; ++i) {
        Key best = key[0];
        int at = l;
#pragma unroll
        for (int j = 1; j < PER; ++j)
            if (key[j] > best) {
                best = key[j];
                at = l + L * j;
            }
#pragma unroll
        for (int d = 1; d < L; d *= 2) {
            const Key other = __shfl_xor(best, d);
            const int e = __shfl_xor(at, d);
            if (other > best || (other == best && e < at)) {
                best = other;
                at = e;
            }
        }
        const bool found = best > (Key)kNone;
        if (l == 0) s_ids[wave][r][i] = found ? at : -1;
#pragma unroll
        for (int j = 0; j < PER; ++j)
            if (found && at == l + L * j) key[j] = (Key)kNone;
    }
    wave_sync();
    // weights. Renormalised ones are formed relative to the largest of the chosen.
    float sum = 0.f, shift = top;
    const bool soft = p.score == CGTP_SCORE_SOFTMAX;
    if (p.renorm) {
        shift = kNone;
        for (int i = l; i < p.k; i += L) {
            const int e = s_ids[wave][r][i];
            if (e >= 0) shift = fmaxf(shift, soft ? (float)from[e] : fminf((float)from[e], 0.f));
        }
        shift = row_max<L>(shift);
    } else if (soft) {
#pragma unroll
        for (int j = 0; j < PER; ++j) sum += there(x[j]) ? expf(x[j] - top) : 0.f;
        sum = row_sum<L>(sum);
    } else {
        shift = 0.f;
    }
    auto part = [&](int e) {
        const float v = (float)from[e];
        return soft ? expf(v - shift) : expf(fminf(v, 0.f) - shift) / (1.f + expf(-fabsf(v)));
    };
    if (p.renorm) {
        for (int i = l; i < p.k; i += L) {
            const int e = s_ids[wave][r][i];
            if (e >= 0) sum += part(e);
        }
        sum = row_sum<L>(sum);
    } else if (!soft) {
        sum = 1.f;
    }
    unsigned long long any = __ballot(odd);
    if (L < 64) any = any >> (lane / L * L) & ((1ull << (L % 64)) - 1);
    if (!stores) return;
    for (int i = l; i < p.k; i += L) {
        const int e = s_ids[wave][r][i];
        p.ids[row * p.k + i] = e;
        float w = e >= 0 ? part(e) / sum * p.scale : 0.f;
        if (soft && any) w = __builtin_nanf("");
        p.weights[row * p.k + i] = w;
    }
}

// dl of the chosen and, for softmax without renormalising, of all experts.
template <typename T, int L, int PER>
__global__ __launch_bounds__(kThreads) void k_route_grad(RowRoute p)
{
    constexpr int R = 64 / L;
    constexpr float kNone = -__builtin_inff();
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l = lane % L, r = lane / L;
    int64_t row = (tile_at(blockIdx.x, blockIdx.z, gridDim.x) * kWaves + wave) * R + r;
    const bool stores = row < p.n;
    if (!stores) row = p.n - 1;
    const T *const from = static_cast<const T *>(p.logits) + row * p.stride;
    const int32_t *const ids = p.ids + row * p.k;
    const float *const u = p.dweights + row * p.k;
    const bool soft = p.score == CGTP_SCORE_SOFTMAX;
    auto chosen = [&](int i) { return (unsigned)ids[i] < (unsigned)p.E && there((float)from[ids[i]]); };
    float x[PER], dl[PER];
    float shift = kNone, sum = 0.f;
    if (soft && !p.renorm) {
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            const int e = l + L * j;
            x[j] = e < p.E ? (float)from[e] : kNone;
            shift = fmaxf(shift, there(x[j]) ? x[j] : kNone);
        }
        shift = row_max<L>(shift);
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            x[j] = there(x[j]) ? expf(x[j] - shift) : x[j] == kNone ? 0.f : x[j];  // NaN stays
            sum += x[j];
        }
        sum = row_sum<L>(sum);
        sum = sum == 0.f ? 1.f : sum;
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            x[j] /= sum;
            dl[j] = 0.f;
        }
    } else {
#pragma unroll
        for (int j = 0; j < PER; ++j) dl[j] = 0.f;
        if (p.renorm) {
            for (int i = l; i < p.k; i += L)
                if (chosen(i)) shift = fmaxf(shift, soft ? (float)from[ids[i]] : fminf((float)from[ids[i]], 0.f));
            shift = row_max<L>(shift);
        } else {
            shift = 0.f;
        }
    }
    auto part = [&](int e) {
        const float v = (float)from[e];
        return soft ? expf(v - shift) : expf(fminf(v, 0.f) - shift) / (1.f + expf(-fabsf(v)));
    };
    if (p.renorm) {
        for (int i = l; i < p.k; i += L)
            if (chosen(i)) sum += part(ids[i]);
        sum = row_sum<L>(sum);
        sum = sum == 0.f ? 1.f : sum;
    } else if (!soft) {
        sum = 1.f;
    }
    // the mean of u over the shares
    float mean = 0.f;
    if (soft || p.renorm) {
        for (int i = l; i < p.k; i += L)
            if (chosen(i)) mean += u[i] * (part(ids[i]) / sum);
        mean = row_sum<L>(mean);
    }
    for (int i = 0; i < p.k; ++i) {
        if (!chosen(i)) continue;
        const int e = ids[i];
        const float share = part(e) / sum, v = (float)from[e];
        float g = share * (p.renorm ? u[i] - mean : u[i]);
        if (!soft) g *= 1.f / (1.f + expf(v));  // 1 - s
#pragma unroll
        for (int j = 0; j < PER; ++j)
            if (e == l + L * j) dl[j] += g;
    }
    if (!stores) return;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        const int e = l + L * j;
        if (e >= p.E) continue;
        float g = dl[j];
        if (soft && !p.renorm) g -= x[j] * mean;
        static_cast<T *>(p.dlogits)[row * p.dstride + e] = (T)(p.scale * g);
    }
}

template <typename T, int L, int PER> hipError_t launch(const RowRoute &p, bool gradient, hipStream_t s)
{
    constexpr int rows = kWaves * (64 / L);
    const TileGrid grid = tile_grid((p.n + rows - 1) / rows);
    const dim3 blocks(grid.x, 1, grid.z);
    if (gradient) {
        hipLaunchKernelGGL((k_route_grad<T, L, PER>), blocks, dim3(kThreads), 0, s, p);
        return hipGetLastError();
    }
    const bool keys = p.bias || p.blocks > 1;
    const size_t lds = p.blocks > 1 ? sizeof(double) * rows * (p.E + p.blocks) : 0;
    auto *kernel = keys ? k_route<T, L, PER, true> : k_route<T, L, PER, false>;
    hipLaunchKernelGGL(kernel, blocks, dim3(kThreads), lds, s, p);
    return hipGetLastError();
}

template <typename T> hipError_t pick(const RowRoute &p, bool gradient, hipStream_t s)
{
    if (p.E <= 8) return launch<T, 8, 1>(p, gradient, s);
    if (p.E <= 32) return launch<T, 8, 4>(p, gradient, s);
    if (p.E <= 128) return launch<T, 16, 8>(p, gradient, s);
    if (p.E <= 512) return launch<T, 64, 8>(p, gradient, s);
    return launch<T, 64, 64>(p, gradient, s);
}

}  // namespace

hipError_t launch_route_rows(int dtype, const RowRoute &p, hipStream_t s)
{
    return dtype == CGTP_BF16 ? pick<bf16_t>(p, false, s) : pick<float>(p, false, s);
}

hipError_t launch_route_rows_grad(int dtype, const RowRoute &p, hipStream_t s)
{
    return dtype == CGTP_BF16 ? pick<bf16_t>(p, true, s) : pick<float>(p, true, s);
}

}  // namespace cgtp
