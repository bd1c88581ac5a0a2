// Rows to experts (cgtp_route_rows): scores, the choice of the largest keys, and the weights; and its gradient.
//
// L lanes of a wave share a row; lane l has the experts l PER .. l PER + PER - 1 in registers. The choice takes the
// largest key k times: each lane its own, then the lanes of the row, the lowest expert among equals. Without a bias and
// blocks the keys are the logits. Else they are formed in fp32 first, and again in 64 bits by the waves that hold a row
// in which two keys, or blocks' scores, that decide are nearer than fp32's error: the choice is then the formula's.
#include <type_traits>

#include "internal.h"
#include "rows_layer.h"

namespace cgtp {

namespace {

using namespace rows;

constexpr int kWaves = kThreads / 64;
template <int E> constexpr int kMost = E < CGTP_MAX_TOP_K ? E : CGTP_MAX_TOP_K;  // chosen of a row of up to E
// LDS of a wave's rows: keys and blocks' scores, in 64 bits or (the row 4 longer) in 32.
__host__ __device__ constexpr int wave_bytes(int rows, int keys, int blocks) { return rows * (8 * (keys + blocks) + 16); }

// Orders a wave's LDS writes before its other lanes' reads.
__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// A logit of -inf, or NaN, is of an expert that the row may not have.
__device__ __forceinline__ bool there(float l) { return l > -__builtin_inff(); }

// Logits first .. first + PER - 1 of a row of E, -inf past its end.
template <typename T, int PER> __device__ __forceinline__ void load_logits(float (&x)[PER], const T *from, int first, int E)
{
    constexpr int V = 16 / (int)sizeof(T);
    static_assert(PER % V == 0, "whole vectors");
#pragma unroll
    for (int v = 0; v < PER; v += V) {
        const uint4_t u = load_16<T, false>(from + first + v, E - (first + v));
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const float f = sizeof(T) == 4 ? __builtin_bit_cast(float, (unsigned)u[e % 4])
                                           : __builtin_bit_cast(float, e % 2 ? u[e / 2 % 4] & 0xffff0000u : u[e / 2 % 4] << 16);
            x[v + e] = first + v + e < E ? f : -__builtin_inff();
        }
    }
}

// The value of the lane that differs in the bits of D, D < 16: no trip through LDS.
template <int D> __device__ __forceinline__ int other_lane(int v)
{
    constexpr int ctrl = D == 1 ? 0xb1 : D == 2 ? 0x4e : D == 4 ? 0x141 : 0x140;  // quads, half a row and a row mirrored
    return __builtin_amdgcn_update_dpp(v, v, ctrl, 0xf, 0xf, false);
}
template <int D> __device__ __forceinline__ float other(float v)
{
    if constexpr (D < 16) return __builtin_bit_cast(float, other_lane<D>(__builtin_bit_cast(int, v)));
    else return __shfl_xor(v, D);
}
template <int D> __device__ __forceinline__ double other(double v)
{
    if constexpr (D < 16) {
        const int2 w = __builtin_bit_cast(int2, v);
        return __builtin_bit_cast(double, int2{other_lane<D>(w.x), other_lane<D>(w.y)});
    } else return __shfl_xor(v, D);
}

// Over the L lanes of a row; a mirrored half serves as the other one, as its lanes agree by then.
template <int L, typename F, int D = 1> __device__ __forceinline__ F row_max(F v)
{
    if constexpr (D < L) {
        const F o = other<D>(v);
        return row_max<L, F, 2 * D>(o > v ? o : v);
    } else return v;
}
template <int L, typename F, int D = 1> __device__ __forceinline__ F row_sum(F v)
{
    if constexpr (D < L) return row_sum<L, F, 2 * D>(v + other<D>(v));
    else return v;
}

__device__ __forceinline__ float exponential(float x) { return __expf(x); }
__device__ __forceinline__ double exponential(double x) { return exp(x); }
__device__ __forceinline__ float inverse(float x) { return __builtin_amdgcn_rcpf(x); }
__device__ __forceinline__ double inverse(double x) { return 1.0 / x; }

// How far a key in fp32 may be off. s = 1 / (1 + e), and s times a share of at most one: their exponentials are off by
// 2^-24 (2 + 2.5 |a|) of themselves, a the argument: a score by 2.9 2^-24 of the largest from its own, where s |a| is
// below 0.37 of that; by 23 from a sum of 512, where the mean of |a| is below log 512 + 2; by 14 more from its
// additions, 8 of a lane and 6 over lanes, and by 3 from reciprocal and product. The bias adds the rounding of the key.
constexpr float kOffScore = 48 * 0x1p-24f, kOffKey = 0x1p-23f;

// The choice, experts in s_ids. Key float: false where keys in fp32 do not settle it (the caller then takes 64 bits).
template <int L, int PER, bool KEYS, typename Key>
__device__ __forceinline__ bool choose(const RowRoute &p, const float (&x)[PER], float top, int l, Key *row_keys, int *ids)
{
    constexpr Key kNone = -(Key)__builtin_inff();
    constexpr bool kExact = sizeof(Key) == 8 || !KEYS;
    Key key[PER];
    Key most = 1;  // the largest score
    if constexpr (KEYS) {
        if (p.score == CGTP_SCORE_SOFTMAX) {
            Key sum = 0;
#pragma unroll
            for (int j = 0; j < PER; ++j) {
                key[j] = there(x[j]) ? exponential((Key)x[j] - (Key)top) : (Key)0;
                sum += key[j];
            }
            most = inverse(row_sum<L>(sum));
#pragma unroll
            for (int j = 0; j < PER; ++j) key[j] *= most;
        } else {
#pragma unroll
            for (int j = 0; j < PER; ++j) key[j] = inverse((Key)1 + exponential(-(Key)x[j]));
        }
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            const int e = l * PER + j;
            if (p.bias) key[j] += (Key)p.bias[e < p.E ? e : 0];
            if (!there(x[j]) || !(key[j] > kNone)) key[j] = kNone;
        }
    } else {
#pragma unroll
        for (int j = 0; j < PER; ++j) key[j] = there(x[j]) ? x[j] : kNone;
    }
    bool sure = true;
    if (KEYS && p.blocks > 1) {
        // keys of the row, then scores of its blocks; those left out lose their keys
        const int size = p.E / p.blocks;
        Key *const scores = row_keys + L * PER;
#pragma unroll
        for (int j = 0; j < PER; ++j) row_keys[l * PER + j] = key[j];
        wave_sync();
        for (int b = l; b < p.blocks; b += L) {
            Key first = kNone, second = kNone;
            for (int i = 0; i < size; ++i) {
                const Key v = row_keys[b * size + i];
                const Key low = v > first ? first : v;
                first = v > first ? v : first;
                second = low > second ? low : second;
            }
            scores[b] = second > kNone ? first + second : first;
        }
        wave_sync();
        for (int b = l; b < p.blocks; b += L) {
            const Key own = scores[b];
            int ahead = 0, perhaps = 0;
            for (int i = 0; i < p.blocks; ++i) {
                const Key v = scores[i];
                if constexpr (kExact) {
                    ahead += v > own || (v == own && i < b);
                } else {
                    const Key off = 4 * (kOffScore * most + kOffKey * (fabsf(own) + fabsf(v)));
                    ahead += v > own + off;
                    perhaps += i != b && v > own - off;
                    if (v == own && i != b && own > kNone) ++perhaps;  // infinite ones
                }
            }
            const bool out = ahead >= p.keep;
            if (!kExact && !out && perhaps >= p.keep && own > kNone) sure = false;
            if (out)
                for (int i = 0; i < size; ++i) row_keys[b * size + i] = kNone;
        }
        wave_sync();
#pragma unroll
        for (int j = 0; j < PER; ++j) key[j] = row_keys[l * PER + j];
    }
    Key before = -kNone;
    const int lane = threadIdx.x & 63, first = lane / L * L;
    // one more round where the last chosen has to be told from the next
    for (int i = 0; i < p.k + !kExact; ++i) {
        Key own = key[0];
#pragma unroll
        for (int j = 1; j < PER; ++j) own = key[j] > own ? key[j] : own;
        const Key best = row_max<L>(own);
        if constexpr (!kExact) {
            const Key off = 2 * (kOffScore * most + kOffKey * (fabsf(best) + fabsf(before)));
            if (best > kNone && !(best < before - off) && i > 0) sure = false;
            before = best;
            if (i == p.k) break;
        }
        int winner = l;
        if constexpr (L > 1) {
            const unsigned long long same = __ballot(own == best) >> first;
            winner = __ffsll((unsigned long long)same) - 1;  // the lowest of the row: others' bits lie above
        }
        if (l == winner) {
            int at = -1;
#pragma unroll
            for (int j = PER - 1; j >= 0; --j) at = key[j] == best ? j : at;
#pragma unroll
            for (int j = 0; j < PER; ++j) key[j] = j == at ? kNone : key[j];
            ids[i] = best > kNone ? l * PER + at : -1;
        }
    }
    return sure;
}

// KEYS: keys are scores with a bias or of blocks; else the logits.
template <typename T, int L, int PER, bool KEYS>
__global__ __launch_bounds__(kThreads) void k_route(RowRoute p)
{
    constexpr int R = 64 / L;  // rows of a wave
    constexpr float kNone = -__builtin_inff();
    extern __shared__ __align__(16) char sh[];
    __shared__ int s_ids[kWaves][R][kMost<L * PER>];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l = lane % L, r = lane / L;
    int64_t row = (tile_at(blockIdx.x, blockIdx.z, gridDim.x) * kWaves + wave) * R + r;
    const bool stores = row < p.n;
    if (!stores) row = p.n - 1;
    const T *const from = static_cast<const T *>(p.logits) + row * p.stride;
    float x[PER];
    load_logits(x, from, l * PER, p.E);
    float top = kNone;
    bool odd = false;  // NaN or +inf among the logits
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        top = fmaxf(top, there(x[j]) ? x[j] : kNone);
        odd |= !(x[j] < __builtin_inff());
    }
    top = row_max<L>(top);
    int *const ids = s_ids[wave][r];
    char *const mine = sh + wave * wave_bytes(R, L * PER, p.blocks);
    double *const keys = reinterpret_cast<double *>(mine) + r * (L * PER + p.blocks);
    if constexpr (!KEYS) choose<L, PER, false, float>(p, x, top, l, nullptr, ids);
    else if constexpr (PER > 8) choose<L, PER, true, double>(p, x, top, l, keys, ids);
    else {
        float *const near = reinterpret_cast<float *>(mine) + r * (L * PER + p.blocks + 4);
        const bool sure = choose<L, PER, true, float>(p, x, top, l, near, ids);
        if (__any(!sure)) {
            wave_sync();
            choose<L, PER, true, double>(p, x, top, l, keys, ids);
        }
    }
    wave_sync();
    // weights. Renormalised ones are formed relative to the largest of the chosen.
    float sum = 0.f, shift = top;
    const bool soft = p.score == CGTP_SCORE_SOFTMAX;
    if (p.renorm) {
        shift = kNone;
        for (int i = l; i < p.k; i += L) {
            const int e = ids[i];
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
        for (int i = l; i < p.k; i += L)
            if (ids[i] >= 0) sum += part(ids[i]);
        sum = row_sum<L>(sum);
    } else if (!soft) {
        sum = 1.f;
    }
    unsigned long long any = __ballot(odd);
    if (L < 64) any = any >> (lane / L * L) & ((1ull << (L % 64)) - 1);
    if (!stores) return;
    for (int i = l; i < p.k; i += L) {
        const int e = ids[i];
        p.ids[row * p.k + i] = e;
        float w = e >= 0 ? part(e) / sum * p.scale : 0.f;
        if (soft && any) w = __builtin_nanf("");
        p.weights[row * p.k + i] = w;
    }
}

// dl of the chosen and, for softmax without renormalising, of all experts. The lanes of a row form the parts of its
// chosen experts, one each, and pass them through LDS to the lanes that hold those.
template <typename T, int L, int PER>
__global__ __launch_bounds__(kThreads) void k_route_grad(RowRoute p)
{
    constexpr int R = 64 / L, M = kMost<L * PER>, NI = (M + L - 1) / L;
    constexpr float kNone = -__builtin_inff();
    __shared__ int s_e[kWaves][R][M];
    __shared__ float s_g[kWaves][R][M];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l = lane % L, r = lane / L;
    int64_t row = (tile_at(blockIdx.x, blockIdx.z, gridDim.x) * kWaves + wave) * R + r;
    const bool stores = row < p.n;
    if (!stores) row = p.n - 1;
    const T *const from = static_cast<const T *>(p.logits) + row * p.stride;
    const bool soft = p.score == CGTP_SCORE_SOFTMAX, whole = soft && !p.renorm;
    float x[PER], dl[PER], v[NI], u[NI];
    // chosen l + L i
#pragma unroll
    for (int i = 0; i < NI; ++i) {
        const int c = l + L * i;
        if (c >= p.k) break;
        const int e = p.ids[row * p.k + c];
        u[i] = p.dweights[row * p.k + c];
        v[i] = (unsigned)e < (unsigned)p.E ? (float)from[e] : kNone;
        s_e[wave][r][c] = there(v[i]) ? e : -1;
    }
    float shift = kNone, sum = 0.f;
    if (whole) {
        load_logits(x, from, l * PER, p.E);
#pragma unroll
        for (int j = 0; j < PER; ++j) shift = fmaxf(shift, there(x[j]) ? x[j] : kNone);
        shift = row_max<L>(shift);
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            x[j] = there(x[j]) ? expf(x[j] - shift) : x[j] == kNone ? 0.f : x[j];  // NaN stays
            sum += x[j];
        }
        sum = row_sum<L>(sum);
    } else if (p.renorm) {
#pragma unroll
        for (int i = 0; i < NI; ++i)
            if (l + L * i < p.k && there(v[i])) shift = fmaxf(shift, soft ? v[i] : fminf(v[i], 0.f));
        shift = row_max<L>(shift);
    } else {
        shift = 0.f;
    }
    // shares of the chosen, in v, and 1 - s beside them
    float rest[NI], total = 0.f;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
        if (l + L * i >= p.k) break;
        const float a = v[i];
        rest[i] = soft ? 1.f : 1.f / (1.f + expf(a));
        v[i] = !there(a) ? 0.f : soft ? expf(a - shift) : expf(fminf(a, 0.f) - shift) / (1.f + expf(-fabsf(a)));
        total += v[i];
    }
    if (p.renorm) sum = row_sum<L>(total);
    else if (!soft) sum = 1.f;
    const float inv = sum == 0.f ? 1.f : 1.f / sum;
    float mean = 0.f;  // of u, over the shares
#pragma unroll
    for (int i = 0; i < NI; ++i) {
        if (l + L * i >= p.k) break;
        v[i] *= inv;
        mean += v[i] > 0.f || v[i] != v[i] ? u[i] * v[i] : 0.f;
    }
    mean = soft || p.renorm ? row_sum<L>(mean) : 0.f;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
        if (l + L * i >= p.k) break;
        s_g[wave][r][l + L * i] = v[i] * rest[i] * (p.renorm ? u[i] - mean : u[i]);
    }
    wave_sync();
#pragma unroll
    for (int j = 0; j < PER; ++j) dl[j] = 0.f;
    for (int i = 0; i < p.k; ++i) {
        const int at = s_e[wave][r][i] - l * PER;
        const float g = s_g[wave][r][i];
#pragma unroll
        for (int j = 0; j < PER; ++j) dl[j] = at == j ? dl[j] + g : dl[j];
    }
#pragma unroll
    for (int j = 0; j < PER; ++j)
        if (whole) x[j] *= inv;
    if (!stores) return;
    constexpr int V = 16 / (int)sizeof(T);
    T *const to = static_cast<T *>(p.dlogits) + row * p.dstride;
#pragma unroll
    for (int v = 0; v < PER; v += V) {
        float g[V];
#pragma unroll
        for (int e = 0; e < V; ++e) {
            g[e] = dl[v + e];
            if (whole) g[e] -= x[v + e] * mean;
            g[e] *= p.scale;
        }
        store_values(to + l * PER + v, g, p.E - (l * PER + v));
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
    const size_t lds = p.blocks > 1 ? (size_t)kWaves * wave_bytes(64 / L, L * PER, p.blocks) : 0;
    auto *kernel = keys ? k_route<T, L, PER, true> : k_route<T, L, PER, false>;
    hipLaunchKernelGGL(kernel, blocks, dim3(kThreads), lds, s, p);
    return hipGetLastError();
}

template <typename T> hipError_t pick(const RowRoute &p, bool gradient, hipStream_t s)
{
    if (p.E <= 8) return launch<T, 1, 8>(p, gradient, s);
    if (p.E <= 16) return launch<T, 2, 8>(p, gradient, s);
    if (p.E <= 32) return launch<T, 4, 8>(p, gradient, s);
    if (p.E <= 64) return launch<T, 8, 8>(p, gradient, s);
    if (p.E <= 128) return launch<T, 16, 8>(p, gradient, s);
    if (p.E <= 256) return launch<T, 32, 8>(p, gradient, s);
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
