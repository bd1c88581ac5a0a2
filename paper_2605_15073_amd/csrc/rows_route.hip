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
            x[v + e] = f;
        }
    }
    if (first + PER > E)
#pragma unroll
        for (int j = 0; j < PER; ++j) x[j] = first + j < E ? x[j] : -__builtin_inff();
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

// Keys whose order is that of ints: of fp32 values above -inf, all of them above kGone. Low bits say where a key is, so
// that the largest tells: kPlace, PER - 1 - j, which tells a lane's keys apart; kExpert, 16 bits, 65535 - e, the order of
// equals too.
enum Embed { kNothing, kPlace, kExpert };
constexpr int kGone = -0x7fffffff - 1;
__device__ __forceinline__ int ordered(float f)
{
    const int b = __builtin_bit_cast(int, f);
    return b ^ (b >> 31 & 0x7fffffff);
}
__device__ __forceinline__ float value_of(int k) { return __builtin_bit_cast(float, k ^ (k >> 31 & 0x7fffffff)); }

// A logit of expert e: bf16's lower half is free.
template <typename T> constexpr Embed kByLogit = sizeof(T) == 2 ? kExpert : kNothing;
template <typename T> __device__ __forceinline__ int logit_key(float x, int e)
{
    const int k = ordered(x + 0.f);  // one zero
    if (!there(x)) return kGone;
    return sizeof(T) == 2 ? (k & -65536) | (65535 - e) : k;
}

template <int L, int D = 1> __device__ __forceinline__ int row_max(int v)
{
    if constexpr (D < L) {
        int o;
        if constexpr (D < 16) o = other_lane<D>(v);
        else o = __shfl_xor(v, D);
        return row_max<L, 2 * D>(o > v ? o : v);
    } else return v;
}

// The lowest lane of a row, counted from its first, for which it holds (one does).
template <int L> __device__ __forceinline__ int lowest(bool it)
{
    const unsigned long long m = __ballot(it);
    if constexpr (L == 1) return 0;
    else if constexpr (L == 64) return __ffsll(m) - 1;
    else return __ffs((int)(m >> ((threadIdx.x & 63) / L * L))) - 1;  // other rows' bits lie above
}

// Whether a key is within off[0], and off[1] of their magnitudes, of the one before.
__device__ __forceinline__ bool near(int before, int key, const float *off)
{
    const float a = value_of(before), b = value_of(key);
    return key != kGone && !(b < a - (off[0] + off[1] * (fabsf(a) + fabsf(b))));
}

// Experts of the k largest keys to ids. With `off`, false where a chosen key is within that (off[0],
// and off[1] of their magnitudes) of the next; the lanes of a row say it for a part of them each.
template <int L, int PER, Embed EMBED>
__device__ __forceinline__ bool take(int (&key)[PER], int k, int l, const float *off, int *ids)
{
    bool sure = true;
    int mine = kGone, before = kGone;  // the key of rank l, the one before
    const int rounds = off ? k + 1 : k;
    for (int i = 0; i < rounds; ++i) {
        int own = key[0];
#pragma unroll
        for (int j = 1; j < PER; ++j) own = key[j] > own ? key[j] : own;
        const int best = row_max<L>(own);
        if (off) {
            if (rounds <= L) {
                mine = l == i ? best : mine;
            } else {
                if (i > 0 && near(before, best, off)) sure = false;
                before = best;
            }
            if (i == k) break;
        }
        if constexpr (EMBED == kExpert) {
#pragma unroll
            for (int j = 0; j < PER; ++j) key[j] = key[j] == best ? kGone : key[j];
            if (l == 0) ids[i] = best == kGone ? -1 : 65535 - (best & 65535);
            continue;
        }
        const int winner = lowest<L>(own == best);
        if constexpr (EMBED == kPlace) {
            const int gone = l == winner ? best : kGone;
#pragma unroll
            for (int j = 0; j < PER; ++j) key[j] = key[j] == gone ? kGone : key[j];
            if (l == winner) ids[i] = best == kGone ? -1 : l * PER + (PER - 1 - (best & (PER - 1)));
        } else if (l == winner) {
            int at = 0;
#pragma unroll
            for (int j = PER - 1; j >= 0; --j) at = key[j] == best ? j : at;
#pragma unroll
            for (int j = 0; j < PER; ++j) key[j] = j == at ? kGone : key[j];
            ids[i] = best == kGone ? -1 : l * PER + at;
        }
    }
    if (off && rounds <= L) {
        before = __shfl_up(mine, 1);
        sure = !(l > 0 && near(before, mine, off));
    }
    return sure;
}

// How far a score in fp32 may be off, in 2^-24 of the largest. Exponentials of an argument a are off by 2 + 2.5 |a| of
// 2^-24 of themselves. s = 1 / (1 + e): s (1 - s) of that is below 1.1; the sum and the reciprocal add 1 and 2. A share
// of a sum: 2.9 from its own, where s |a| is below 0.37 of the largest; 23 from a sum of 512, where the mean of |a| is
// below log 512 + 2; 14 from its additions, of a lane and over lanes; 3 from reciprocal and product. A bias adds the
// rounding of the key, kStep of it; the lane's place PER - 1 steps.
constexpr float kStep = 0x1p-23f;
__device__ __forceinline__ float off_score(int score) { return (score == CGTP_SCORE_SOFTMAX ? 48.f : 6.f) * 0x1p-24f; }

// The two largest keys of a block, added (one where there is one).
template <typename Key> struct Two {
    Key first = -(Key)__builtin_inff(), second = first;
    __device__ __forceinline__ void add(Key v)
    {
        const Key low = v > first ? first : v;
        first = v > first ? v : first;
        second = low > second ? low : second;
    }
    __device__ __forceinline__ Key sum() const { return second > -(Key)__builtin_inff() ? first + second : first; }
};

// The choice by keys in fp32. False where it does not settle it.
template <typename T, int L, int PER>
__device__ __forceinline__ bool choose_near(const RowRoute &p, const float (&x)[PER], float top, int l, float *row_keys,
                                            int *ids)
{
    constexpr float kNone = -__builtin_inff();
    float f[PER], bias[PER], most = 1.f;  // the largest score
    if (p.bias) load_logits(bias, p.bias, l * PER, p.E);
    if (p.score == CGTP_SCORE_SOFTMAX) {
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            f[j] = there(x[j]) ? __expf(x[j] - top) : 0.f;
            sum += f[j];
        }
        most = __builtin_amdgcn_rcpf(row_sum<L>(sum));
#pragma unroll
        for (int j = 0; j < PER; ++j) f[j] *= most;
    } else {
#pragma unroll
        for (int j = 0; j < PER; ++j) f[j] = __builtin_amdgcn_rcpf(1.f + __expf(-x[j]));
    }
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        if (p.bias) f[j] += bias[j];
        f[j] = (there(x[j]) & (f[j] > kNone)) ? f[j] : kNone;
    }
    bool sure = true;
    if (p.blocks > 1) {
        const int size = p.E / p.blocks;
        float *const scores = row_keys + L * PER;
        // Keys of a sum add up to its magnitude and twice the largest score at most, or they are for 64 bits.
        auto sum_of = [&](const Two<float> &two) {
            if (two.second > kNone && two.second < -most) sure = false;
            return two.sum();
        };
        // whether block b is left, by the scores
        auto left = [&](int b) {
            const float own = scores[b], off = 4 * off_score(p.score) * most + 4 * kStep * (fabsf(own) + most);
            int ahead = 0, perhaps = 0;
            for (int i = 0; i < p.blocks; ++i) {
                const float v = scores[i];
                ahead += v > own + off;
                perhaps += v >= own - off;  // itself among them
            }
            // infinite ones are for 64 bits
            if (own > kNone && (!(own < -kNone) || (ahead < p.keep && perhaps > p.keep))) sure = false;
            return ahead < p.keep;
        };
        const int lanes = size / PER;
        if (size % PER == 0 && (lanes & (lanes - 1)) == 0) {  // a block is one lane's, or 2, 4, 8, ... lanes'
            Two<float> two;
#pragma unroll
            for (int j = 0; j < PER; ++j) two.add(f[j]);
            for (int d = 1; d < lanes; d *= 2) {
                const float first = __shfl_xor(two.first, d), second = __shfl_xor(two.second, d);
                two.add(first);
                two.add(second);
            }
            const int b = l / lanes;
            if (b < p.blocks && l % lanes == 0) scores[b] = sum_of(two);
            wave_sync();
            if (b < p.blocks && !left(b))
#pragma unroll
                for (int j = 0; j < PER; ++j) f[j] = kNone;
        } else {
#pragma unroll
            for (int j = 0; j < PER; ++j) row_keys[l * PER + j] = f[j];
            wave_sync();
            for (int b = l; b < p.blocks; b += L) {
                Two<float> two;
                for (int i = 0; i < size; ++i) two.add(row_keys[b * size + i]);
                scores[b] = sum_of(two);
            }
            wave_sync();
            for (int b = l; b < p.blocks; b += L)
                if (!left(b))
                    for (int i = 0; i < size; ++i) row_keys[b * size + i] = kNone;
            wave_sync();
#pragma unroll
            for (int j = 0; j < PER; ++j) f[j] = row_keys[l * PER + j];
        }
    }
    int key[PER];
    if (!p.bias) {  // the scores' order is the logits'
#pragma unroll
        for (int j = 0; j < PER; ++j) key[j] = f[j] > kNone ? logit_key<T>(x[j], l * PER + j) : kGone;
        return take<L, PER, kByLogit<T>>(key, p.k, l, nullptr, ids) && sure;
    }
#pragma unroll
    for (int j = 0; j < PER; ++j) key[j] = f[j] > kNone ? (ordered(f[j]) & -PER) | (PER - 1 - j) : kGone;
    const float off[2] = {2 * off_score(p.score) * most, (PER + 1) * kStep};
    return take<L, PER, kPlace>(key, p.k, l, off, ids) && sure;
}

// The same in 64 bits.
template <int L, int PER>
__device__ __forceinline__ void choose_exact(const RowRoute &p, const float (&x)[PER], float top, int l, double *row_keys,
                                             int *ids)
{
    constexpr double kNone = -(double)__builtin_inff();
    double key[PER];
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
        const int e = l * PER + j;
        if (p.bias) key[j] += (double)p.bias[e < p.E ? e : 0];
        if (!there(x[j]) || !(key[j] > kNone)) key[j] = kNone;
    }
    if (p.blocks > 1) {
        // keys of the row, then scores of its blocks; those left out lose their keys
        const int size = p.E / p.blocks;
        double *const scores = row_keys + L * PER;
#pragma unroll
        for (int j = 0; j < PER; ++j) row_keys[l * PER + j] = key[j];
        wave_sync();
        for (int b = l; b < p.blocks; b += L) {
            Two<double> two;
            for (int i = 0; i < size; ++i) two.add(row_keys[b * size + i]);
            scores[b] = two.sum();
        }
        wave_sync();
        for (int b = l; b < p.blocks; b += L) {
            int ahead = 0;
            for (int i = 0; i < p.blocks; ++i) ahead += scores[i] > scores[b] || (scores[i] == scores[b] && i < b);
            if (ahead >= p.keep)
                for (int i = 0; i < size; ++i) row_keys[b * size + i] = kNone;
        }
        wave_sync();
#pragma unroll
        for (int j = 0; j < PER; ++j) key[j] = row_keys[l * PER + j];
    }
    if (!p.bias)  // the scores' order is the logits'
#pragma unroll
        for (int j = 0; j < PER; ++j) key[j] = key[j] > kNone ? (double)x[j] : kNone;
    for (int i = 0; i < p.k; ++i) {
        double own = key[0];
#pragma unroll
        for (int j = 1; j < PER; ++j) own = key[j] > own ? key[j] : own;
        const double best = row_max<L>(own);
        const int winner = lowest<L>(own == best);
        if (l == winner) {
            int at = 0;
#pragma unroll
            for (int j = PER - 1; j >= 0; --j) at = key[j] == best ? j : at;
#pragma unroll
            for (int j = 0; j < PER; ++j) key[j] = j == at ? kNone : key[j];
            ids[i] = best > kNone ? l * PER + at : -1;
        }
    }
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
    const bool soft = p.score == CGTP_SCORE_SOFTMAX;
    float top = kNone;
    bool odd = false;  // NaN or +inf among the logits
    if (soft) {
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            top = fmaxf(top, there(x[j]) ? x[j] : kNone);
            odd |= !(x[j] < __builtin_inff());
        }
        top = row_max<L>(top);
    }
    int *const ids = s_ids[wave][r];
    char *const mine = sh + wave * wave_bytes(R, L * PER, p.blocks);
    double *const keys = reinterpret_cast<double *>(mine) + r * (L * PER + p.blocks);
    if constexpr (!KEYS) {
        int key[PER];
#pragma unroll
        for (int j = 0; j < PER; ++j) key[j] = logit_key<T>(x[j], l * PER + j);
        take<L, PER, kByLogit<T>>(key, p.k, l, nullptr, ids);
    } else if constexpr (PER > 8) {
        choose_exact<L, PER>(p, x, top, l, keys, ids);
    } else {
        float *const keys32 = reinterpret_cast<float *>(mine) + r * (L * PER + p.blocks + 4);
        const bool sure = choose_near<T, L, PER>(p, x, top, l, keys32, ids);
        if (__any(!sure)) {
            wave_sync();
            choose_exact<L, PER>(p, x, top, l, keys, ids);
        }
    }
    wave_sync();
    // weights, rank l + L i. Renormalised ones are formed relative to the largest of the chosen.
    constexpr int NI = (kMost<L * PER> + L - 1) / L;
    float w[NI], sum = 0.f, shift = 0.f;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
        if (l + L * i >= p.k) break;
        const int e = ids[l + L * i];
        w[i] = e >= 0 ? (float)from[e] : kNone;
    }
    if (p.renorm) {
        shift = kNone;
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            if (l + L * i >= p.k) break;
            shift = fmaxf(shift, soft ? w[i] : fminf(w[i], 0.f));
        }
        shift = row_max<L>(shift);
    } else if (soft) {
        shift = top;
#pragma unroll
        for (int j = 0; j < PER; ++j) sum += there(x[j]) ? exp_far(x[j] - top) : 0.f;
        sum = row_sum<L>(sum);
    }
    float total = 0.f;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
        if (l + L * i >= p.k) break;
        const float v = w[i];
        w[i] = !there(v) ? 0.f : soft ? exp_far(v - shift) : exp_far(fminf(v, 0.f) - shift) / (1.f + exp_far(-fabsf(v)));
        total += w[i];
    }
    if (p.renorm) sum = row_sum<L>(total);
    else if (!soft) sum = 1.f;
    unsigned long long any = soft ? __ballot(odd) : 0;
    if (L < 64) any = any >> (lane / L * L) & ((1ull << (L % 64)) - 1);
    if (!stores) return;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
        const int c = l + L * i;
        if (c >= p.k) break;
        p.ids[row * p.k + c] = ids[c];
        p.weights[row * p.k + c] = any ? __builtin_nanf("") : w[i] == 0.f ? 0.f : w[i] / sum * p.scale;
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

template <typename T, int L, int PER, bool KEYS> hipError_t route(const RowRoute &p, hipStream_t s)
{
    constexpr int rows = kWaves * (64 / L);
    const TileGrid grid = tile_grid((p.n + rows - 1) / rows);
    const size_t lds = p.blocks > 1 ? (size_t)kWaves * wave_bytes(64 / L, L * PER, p.blocks) : 0;
    hipLaunchKernelGGL((k_route<T, L, PER, KEYS>), dim3(grid.x, 1, grid.z), dim3(kThreads), lds, s, p);
    return hipGetLastError();
}

// Sixteen logits a lane, eight keys: us with eight and sixteen, bf16, 525,308 rows of 64, 4 of them, by the logits 32
// and 27, by a bias 51 and 54, in blocks 71 and 112 (more rows of a wave share the 64-bit choice of one); with eight these two
// take 49 and 66 by now.
template <typename T, int L> hipError_t route(const RowRoute &p, hipStream_t s)
{
    if (p.bias || p.blocks > 1) return route<T, L, 8, true>(p, s);
    return route<T, L / 2, 16, false>(p, s);
}

template <typename T, int L, int PER> hipError_t gradient(const RowRoute &p, hipStream_t s)
{
    constexpr int rows = kWaves * (64 / L);
    const TileGrid grid = tile_grid((p.n + rows - 1) / rows);
    hipLaunchKernelGGL((k_route_grad<T, L, PER>), dim3(grid.x, 1, grid.z), dim3(kThreads), 0, s, p);
    return hipGetLastError();
}

template <typename T> hipError_t pick(const RowRoute &p, hipStream_t s)
{
    const bool keys = p.bias || p.blocks > 1;
    if (p.E <= 8) return keys ? route<T, 1, 8, true>(p, s) : route<T, 1, 8, false>(p, s);
    if (p.E <= 16) return route<T, 2>(p, s);
    if (p.E <= 32) return route<T, 4>(p, s);
    if (p.E <= 64) return route<T, 8>(p, s);
    if (p.E <= 128) return route<T, 16>(p, s);
    if (p.E <= 256) return route<T, 32>(p, s);
    if (p.E <= 512) return route<T, 64>(p, s);
    return keys ? route<T, 64, 64, true>(p, s) : route<T, 64, 64, false>(p, s);
}

template <typename T> hipError_t pick_gradient(const RowRoute &p, hipStream_t s)
{
    if (p.E <= 8) return gradient<T, 1, 8>(p, s);
    if (p.E <= 16) return gradient<T, 2, 8>(p, s);
    if (p.E <= 32) return gradient<T, 4, 8>(p, s);
    if (p.E <= 64) return gradient<T, 8, 8>(p, s);
    if (p.E <= 128) return gradient<T, 16, 8>(p, s);
    if (p.E <= 256) return gradient<T, 32, 8>(p, s);
    if (p.E <= 512) return gradient<T, 64, 8>(p, s);
    return gradient<T, 64, 64>(p, s);
}

}  // namespace

hipError_t launch_route_rows(int dtype, const RowRoute &p, hipStream_t s)
{
    return dtype == CGTP_BF16 ? pick<bf16_t>(p, s) : pick<float>(p, s);
}

hipError_t launch_route_rows_grad(int dtype, const RowRoute &p, hipStream_t s)
{
    return dtype == CGTP_BF16 ? pick_gradient<bf16_t>(p, s) : pick_gradient<float>(p, s);
}

}  // namespace cgtp
