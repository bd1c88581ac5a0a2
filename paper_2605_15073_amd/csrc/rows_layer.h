// The activations of layers (cgtp_grouped_layer) and what a product's tile does with them.
#ifndef CGTP_ROWS_LAYER_H
#define CGTP_ROWS_LAYER_H

#include <type_traits>

#include "rows_tile.h"

namespace cgtp {
namespace rows {

// What a launch does beside the product: nothing, a layer's bias, activation and residual, or rows of sums in fp32; kGrad:
// nothing, for a layer's row gradient. Z: that forms its rows dz = dy act'(z) in bf16 from both.
enum Extra { kBare, kLayer, kSums, kGrad, kSumsZ, kGradZ };
template <Extra EX> constexpr bool kForms = EX == kSumsZ || EX == kGradZ;
template <Extra EX> constexpr int kRowParts = kForms<EX> ? 2 : 1;  // bf16 operands that a row of the input is

// exp(a), 4 2^-24 of it off whatever a is: the rounding of a / log 2, which alone would be off by that times |a|, is put
// back behind the exponential. Arguments are held where the results are 0 or infinite already. Layers in fp32, silu, us with
// the plain exponential and with it: 525,308 rows, 64 -> 64, z, 84 and 88, 262,144, 64 -> 448, 140 and 152, gradients 116 and 120.
__device__ __forceinline__ float exp_far(float a)
{
    constexpr float kLog2e = 1.44269502f, kRest = 1.92596303e-8f;  // 1 / log 2 in two parts
    a = __builtin_amdgcn_fmed3f(a, -150.f, 150.f);
    const float t = a * kLog2e, off = fmaf(a, kRest, fmaf(a, kLog2e, -t));
    return __builtin_amdgcn_exp2f(t) * fmaf(0.693147182f, off, 1.f);
}

// silu: z s(z), s the logistic function; gelu: z P(z), P the normal distribution function; relu: max(z, 0).
// An infinite z gives what the formula's products do: -inf s(-inf) is NaN. The exponential of bf16 results is the plain
// one, off by 2.5 |z| 2^-24.
template <typename T> __device__ __forceinline__ float logistic(float z)
{
    return __builtin_amdgcn_rcpf(1.f + (sizeof(T) == 2 ? __expf(-z) : exp_far(-z)));
}

__device__ __forceinline__ float bell(float z) { return __builtin_amdgcn_exp2f(-0.72134752f * z * z); }  // exp(-z^2 / 2)

// P(z), from the tail P(-|z|). Of bf16 results it is 2 to the power of a polynomial in |z|, whose relative error up to
// |z| = 8 is 2^-15, under a fiftieth of bf16's rounding; past it the tail is below 2^-50, and falls on to zero. Of fp32
// ones it is exp(-z^2 / 2) t times a polynomial in t = 1 / (1 + |z| / 4): 2^-25 for all z, 8 2^-24 as fp32 evaluates it.
// Linear programs chose the coefficients for the smallest relative error. Seven products and one exponential, or eleven,
// one and a reciprocal: 525,308 rows, 64 to 64, z, fp32, 90 us where erfc takes 118.
template <typename T> __device__ __forceinline__ float normal_cdf(float z)
{
    const float a = fabsf(z);
    float tail;
    if constexpr (sizeof(T) == 2) {
        float q = fmaf(-1.2625606e-06f, a, 4.82061895e-05f);
        q = fmaf(q, a, -0.000807280284f);
        q = fmaf(q, a, 0.00794475241f);
        q = fmaf(q, a, -0.0526358583f);
        q = fmaf(q, a, -0.459956224f);
        q = fmaf(q, a, -1.15061022f);
        q = fmaf(q, a, -1.00004307f);
        tail = __builtin_amdgcn_exp2f(q);
    } else {
        const float t = __builtin_amdgcn_rcpf(fmaf(0.25f, a, 1.f));
        float q = fmaf(0.019811204f, t, -0.080998263f);
        q = fmaf(q, t, 0.095814106f);
        q = fmaf(q, t, -0.03194117f);
        q = fmaf(q, t, 0.063844485f);
        q = fmaf(q, t, 0.058915387f);
        q = fmaf(q, t, 0.081617557f);
        q = fmaf(q, t, 0.0934646f);
        q = fmaf(q, t, 0.099736505f);
        q = fmaf(q, t, 0.099735568f);
        tail = bell(z) * (q * t);
    }
    return z < 0.f ? tail : 1.f - tail;
}

// T: the type that the result is rounded to.
template <typename T> __device__ __forceinline__ float activate(float z, int act)
{
    if (act == CGTP_ACT_SILU) return z * logistic<T>(z);
    if (act == CGTP_ACT_GELU) return z * normal_cdf<T>(z);
    if (act == CGTP_ACT_RELU) return z <= 0.f ? 0.f : z;
    return z;
}

// The derivative.
template <typename T> __device__ __forceinline__ float activate_slope(float z, int act)
{
    if (act == CGTP_ACT_SILU) {
        const float f = logistic<T>(z);
        return f * (1.f + z * (1.f - f));
    }
    if (act == CGTP_ACT_GELU) return normal_cdf<T>(z) + z * 0.39894228f * bell(z);
    if (act == CGTP_ACT_RELU) return z > 0.f ? 1.f : z <= 0.f ? 0.f : z;
    return 1.f;
}

// dz = dy act'(z) of bf16 rows is an operand of two products. It is held in two bf16 parts, 16 bits of significand: off by
// 2^-17, a five-hundredth of what the rounding of the results may be. In one, gradients were 2.4e-3 off (relative norm)
// where that rounding alone gives 1.7e-3. The products form it where they load dy and z, or load the parts (kDzHeld).
// One that is not finite makes results that are not, which are formed again.
__device__ __forceinline__ unsigned pack_pair(float a, float b)
{
    const bf2_t h = {(bf16_t)a, (bf16_t)b};
    return __builtin_bit_cast(unsigned, h);
}
__device__ __forceinline__ void split_pair(float a, float b, unsigned &high, unsigned &low)
{
    high = pack_pair(a, b);
    const float ra = a - __builtin_bit_cast(float, high << 16), rb = b - __builtin_bit_cast(float, high & 0xffff0000u);
    low = pack_pair(ra, rb);
}

template <typename F> __device__ __forceinline__ float sum_of_eight(F f)
{
    return ((f(0) + f(1)) + (f(2) + f(3))) + ((f(4) + f(5)) + (f(6) + f(7)));
}

// Calls f with the activation, or kDzHeld, as a constant.
template <typename F> __device__ __forceinline__ void with_act(int act, F f)
{
    if (act == CGTP_ACT_SILU) f(std::integral_constant<int, CGTP_ACT_SILU>());
    else if (act == CGTP_ACT_GELU) f(std::integral_constant<int, CGTP_ACT_GELU>());
    else if (act == CGTP_ACT_RELU) f(std::integral_constant<int, CGTP_ACT_RELU>());
    else f(std::integral_constant<int, kDzHeld>());
}

// The parts of two values of dz, from a pair of dy and of z.
template <int ACT> __device__ __forceinline__ void dz_pair(unsigned dy, unsigned z, unsigned &high, unsigned &low)
{
    if constexpr (ACT == kDzHeld) {
        high = dy;
        low = z;
    } else {
        const float a = __builtin_bit_cast(float, dy << 16) * activate_slope<bf16_t>(__builtin_bit_cast(float, z << 16), ACT);
        const float b = __builtin_bit_cast(float, dy & 0xffff0000u) *
                        activate_slope<bf16_t>(__builtin_bit_cast(float, z & 0xffff0000u), ACT);
        split_pair(a, b, high, low);
    }
}

// The parts of eight.
template <int ACT> __device__ __forceinline__ void dz_parts(uint4_t dy, uint4_t z, uint4_t (&part)[2])
{
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        unsigned high, low;
        dz_pair<ACT>(dy[k], z[k], high, low);
        part[0][k] = high;
        part[1][k] = low;
    }
}

// One value of it.
__device__ __forceinline__ float dz_value(float dy, float z, int act)
{
    return act == kDzHeld ? (__builtin_isfinite(dy) ? dy + z : dy) : dy * activate_slope<bf16_t>(z, act);
}

// All sums of a lane in place. MARK: NaN where z is not finite.
template <typename T, bool MARK> __device__ __forceinline__ void activate_all(float16_t &z, int act)
{
    auto all = [&](auto kind) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float a = activate<T>(z[i], decltype(kind)::value);
            z[i] = MARK ? fmaf(z[i], 0.f, a) : a;
        }
    };
    if (act == CGTP_ACT_SILU) all(std::integral_constant<int, CGTP_ACT_SILU>());
    else if (act == CGTP_ACT_GELU) all(std::integral_constant<int, CGTP_ACT_GELU>());
    else if (act == CGTP_ACT_RELU) all(std::integral_constant<int, CGTP_ACT_RELU>());
    else if (MARK) all(std::integral_constant<int, CGTP_ACT_NONE>());
}

// Four columns of a lane's row into its sums, as vec_val takes them out.
template <typename T, bool TRANS> __device__ __forceinline__ void set_vec(float16_t &acc, int v, float4_t x)
{
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int pair = 4 * (v >> 1) + 2 * (v & 1);
        const int i = !TRANS ? 4 * v + e : sizeof(T) == 2 ? 4 * e + v : pair + (e == 1 ? 8 : e == 2 ? 1 : e == 3 ? 9 : 0);
        acc[i] = x[e];
    }
}

// Four values from p on, zero past the `left` that exist.
__device__ __forceinline__ float4_t load_four(const float *p, int64_t left)
{
    if (left >= 4) return *reinterpret_cast<const float4_any *>(p);
    float4_t v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (left > e) v[e] = p[e];
    return v;
}
__device__ __forceinline__ float4_t load_four(const bf16_t *p, int64_t left)
{
    float4_t v = {0.f, 0.f, 0.f, 0.f};
    if (left >= 4) {
        const bf4_t h = *reinterpret_cast<const bf4_any *>(p);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = (float)h[e];
        return v;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (left > e) v[e] = (float)p[e];
    return v;
}

// V values to p on, of which `left` exist.
template <typename T, int V> __device__ __forceinline__ void store_values(T *p, const float (&v)[V], int left)
{
    if (left >= V) {
        typedef T vec_t __attribute__((ext_vector_type(V)));
        typedef vec_t any_t __attribute__((aligned(sizeof(T))));
        vec_t h;
#pragma unroll
        for (int e = 0; e < V; ++e) h[e] = (T)v[e];
        *reinterpret_cast<any_t *>(p) = h;
        return;
    }
#pragma unroll
    for (int e = 0; e < V; ++e)
        if (e < left) p[e] = (T)v[e];
}

// Columns col .. col + 3 of row `row` of group g of a layer, from the product's sums (not grouped: of no group, whose
// z is zero). MARK: a sum that is not finite leaves NaN in y whatever the activation makes of it, for
// layer_plain_sums to find.
template <typename T, bool MARK>
__device__ __forceinline__ void store_layer(const RowProduct &p, int g, bool grouped, int64_t row, int col, float4_t sum)
{
    const int left = p.N - col;
    if (left <= 0) return;
    float4_t x = sum;
    if (p.bias && grouped) x += load_four(static_cast<const T *>(p.bias) + (int64_t)g * p.N + col, left);
    if (p.z) store_four<false>(static_cast<T *>(p.z) + row * p.z_stride + col, x, left);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        x[e] = activate<T>(x[e], p.act);
        if (MARK) x[e] = fmaf(sum[e], 0.f, x[e]);
    }
    if (p.residual) x += load_four(static_cast<const T *>(p.residual) + row * p.residual_stride + col, left);
    store_four<false>(static_cast<T *>(p.out) + row * p.out_stride + col, x, left);
}

// Columns col .. col + 7 of it in bf16, in vectors of 16 bytes: 131,327 rows of four, 448 -> 128, with z 282 us by fours, 231
// by eights; 20,000 of 10 groups, 300 -> 897, 81 and 66; 262,144, 448 -> 128, 102 and 95.
__device__ __forceinline__ void store_layer8(const RowProduct &p, int g, int64_t row, int col, float4_t lo, float4_t hi)
{
    typedef bf8_t any_t __attribute__((aligned(2)));
    const int left = p.N - col;
    if (left < 8) {
        store_layer<bf16_t, false>(p, g, true, row, col, lo);
        store_layer<bf16_t, false>(p, g, true, row, col + 4, hi);
        return;
    }
    float x[8];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        x[e] = lo[e];
        x[4 + e] = hi[e];
    }
    auto add = [&](const void *from, int64_t at) {
        const bf8_t b = *reinterpret_cast<const any_t *>(static_cast<const bf16_t *>(from) + at);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] += (float)b[e];
    };
    if (p.bias) add(p.bias, (int64_t)g * p.N + col);
    if (p.z) store_values(static_cast<bf16_t *>(p.z) + row * p.z_stride + col, x, 8);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = activate<bf16_t>(x[e], p.act);
    if (p.residual) add(p.residual, row * p.residual_stride + col);
    store_values(static_cast<bf16_t *>(p.out) + row * p.out_stride + col, x, 8);
}

// One value of it, from its sum.
template <typename T> __device__ __forceinline__ void store_layer_one(const RowProduct &p, int g, int64_t row, int c, float x)
{
    if (p.bias) x += (float)static_cast<const T *>(p.bias)[(int64_t)g * p.N + c];
    if (p.z) static_cast<T *>(p.z)[row * p.z_stride + c] = (T)x;
    x = activate<T>(x, p.act);
    if (p.residual) x += (float)static_cast<const T *>(p.residual)[row * p.residual_stride + c];
    static_cast<T *>(p.out)[row * p.out_stride + c] = (T)x;
}

// Columns [c0, c1) of a tile's rows of no group.
template <typename T>
__device__ __forceinline__ void store_bare(const RowProduct &p, const int *row, int rows, int c0, int c1)
{
    const int quads = (c1 - c0 + 3) / 4;
    for (int i = threadIdx.x; i < rows * quads; i += kThreads) {
        const int r = row[i / quads], col = c0 + 4 * (i % quads);
        if (r < 0) continue;
        if (p.out_f32)
            store_four<false>(static_cast<float *>(p.out) + r * p.out_stride + col, float4_t{0.f, 0.f, 0.f, 0.f}, p.N - col);
        else store_layer<T, false>(p, 0, false, r, col, float4_t{0.f, 0.f, 0.f, 0.f});
    }
}

// The same of row gradients whose rows are formed in parts: an infinite weight times a part of the other sign, or times
// none, is NaN.
template <typename Out> __device__ void grad_plain_sums(const RowProduct &p, int group, int rows, const int *s_row, int c0, int c1)
{
    stores_done();
    const int width = c1 - c0;
    const bf16_t *const w = static_cast<const bf16_t *>(p.w) + (int64_t)group * p.w_group;
    for (int i = threadIdx.x; i < rows * width; i += kThreads) {
        const int64_t row = s_row[i / width];
        const int c = c0 + i % width;
        if (row < 0) continue;
        Out *const out = static_cast<Out *>(p.out) + row * p.out_stride + c;
        if (__builtin_isfinite(stored(out))) continue;
        const bf16_t *const dy = static_cast<const bf16_t *>(p.in) + row * p.in_stride;
        const bf16_t *const z = static_cast<const bf16_t *>(p.slope_z) + row * p.slope_stride;
        float x = 0.f;
        for (int k = 0; k < p.K && x == x; ++k) x = fmaf(dz_value((float)dy[k], (float)z[k], p.act), (float)w[(int64_t)c * p.K + k], x);  // NaN stays
        *out = (Out)x;
    }
}

// The results of a workgroup's rows that are not finite, in the columns [c0, c1), in plain fp32.
template <typename T, bool WNK>
__device__ void layer_plain_sums(const RowProduct &p, int group, int rows, const int *s_row, int c0, int c1)
{
    stores_done();
    const int width = c1 - c0;
    const T *const w = static_cast<const T *>(p.w) + (int64_t)group * p.w_group;
    for (int i = threadIdx.x; i < rows * width; i += kThreads) {
        const int64_t row = s_row[i / width];
        const int c = c0 + i % width;
        if (row < 0) continue;
        T *const out = static_cast<T *>(p.out) + row * p.out_stride + c;
        if (__builtin_isfinite(stored(out))) continue;
        const T *const in = static_cast<const T *>(p.in) + (int64_t)((unsigned)row / (unsigned)p.per) * p.in_stride;
        float x = 0.f;
        for (int k = 0; k < p.K && x == x; ++k)  // NaN stays
            x += (float)in[k] * (float)w[WNK ? (int64_t)c * p.K + k : (int64_t)k * p.N + c];
        store_layer_one<T>(p, group, row, c, x);
    }
}

}  // namespace rows
}  // namespace cgtp

#endif
