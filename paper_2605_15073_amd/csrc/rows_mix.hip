// Rows joined with weights (cgtp_mix_rows), the gradient of that, and the gradient at a layer's activation.
// All of them pass over memory once: bound by it.
#include "internal.h"
#include "rows_layer.h"

namespace cgtp {

namespace {

using namespace rows;

template <typename T> constexpr int kVec = 16 / (int)sizeof(T);

// Values of one vector in fp32. Vectors do not pass the end of a row of N: the last starts early, where there are
// so many values at all; else the missing ones are zero.
template <typename T> struct Vals { float v[kVec<T>]; };

// Past the caches, where a call is too large to be found there again: nothing, loads alone, or all. Stores go there
// where rows begin on half a line; else a row's two broken lines would leave in parts.
enum Past { kThrough, kLoads, kAll };
template <Past PAST, typename T> __device__ __forceinline__ Vals<T> load_vals(const T *p, int left)
{
    const uint4_t u = PAST != kThrough && left >= kVec<T> ? __builtin_nontemporal_load(reinterpret_cast<const uint4_any *>(p))
                                              : load_16<T, false>(p, left);
    Vals<T> r;
#pragma unroll
    for (int e = 0; e < kVec<T>; ++e) {
        if constexpr (sizeof(T) == 4) r.v[e] = __builtin_bit_cast(float, (unsigned)u[e]);
        else r.v[e] = __builtin_bit_cast(float, e % 2 ? u[e / 2] & 0xffff0000u : u[e / 2] << 16);
    }
    return r;
}

template <Past PAST, typename T, int V> __device__ __forceinline__ void store_vals(T *p, const float (&v)[V], int left)
{
    if (PAST == kAll && left >= V) {
        typedef T vec_t __attribute__((ext_vector_type(V)));
        typedef vec_t any_t __attribute__((aligned(sizeof(T))));
        vec_t h;
#pragma unroll
        for (int e = 0; e < V; ++e) h[e] = (T)v[e];
        __builtin_nontemporal_store(h, reinterpret_cast<any_t *>(p));
        return;
    }
    store_values(p, v, left);
}

// By what a call moves (the memory-side cache holds 256 MB) and where its output's rows lie.
Past past_caches(double bytes, const void *out, int64_t stride, size_t es)
{
    if (bytes <= (double)((int64_t)256 << 20)) return kThrough;
    return reinterpret_cast<uintptr_t>(out) % 64 == 0 && stride * es % 64 == 0 ? kAll : kLoads;
}

// Where vector i of a row of N starts.
template <int V> __device__ __forceinline__ int vec_at(int i, int N) { return i * V + V <= N || N < V ? i * V : N - V; }

constexpr int kRowsTasks = 1024;  // vectors of a workgroup, about

// out_t = residual_t + sum_j weights_tj y_(t k + j), in fp32, j ascending. Y: the type of y.
template <typename T, typename Y, Past PAST>
__global__ __launch_bounds__(kThreads) void k_mix_rows(RowMix p, int rows)
{
    constexpr int V = kVec<Y>, kAhead = 4;
    const int nv = (p.N + V - 1) / V;
    const int64_t t0 = tile_at(blockIdx.x, blockIdx.z, gridDim.x) * rows;
    if (t0 >= p.n) return;
    const int mine = p.n - t0 < rows ? (int)(p.n - t0) : rows;
    for (int i = threadIdx.x; i < mine * nv; i += kThreads) {
        const int r = i / nv, c = vec_at<V>(i % nv, p.N), left = p.N - c;
        const int64_t t = t0 + r;
        float sum[V];
#pragma unroll
        for (int e = 0; e < V; ++e) sum[e] = 0.f;
        const Y *y = static_cast<const Y *>(p.y) + t * p.k * p.y_stride + c;
        const float *const w = p.weights ? p.weights + t * p.k : nullptr;
        int j = 0;
        for (; j + kAhead <= p.k; j += kAhead) {
            Vals<Y> v[kAhead];
#pragma unroll
            for (int a = 0; a < kAhead; ++a) v[a] = load_vals<PAST>(y + (j + a) * p.y_stride, left);
#pragma unroll
            for (int a = 0; a < kAhead; ++a) {
                const float f = w ? w[j + a] : 1.f;
#pragma unroll
                for (int e = 0; e < V; ++e) sum[e] = fmaf(f, v[a].v[e], sum[e]);
            }
        }
        for (; j < p.k; ++j) {
            const Vals<Y> v = load_vals<PAST>(y + j * p.y_stride, left);
            const float f = w ? w[j] : 1.f;
#pragma unroll
            for (int e = 0; e < V; ++e) sum[e] = fmaf(f, v.v[e], sum[e]);
        }
        if (p.residual) {
            const T *const q = static_cast<const T *>(p.residual) + t * p.residual_stride + c;
            if constexpr (sizeof(T) == sizeof(Y)) {
                const Vals<T> v = load_vals<PAST>(q, left);
#pragma unroll
                for (int e = 0; e < V; ++e) sum[e] += v.v[e];
            } else {
#pragma unroll
                for (int e = 0; e < V; ++e)
                    if (e < left) sum[e] += (float)q[e];
            }
        }
        store_vals<PAST>(static_cast<T *>(p.out) + t * p.out_stride + c, sum, left);
    }
}

// dy_(t k + j) = weights_tj dout_t, dweights_tj = y_(t k + j) . dout_t. L lanes of a wave to a row t, whose dout they
// hold, NI vectors each (0: read again for each j).
template <typename T, int L, int NI, Past PAST>
__global__ __launch_bounds__(kThreads) void k_mix_rows_grad(RowMixGrad p)
{
    constexpr int V = kVec<T>, kHeld = NI > 0 ? NI : 1, kAhead = NI > 0 ? (NI <= 2 ? 4 / NI : 1) : 1;
    const int nv = (p.N + V - 1) / V, lane = threadIdx.x % L;
    const int64_t t = tile_at(blockIdx.x, blockIdx.z, gridDim.x) * (kThreads / L) + threadIdx.x / L;
    if (t >= p.n) return;
    const T *const d = static_cast<const T *>(p.dout) + t * p.dout_stride;
    const T *const y = static_cast<const T *>(p.y) + t * p.k * p.y_stride;
    T *const dy = static_cast<T *>(p.dy) + t * p.k * p.dy_stride;
    auto at = [&](int i) { return vec_at<V>(i < nv ? i : nv - 1, p.N); };
    Vals<T> g[kHeld];
#pragma unroll
    for (int h = 0; h < NI; ++h) {
        const int i = lane + L * h, c = at(i);
        g[h] = load_vals<PAST>(d + c, p.N - c);
    }
    auto add = [&](float dot, const Vals<T> &v, const Vals<T> &o, int i) {
        const int again = i < nv ? i * V - at(i) : V;  // values that the vector before has too; past the row all
#pragma unroll
        for (int e = 0; e < V; ++e) dot = e >= again ? fmaf(v.v[e], o.v[e], dot) : dot;
        return dot;
    };
    auto scaled = [&](int j, float w, const Vals<T> &v, int i) {
        const int c = at(i);
        float out[V];
#pragma unroll
        for (int e = 0; e < V; ++e) out[e] = w * v.v[e];
        if (i < nv) store_vals<PAST>(dy + j * p.dy_stride + c, out, p.N - c);
    };
    auto finish = [&](int j, float dot) {
#pragma unroll
        for (int s = L / 2; s > 0; s /= 2) dot += __shfl_xor(dot, s);
        if (lane == 0) p.dweights[t * p.k + j] = dot;
    };
    for (int j0 = 0; j0 < p.k; j0 += kAhead) {
        float w[kAhead];
#pragma unroll
        for (int a = 0; a < kAhead; ++a) w[a] = p.weights ? p.weights[t * p.k + (j0 + a < p.k ? j0 + a : 0)] : 1.f;
        if constexpr (NI > 0) {
            Vals<T> v[kAhead][NI];
            if (p.dweights)
#pragma unroll
                for (int a = 0; a < kAhead; ++a)
#pragma unroll
                    for (int h = 0; h < NI; ++h) {
                        const int c = at(lane + L * h);
                        v[a][h] = load_vals<PAST>(y + (j0 + a < p.k ? j0 + a : j0) * p.y_stride + c, p.N - c);
                    }
#pragma unroll
            for (int a = 0; a < kAhead; ++a) {
                if (j0 + a >= p.k) break;
                if (p.dy)
#pragma unroll
                    for (int h = 0; h < NI; ++h) scaled(j0 + a, w[a], g[h], lane + L * h);
                if (p.dweights) {
                    float dot = 0.f;
#pragma unroll
                    for (int h = 0; h < NI; ++h) dot = add(dot, v[a][h], g[h], lane + L * h);
                    finish(j0 + a, dot);
                }
            }
        } else {
            float dot = 0.f;
            for (int i = lane; i < nv; i += L) {
                const int c = at(i);
                const Vals<T> o = load_vals<kThrough>(d + c, p.N - c);
                if (p.dweights) dot = add(dot, load_vals<PAST>(y + j0 * p.y_stride + c, p.N - c), o, i);
                if (p.dy) scaled(j0, w[0], o, i);
            }
            if (p.dweights) finish(j0, dot);
        }
    }
}

// dz = dy act'(z); of bf16 the two parts of rows_layer.h, one behind the other: an infinity or NaN has one.
template <typename T>
__global__ __launch_bounds__(kThreads) void k_layer_dz(int64_t n, int N, int act, const T *dy, int64_t dy_stride,
                                                       const T *z, int64_t z_stride, T *dz, int rows)
{
    constexpr int V = kVec<T>, P = sizeof(T) == 2 ? 2 : 1;
    const int nv = (N + V - 1) / V;
    const int64_t t0 = tile_at(blockIdx.x, blockIdx.z, gridDim.x) * rows;
    if (t0 >= n) return;
    const int mine = n - t0 < rows ? (int)(n - t0) : rows;
    for (int i = threadIdx.x; i < mine * nv; i += kThreads) {
        const int64_t t = t0 + i / nv;
        const int c = vec_at<V>(i % nv, N), left = N - c;
        const Vals<T> g = load_vals<kThrough>(dy + t * dy_stride + c, left), a = load_vals<kThrough>(z + t * z_stride + c, left);
        float out[V];
#pragma unroll
        for (int e = 0; e < V; ++e) out[e] = g.v[e] * activate_slope<T>(a.v[e], act);
        T *const to = dz + t * N * P + c;
        store_values(to, out, left);
        if constexpr (P == 2) {
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float high = (float)(T)out[e];
                out[e] = __builtin_isfinite(high) ? out[e] - high : 0.f;
            }
            store_values(to + N, out, left);
        }
    }
}

// Rows of a workgroup, of n with nv vectors each: four vectors a thread, one where that leaves too few workgroups.
int rows_of(int64_t n, int nv)
{
    const int tasks = n * nv < (int64_t)2048 * kRowsTasks ? kThreads : kRowsTasks;
    return nv >= tasks ? 1 : tasks / nv;
}

template <typename T, typename Y> hipError_t mix(const RowMix &p, hipStream_t s)
{
    const int rows = rows_of(p.n, (p.N + kVec<Y> - 1) / kVec<Y>);
    const TileGrid grid = tile_grid((p.n + rows - 1) / rows);
    const Past past = past_caches((double)p.n * p.N * (p.k * sizeof(Y) + sizeof(T)), p.out, p.out_stride, sizeof(T));
    auto *kernel = past == kAll ? k_mix_rows<T, Y, kAll> : past == kLoads ? k_mix_rows<T, Y, kLoads> : k_mix_rows<T, Y, kThrough>;
    hipLaunchKernelGGL(kernel, dim3(grid.x, 1, grid.z), dim3(kThreads), 0, s, p, rows);
    return hipGetLastError();
}

template <typename T, int L, int NI> hipError_t grad(const RowMixGrad &p, hipStream_t s)
{
    constexpr int rows = kThreads / L;
    const TileGrid grid = tile_grid((p.n + rows - 1) / rows);
    const Past past = past_caches((double)p.n * p.N * p.k * sizeof(T) * 2, p.dy, p.dy_stride, sizeof(T));
    auto *kernel = past == kAll ? k_mix_rows_grad<T, L, NI, kAll>
                                : past == kLoads ? k_mix_rows_grad<T, L, NI, kLoads> : k_mix_rows_grad<T, L, NI, kThrough>;
    hipLaunchKernelGGL(kernel, dim3(grid.x, 1, grid.z), dim3(kThreads), 0, s, p);
    return hipGetLastError();
}

template <typename T> hipError_t grad(const RowMixGrad &p, hipStream_t s)
{
    const int nv = (p.N + kVec<T> - 1) / kVec<T>;
    if (nv <= 4) return grad<T, 4, 1>(p, s);
    if (nv <= 16) return grad<T, 16, 1>(p, s);
    if (nv <= 64) return grad<T, 64, 1>(p, s);
    if (nv <= 128) return grad<T, 64, 2>(p, s);
    if (nv <= 256) return grad<T, 64, 4>(p, s);
    return grad<T, 64, 0>(p, s);
}

template <typename T>
hipError_t layer_dz(int64_t n, int N, int act, const void *dy, int64_t dy_stride, const void *z, int64_t z_stride,
                    void *dz, hipStream_t s)
{
    const int rows = rows_of(n, (N + kVec<T> - 1) / kVec<T>);
    const TileGrid grid = tile_grid((n + rows - 1) / rows);
    hipLaunchKernelGGL(k_layer_dz<T>, dim3(grid.x, 1, grid.z), dim3(kThreads), 0, s, n, N, act,
                       static_cast<const T *>(dy), dy_stride, static_cast<const T *>(z), z_stride, static_cast<T *>(dz),
                       rows);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_mix_rows(int dtype, const RowMix &p, bool y_f32, hipStream_t s)
{
    if (dtype == CGTP_F32) return mix<float, float>(p, s);
    return y_f32 ? mix<bf16_t, float>(p, s) : mix<bf16_t, bf16_t>(p, s);
}

hipError_t launch_mix_rows_grad(int dtype, const RowMixGrad &p, hipStream_t s)
{
    return dtype == CGTP_BF16 ? grad<bf16_t>(p, s) : grad<float>(p, s);
}

hipError_t launch_layer_dz(int dtype, int64_t n, int N, int act, const void *dy, int64_t dy_stride, const void *z,
                           int64_t z_stride, void *dz, hipStream_t s)
{
    return dtype == CGTP_BF16 ? layer_dz<bf16_t>(n, N, act, dy, dy_stride, z, z_stride, dz, s)
                              : layer_dz<float>(n, N, act, dy, dy_stride, z, z_stride, dz, s);
}

}  // namespace cgtp
