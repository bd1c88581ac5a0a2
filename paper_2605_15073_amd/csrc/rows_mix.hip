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

template <typename T> __device__ __forceinline__ Vals<T> load_vals(const T *p, int left)
{
    const uint4_t u = load_16<T, false>(p, left);
    Vals<T> r;
#pragma unroll
    for (int e = 0; e < kVec<T>; ++e) {
        if constexpr (sizeof(T) == 4) r.v[e] = __builtin_bit_cast(float, (unsigned)u[e]);
        else r.v[e] = __builtin_bit_cast(float, e % 2 ? u[e / 2] & 0xffff0000u : u[e / 2] << 16);
    }
    return r;
}

// Where vector i of a row of N starts.
template <int V> __device__ __forceinline__ int vec_at(int i, int N) { return i * V + V <= N || N < V ? i * V : N - V; }

constexpr int kRowsTasks = 1024;  // vectors of a workgroup, about

// out_t = residual_t + sum_j weights_tj y_(t k + j), in fp32, j ascending. Y: the type of y.
template <typename T, typename Y>
__global__ __launch_bounds__(kThreads) void k_mix_rows(RowMix p, int rows)
{
    constexpr int V = kVec<Y>;
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
        for (int j = 0; j < p.k; ++j) {
            const Vals<Y> v = load_vals(y + j * p.y_stride, left);
            const float f = w ? w[j] : 1.f;
#pragma unroll
            for (int e = 0; e < V; ++e) sum[e] = fmaf(f, v.v[e], sum[e]);
        }
        if (p.residual) {
            const T *const q = static_cast<const T *>(p.residual) + t * p.residual_stride + c;
#pragma unroll
            for (int e = 0; e < V; ++e)
                if (e < left) sum[e] += (float)q[e];
        }
        store_values(static_cast<T *>(p.out) + t * p.out_stride + c, sum, left);
    }
}

// dy_(t k + j) = weights_tj dout_t, dweights_tj = y_(t k + j) . dout_t. L lanes of a wave to a row t.
template <typename T, int L>
__global__ __launch_bounds__(kThreads) void k_mix_rows_grad(RowMixGrad p)
{
    constexpr int V = kVec<T>;
    const int nv = (p.N + V - 1) / V, lane = threadIdx.x % L;
    const int64_t t = tile_at(blockIdx.x, blockIdx.z, gridDim.x) * (kThreads / L) + threadIdx.x / L;
    if (t >= p.n) return;
    const T *const d = static_cast<const T *>(p.dout) + t * p.dout_stride;
    for (int j = 0; j < p.k; ++j) {
        const int64_t row = t * p.k + j;
        const float w = p.weights ? p.weights[row] : 1.f;
        float dot = 0.f;
        for (int i = lane; i < nv; i += L) {
            const int c = vec_at<V>(i, p.N), left = p.N - c, again = i * V - c;  // values that the vector before has too
            const Vals<T> g = load_vals(d + c, left);
            if (p.dweights) {
                const Vals<T> y = load_vals(static_cast<const T *>(p.y) + row * p.y_stride + c, left);
#pragma unroll
                for (int e = 0; e < V; ++e) dot = e >= again ? fmaf(y.v[e], g.v[e], dot) : dot;
            }
            if (p.dy) {
                float out[V];
#pragma unroll
                for (int e = 0; e < V; ++e) out[e] = w * g.v[e];
                store_values(static_cast<T *>(p.dy) + row * p.dy_stride + c, out, left);
            }
        }
        if (p.dweights) {
#pragma unroll
            for (int s = L / 2; s > 0; s /= 2) dot += __shfl_xor(dot, s);
            if (lane == 0) p.dweights[row] = dot;
        }
    }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void k_layer_dz(int64_t n, int N, int act, const T *dy, int64_t dy_stride,
                                                       const T *z, int64_t z_stride, T *dz, int rows)
{
    constexpr int V = kVec<T>;
    const int nv = (N + V - 1) / V;
    const int64_t t0 = tile_at(blockIdx.x, blockIdx.z, gridDim.x) * rows;
    if (t0 >= n) return;
    const int mine = n - t0 < rows ? (int)(n - t0) : rows;
    for (int i = threadIdx.x; i < mine * nv; i += kThreads) {
        const int64_t t = t0 + i / nv;
        const int c = vec_at<V>(i % nv, N), left = N - c;
        const Vals<T> g = load_vals(dy + t * dy_stride + c, left), a = load_vals(z + t * z_stride + c, left);
        float out[V];
#pragma unroll
        for (int e = 0; e < V; ++e) out[e] = g.v[e] * activate_slope<T>(a.v[e], act);
        store_values(dz + t * N + c, out, left);
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
    hipLaunchKernelGGL((k_mix_rows<T, Y>), dim3(grid.x, 1, grid.z), dim3(kThreads), 0, s, p, rows);
    return hipGetLastError();
}

template <typename T, int L> hipError_t grad(const RowMixGrad &p, hipStream_t s)
{
    constexpr int rows = kThreads / L;
    const TileGrid grid = tile_grid((p.n + rows - 1) / rows);
    hipLaunchKernelGGL((k_mix_rows_grad<T, L>), dim3(grid.x, 1, grid.z), dim3(kThreads), 0, s, p);
    return hipGetLastError();
}

template <typename T> hipError_t grad(const RowMixGrad &p, hipStream_t s)
{
    const int nv = (p.N + kVec<T> - 1) / kVec<T>;
    if (nv <= 4) return grad<T, 4>(p, s);
    if (nv <= 16) return grad<T, 16>(p, s);
    return grad<T, 64>(p, s);
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
