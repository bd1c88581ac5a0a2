// AdamW over many tensors (cgtp_adamw_*), states in 32 or in 8 bits.
//
// A handle holds a table of the tensors and of the work items, kItem consecutive elements of one
// tensor each, so that a step is one launch however many tensors there are. A wave takes 256
// consecutive elements at a time, four to a lane: with 8-bit states exactly one block, whose
// largest magnitudes are wave reductions. Every operation is rounded by itself: the codes then
// depend on nothing but the formulas, and a program that forms them in single fp32 operations
// gets the same ones.
//
// Measured, calls in a row: 5 million parameters in 200 tensors, 32-bit states, 23 us (6.1 TB/s, partly from the
// caches); 64 million, 8-bit states, bf16 gradients and copies, the step 243 us (4.2 TB/s; 80 more with the codes from
// rounded divisions and roots throughout, bound by the vector ALU), the decoding 94 us (6.8 TB/s, partly from the
// caches), step and decoding in turn 331.
#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

#include "internal.h"
#include "rows.h"

#pragma clang fp contract(off)

namespace {

using cgtp::report;

constexpr int kThreads = 256;
constexpr int kItem = 4096;      // elements of a work item: four blocks a wave
constexpr int kStatesMax = 64;   // tensors of one launch of the decoding

typedef __bf16 bf16_t;
typedef float float4_t __attribute__((ext_vector_type(4)));
typedef bf16_t bf4_t __attribute__((ext_vector_type(4)));
typedef signed char char4_t __attribute__((ext_vector_type(4)));
typedef unsigned char uchar4_t __attribute__((ext_vector_type(4)));
static_assert(CGTP_ADAMW_BLOCK == 256, "a wave's elements");

struct Item {
    int tensor;
    int start;  // in units of CGTP_ADAMW_BLOCK
};

struct Hyper {
    float decay, beta1, om1, beta2, om2, rate, inv_c2, eps;
};

// 4 elements from i on of an array of n, zero past its end
template <typename T4, typename T>
__device__ __forceinline__ T4 load4(const T *p, int64_t i, int64_t n, bool vec)
{
    if (vec && i + 4 <= n) return *reinterpret_cast<const T4 *>(p + i);
    T4 v;
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = i + k < n ? p[i + k] : T(0);
    return v;
}

// PAST: past the caches, for what is too large to be found there again.
template <bool PAST, typename T4, typename T>
__device__ __forceinline__ void store4(T *p, int64_t i, int64_t n, bool vec, T4 v)
{
    if (vec && i + 4 <= n) {
        if (PAST) __builtin_nontemporal_store(v, reinterpret_cast<T4 *>(p + i));
        else *reinterpret_cast<T4 *>(p + i) = v;
        return;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (i + k < n) p[i + k] = v[k];
}

constexpr float kInv127 = 1.f / 127.f, kInv255 = 1.f / 255.f;

__device__ __forceinline__ float decode_m(int c, float scale)
{
    const float t = (float)c * kInv127;
    return t * fabsf(t) * scale;
}

__device__ __forceinline__ float decode_v(int c, float scale)
{
    float t = (float)c * kInv255;
    t = t * t;
    return t * t * scale;
}

// The larger of a and b; NaN if either is.
__device__ __forceinline__ float max_nan(float a, float b) { return a > b || a != a ? a : b; }

__device__ __forceinline__ float wave_max(float v)
{
#pragma unroll
    for (int d = 32; d > 0; d /= 2) v = max_nan(v, __shfl_xor(v, d));
    return v;
}

__device__ __forceinline__ float exact_m(float m, float scale)
{
    return rintf(sqrtf(scale > 0.f ? fabsf(m) / scale : 0.f) * 127.f);
}

__device__ __forceinline__ float exact_v(float v, float scale)
{
    return rintf(sqrtf(sqrtf(scale > 0.f ? v / scale : 0.f)) * 255.f);
}

// The codes come from the hardware's reciprocal and square roots, each good to 1 unit in the last place,
// where their rounding to a whole number cannot depend on the difference: t is off by less than 8e-5
// (255 * 5 * 2^-24) from the real value, and the rounded operations' by less than 5e-5. Closer than
// kNear to a half, the rounded operations decide. `fast`: the block's scale is a normal number whose
// reciprocal is one too.
constexpr float kNear = 2e-4f;

__device__ __forceinline__ bool fast_scale(float s) { return s > 0x1p-100f && s < 0x1p100f; }

__device__ __forceinline__ int encode_m(float m, float scale, float inv, bool fast)
{
    const float t = __builtin_amdgcn_sqrtf(fabsf(m) * inv) * 127.f;
    float q = rintf(t);
    if (!fast || !(fabsf(t - q) < 0.5f - kNear)) q = exact_m(m, scale);
    return m < 0.f ? -(int)q : (int)q;
}

__device__ __forceinline__ int encode_v(float v, float scale, float inv, bool fast)
{
    const float t = __builtin_amdgcn_sqrtf(__builtin_amdgcn_sqrtf(v * inv)) * 255.f;
    float q = rintf(t);
    if (!fast || !(fabsf(t - q) < 0.5f - kNear)) q = exact_v(v, scale);
    return v > 0.f && q < 1.f ? 1 : (int)q;
}

bool aligned(const void *p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

struct Tensor {
    cgtp_adamw_tensor t;
    int vec;  // every array starts at a multiple of four of its elements
};

template <typename G, int BITS, bool PAST>
__global__ __launch_bounds__(kThreads) void k_adamw(const Tensor *__restrict__ tensors,
                                                    const Item *__restrict__ items, Hyper h,
                                                    const float *__restrict__ grad_scale)
{
    typedef G g4_t __attribute__((ext_vector_type(4)));
    const Item item = items[blockIdx.x];
    const Tensor &tn = tensors[item.tensor];
    const cgtp_adamw_tensor t = tn.t;
    const bool vec = tn.vec;
    const float gs = grad_scale ? grad_scale[0] : 1.f;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int it = 0; it < kItem / 1024; ++it) {
        const int64_t block = (int64_t)item.start + it * 4 + wave;
        const int64_t i = block * 256 + lane * 4;
        if (block * 256 >= t.n) break;
        float4_t p = load4<float4_t>(t.param, i, t.n, vec);
        const g4_t graw = load4<g4_t>((const G *)t.grad, i, t.n, vec);
        float4_t m, v;
        if (BITS == 32) {
            m = load4<float4_t>((const float *)t.m, i, t.n, vec);
            v = load4<float4_t>((const float *)t.v, i, t.n, vec);
        } else {
            const float ms = t.m_scale[block], vs = t.v_scale[block];
            const char4_t cm = load4<char4_t>((const signed char *)t.m, i, t.n, vec);
            const uchar4_t cv = load4<uchar4_t>((const unsigned char *)t.v, i, t.n, vec);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                m[k] = decode_m(cm[k], ms);
                v[k] = decode_v(cv[k], vs);
            }
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float g = (float)graw[k] * gs;
            m[k] = m[k] * h.beta1 + g * h.om1;
            v[k] = v[k] * h.beta2 + g * g * h.om2;
            const float den = sqrtf(v[k] * h.inv_c2) + h.eps;
            p[k] = p[k] * h.decay - m[k] * h.rate / den;
        }
        store4<PAST, float4_t>(t.param, i, t.n, vec, p);
        if (t.copy) {
            bf4_t c;
#pragma unroll
            for (int k = 0; k < 4; ++k) c[k] = (bf16_t)p[k];
            store4<PAST, bf4_t>((bf16_t *)t.copy, i, t.n, vec, c);
        }
        if (BITS == 32) {
            store4<PAST, float4_t>((float *)t.m, i, t.n, vec, m);
            store4<PAST, float4_t>((float *)t.v, i, t.n, vec, v);
        } else {
            float ms = 0.f, vs = 0.f;
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (i + k < t.n) {
                    ms = max_nan(fabsf(m[k]), ms);
                    vs = max_nan(v[k], vs);
                }
            ms = wave_max(ms);
            vs = wave_max(vs);
            const float im = __builtin_amdgcn_rcpf(ms), iv = __builtin_amdgcn_rcpf(vs);
            const bool fm = fast_scale(ms), fv = fast_scale(vs);
            char4_t cm;
            uchar4_t cv;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                cm[k] = (signed char)encode_m(m[k], ms, im, fm);
                cv[k] = (unsigned char)encode_v(v[k], vs, iv, fv);
            }
            store4<PAST, char4_t>((signed char *)t.m, i, t.n, vec, cm);
            store4<PAST, uchar4_t>((unsigned char *)t.v, i, t.n, vec, cv);
            if (lane == 0) {
                t.m_scale[block] = ms;
                t.v_scale[block] = vs;
            }
        }
    }
}

// The norm of all gradients: sums of squares in 64 bits (the square of an fp32 number is one of them, and none
// passes their range), in one launch: a second one costs the host 3 us, a quarter of a small call. Workgroup b takes the
// items b, b + gridDim.x, ..., leaves its sum in the workspace, and counts itself done: in its group of kDoneGroup,
// whose last one counts the group. The last of all adds the sums in their order; the counters are zero again then.
constexpr int kNormBlocks = 2048, kDoneGroup = 32;
constexpr int kCounters = 1 + kNormBlocks / kDoneGroup, kCounterStride = 16;  // words; half a line each

// What is passed on are 64-bit stores and loads past the caches, which the wait completes before the count: a release
// and acquire of everything (a write-back and an invalidation of the L2 in each workgroup) took 37 us where this takes
// 9.2 (5 million gradients).
__device__ __forceinline__ bool last_of(unsigned *counter, unsigned count)
{
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    const unsigned before = __builtin_amdgcn_atomic_inc32(counter, count - 1, __ATOMIC_RELAXED, "agent");  // the last one's sets it to 0
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    return before == count - 1;
}

__device__ __forceinline__ double block_sum(double sum, double *s_sum)
{
#pragma unroll
    for (int d = 32; d > 0; d /= 2) sum += __shfl_xor(sum, d);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) s_sum[threadIdx.x >> 6] = sum;
    __syncthreads();
    return (s_sum[0] + s_sum[1]) + (s_sum[2] + s_sum[3]);
}

// grad_scale may be scale (or norm): it is read first.
template <typename G>
__global__ __launch_bounds__(kThreads) void k_grad_norm(const Tensor *__restrict__ tensors, const Item *__restrict__ items,
                                                        int64_t n_items, double *sums, unsigned *counters, double max_norm,
                                                        const float *grad_scale, float *norm, float *scale)
{
    typedef G g4_t __attribute__((ext_vector_type(4)));
    __shared__ double s_sum[kThreads / 64];
    __shared__ bool s_last;
    const int blocks = gridDim.x;
    double sum = 0;
    for (int64_t b = blockIdx.x; b < n_items; b += blocks) {
        const Item item = items[b];
        const Tensor &tn = tensors[item.tensor];
        const G *const grad = (const G *)tn.t.grad;
        const int64_t n = tn.t.n, start = (int64_t)item.start * CGTP_ADAMW_BLOCK;
#pragma unroll
        for (int it = 0; it < kItem / 1024; ++it) {
            const int64_t i = start + it * 1024 + threadIdx.x * 4;
            const g4_t g = load4<g4_t>(grad, i, n, tn.vec);
#pragma unroll
            for (int k = 0; k < 4; ++k) sum = fma((double)(float)g[k], (double)(float)g[k], sum);
        }
    }
    sum = block_sum(sum, s_sum);
    if (blocks > 1) {
        if (threadIdx.x == 0) {
            __hip_atomic_store(sums + blockIdx.x, sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            const int groups = (blocks + kDoneGroup - 1) / kDoneGroup, group = blockIdx.x / kDoneGroup;
            const int mine = group + 1 < groups ? kDoneGroup : blocks - group * kDoneGroup;
            s_last = last_of(counters + (1 + group) * kCounterStride, mine) && last_of(counters, groups);
        }
        __syncthreads();
        if (!s_last) return;
        sum = 0;
        for (int i = threadIdx.x; i < blocks; i += kThreads)
            sum += __hip_atomic_load(sums + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        sum = block_sum(sum, s_sum);
    }
    if (threadIdx.x > 0) return;
    const double by = grad_scale ? grad_scale[0] : 1.f, all = sqrt(sum) * fabs(by);
    if (norm) norm[0] = (float)all;
    if (scale) scale[0] = (float)(all > max_norm ? by * (max_norm / all) : by);
}

struct Outs {
    float *m[kStatesMax], *v[kStatesMax];
};

// items: those of the tensors [t0, t0 + kStatesMax)
template <bool PAST>
__global__ __launch_bounds__(kThreads) void k_adamw_states(const Tensor *__restrict__ tensors,
                                                           const Item *__restrict__ items, int t0,
                                                           Outs outs)
{
    const Item item = items[blockIdx.x];
    const Tensor &tn = tensors[item.tensor];
    const cgtp_adamw_tensor t = tn.t;
    float *const mo = outs.m[item.tensor - t0], *const vo = outs.v[item.tensor - t0];
    const bool vec_out = ((uintptr_t)mo | (uintptr_t)vo) % 16 == 0;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int it = 0; it < kItem / 1024; ++it) {
        const int64_t block = (int64_t)item.start + it * 4 + wave;
        const int64_t i = block * 256 + lane * 4;
        if (block * 256 >= t.n) break;
        const float ms = t.m_scale[block], vs = t.v_scale[block];
        const char4_t cm = load4<char4_t>((const signed char *)t.m, i, t.n, tn.vec);
        const uchar4_t cv = load4<uchar4_t>((const unsigned char *)t.v, i, t.n, tn.vec);
        float4_t m, v;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            m[k] = decode_m(cm[k], ms);
            v[k] = decode_v(cv[k], vs);
        }
        store4<PAST, float4_t>(mo, i, t.n, vec_out, m);
        store4<PAST, float4_t>(vo, i, t.n, vec_out, v);
    }
}

// Whether a call over that many items moves more bytes than the memory-side cache holds. Then its stores go past
// the caches: 64 million parameters, 8-bit states, us past and through them: the step 243 and 244, the decoding
// 94 and 143, both in turn 331 and 356; 5 million in 32 bits 24 and 23.
bool past_caches(int64_t items, int bytes) { return items * kItem * bytes > (int64_t)256 << 20; }

template <bool PAST> auto *pick(int grad_dtype, int bits)
{
    return grad_dtype == CGTP_BF16 ? (bits == 8 ? k_adamw<bf16_t, 8, PAST> : k_adamw<bf16_t, 32, PAST>)
                                   : (bits == 8 ? k_adamw<float, 8, PAST> : k_adamw<float, 32, PAST>);
}

int hip_fail(hipError_t e, const char *what)
{
    return report(CGTP_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

}  // namespace

struct cgtp_adamw_s {
    int n_tensors, grad_dtype, state_bits, device;
    int64_t n_items;
    void *table;              // Tensor[n_tensors], then Item[n_items], then counters
    Item *items;
    unsigned *counters;       // of k_grad_norm, zero between calls
    std::vector<int64_t> first_item;  // of each tensor, and the end
};

namespace {

int check_handle(const cgtp_adamw_s *a)
{
    if (!a) return report(CGTP_ERR_ARG, "handle is NULL");
    int dev = -1;
    const hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return hip_fail(e, "hipGetDevice");
    if (dev != a->device)
        return report(CGTP_ERR_ARG, "handle was created on device %d, current device is %d",
                      a->device, dev);
    return CGTP_OK;
}

int check_tensor(const cgtp_adamw_tensor &t, int i, int grad_dtype, int state_bits)
{
    if (t.n < 0) return report(CGTP_ERR_ARG, "tensor %d has %lld elements", i, (long long)t.n);
    if (t.n == 0) return CGTP_OK;
    if (!t.param || !t.grad || !t.m || !t.v)
        return report(CGTP_ERR_ARG, "tensor %d: param, grad, m or v is NULL", i);
    if (state_bits == 8 && (!t.m_scale || !t.v_scale))
        return report(CGTP_ERR_ARG, "tensor %d: m_scale or v_scale is NULL", i);
    const size_t gs = grad_dtype == CGTP_BF16 ? 2 : 4, ss = state_bits == 8 ? 1 : 4;
    if (!aligned(t.param, 4) || !aligned(t.grad, gs) || !aligned(t.m, ss) || !aligned(t.v, ss) ||
        !aligned(t.copy, 2) ||
        (state_bits == 8 && (!aligned(t.m_scale, 4) || !aligned(t.v_scale, 4))))
        return report(CGTP_ERR_ARG, "tensor %d: an array is not aligned to its elements", i);
    return CGTP_OK;
}

// What a step writes, of all tensors, lies apart: a parameter that is listed twice would be updated by two
// workgroups at once.
int check_apart(int n_tensors, const cgtp_adamw_tensor *tensors, int state_bits)
{
    struct Written {
        uintptr_t start, end;
        int tensor;
    };
    std::vector<Written> all;
    const size_t ss = state_bits == 8 ? 1 : 4;
    for (int i = 0; i < n_tensors; ++i) {
        const cgtp_adamw_tensor &t = tensors[i];
        if (t.n == 0) continue;
        const size_t n = (size_t)t.n, blocks = (n + CGTP_ADAMW_BLOCK - 1) / CGTP_ADAMW_BLOCK;
        auto add = [&](const void *p, size_t bytes) {
            const uintptr_t at = reinterpret_cast<uintptr_t>(p);
            if (p) all.push_back({at, at + bytes, i});
        };
        add(t.param, 4 * n);
        add(t.m, ss * n);
        add(t.v, ss * n);
        add(t.copy, 2 * n);
        if (state_bits == 8) {
            add(t.m_scale, 4 * blocks);
            add(t.v_scale, 4 * blocks);
        }
    }
    std::sort(all.begin(), all.end(), [](const Written &a, const Written &b) { return a.start < b.start; });
    for (size_t k = 1; k < all.size(); ++k)
        if (all[k].start < all[k - 1].end)
            return report(CGTP_ERR_ARG, "arrays that a step writes overlap, of tensors %d and %d", all[k - 1].tensor,
                          all[k].tensor);
    return CGTP_OK;
}

int create(int n_tensors, const cgtp_adamw_tensor *tensors, int grad_dtype, int state_bits,
           cgtp_adamw *handle)
{
    std::vector<Tensor> tv((size_t)n_tensors);
    std::vector<int64_t> first;
    int64_t n_items = 0;
    const size_t gs = grad_dtype == CGTP_BF16 ? 2 : 4, ss = state_bits == 8 ? 1 : 4;
    for (int i = 0; i < n_tensors; ++i) {
        const cgtp_adamw_tensor &t = tensors[i];
        const int st = check_tensor(t, i, grad_dtype, state_bits);
        if (st != CGTP_OK) return st;
        if (t.n > (int64_t)0x7fffff00 * CGTP_ADAMW_BLOCK)
            return report(CGTP_ERR_UNSUPPORTED, "tensor %d has 2^31 blocks or more", i);
        tv[i].t = t;
        tv[i].vec = aligned(t.param, 16) && aligned(t.grad, 4 * gs) && aligned(t.m, 4 * ss) &&
                    aligned(t.v, 4 * ss) && aligned(t.copy, 8);
        first.push_back(n_items);
        n_items += (t.n + kItem - 1) / kItem;
    }
    first.push_back(n_items);
    const int apart = check_apart(n_tensors, tensors, state_bits);
    if (apart != CGTP_OK) return apart;
    if (n_items > 0x7fffffffLL)
        return report(CGTP_ERR_UNSUPPORTED, "%lld work items", (long long)n_items);
    std::vector<Item> items;
    items.reserve((size_t)n_items);
    for (int i = 0; i < n_tensors; ++i)
        for (int64_t k = 0; k < first[i + 1] - first[i]; ++k)
            items.push_back({i, (int)(k * (kItem / CGTP_ADAMW_BLOCK))});
    int dev = -1;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return hip_fail(e, "hipGetDevice");
    cgtp_adamw_s *a = new cgtp_adamw_s{n_tensors, grad_dtype, state_bits, dev, n_items,
                                       nullptr,   nullptr,    nullptr,    std::move(first)};
    const size_t tb = tv.size() * sizeof(Tensor), ib = (items.size() * sizeof(Item) + 255) / 256 * 256;
    items.resize(ib / sizeof(Item), Item{0, 0});
    const std::vector<int> zeros(kCounters * kCounterStride, 0);
    const size_t cb = zeros.size() * sizeof(int);
    if (n_items > 0) {
        e = hipMalloc(&a->table, tb + ib + cb);
        if (e == hipSuccess) e = hipMemcpy(a->table, tv.data(), tb, hipMemcpyHostToDevice);
        if (e == hipSuccess)
            e = hipMemcpy(static_cast<char *>(a->table) + tb, items.data(), ib, hipMemcpyHostToDevice);
        if (e == hipSuccess)
            e = hipMemcpy(static_cast<char *>(a->table) + tb + ib, zeros.data(), cb, hipMemcpyHostToDevice);
        if (e != hipSuccess) {
            if (a->table) (void)hipFree(a->table);
            delete a;
            return hip_fail(e, "optimizer table");
        }
        a->items = reinterpret_cast<Item *>(static_cast<char *>(a->table) + tb);
        a->counters = reinterpret_cast<unsigned *>(static_cast<char *>(a->table) + tb + ib);
    }
    *handle = a;
    return CGTP_OK;
}

}  // namespace

extern "C" int cgtp_adamw_create(int n_tensors, const cgtp_adamw_tensor *tensors, int grad_dtype,
                                 int state_bits, cgtp_adamw *handle)
{
    cgtp::clear_error();
    if (!handle) return report(CGTP_ERR_ARG, "handle is NULL");
    *handle = nullptr;
    if (n_tensors < 1 || !tensors) return report(CGTP_ERR_ARG, "no tensors");
    if (grad_dtype != CGTP_F32 && grad_dtype != CGTP_BF16)
        return report(CGTP_ERR_ARG, "grad_dtype %d is neither CGTP_F32 nor CGTP_BF16", grad_dtype);
    if (state_bits != 8 && state_bits != 32)
        return report(CGTP_ERR_ARG, "state_bits %d is neither 8 nor 32", state_bits);
    try {
        return create(n_tensors, tensors, grad_dtype, state_bits, handle);
    } catch (const std::exception &ex) {
        return report(CGTP_ERR_HIP, "host memory: %s", ex.what());
    }
}

extern "C" int cgtp_adamw_step(cgtp_adamw a, double lr, double beta1, double beta2, double eps,
                               double weight_decay, int64_t step, const float *grad_scale,
                               void *stream)
{
    cgtp::clear_error();
    const int st = check_handle(a);
    if (st != CGTP_OK) return st;
    if (!(std::isfinite(lr) && std::isfinite(weight_decay) && std::isfinite(eps) && eps >= 0 &&
          beta1 >= 0 && beta1 < 1 && beta2 >= 0 && beta2 < 1 && step >= 1))
        return report(CGTP_ERR_ARG, "lr %g, beta1 %g, beta2 %g, eps %g, weight_decay %g, step %lld",
                      lr, beta1, beta2, eps, weight_decay, (long long)step);
    if (!aligned(grad_scale, 4)) return report(CGTP_ERR_ARG, "grad_scale is not 4-byte aligned");
    if (a->n_items == 0) return CGTP_OK;
    const double c1 = 1 - std::pow(beta1, (double)step), c2 = 1 - std::pow(beta2, (double)step);
    const Hyper h = {(float)(1 - lr * weight_decay), (float)beta1,  (float)(1 - beta1),
                     (float)beta2,                   (float)(1 - beta2), (float)(lr / c1),
                     (float)(1 / c2),                (float)eps};
    const Tensor *tensors = static_cast<const Tensor *>(a->table);
    auto *kernel = past_caches(a->n_items, a->state_bits == 8 ? 16 : 28)
                       ? pick<true>(a->grad_dtype, a->state_bits) : pick<false>(a->grad_dtype, a->state_bits);
    hipLaunchKernelGGL(kernel, dim3((unsigned)a->n_items), dim3(kThreads), 0,
                       static_cast<hipStream_t>(stream), tensors, a->items, h, grad_scale);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? CGTP_OK : hip_fail(e, "adamw step");
}

extern "C" int cgtp_adamw_states(cgtp_adamw a, float *const *m_out, float *const *v_out, void *stream)
{
    cgtp::clear_error();
    const int st = check_handle(a);
    if (st != CGTP_OK) return st;
    if (a->state_bits != 8) return report(CGTP_ERR_ARG, "the states are held in 32 bits");
    if (!m_out || !v_out) return report(CGTP_ERR_ARG, "m_out or v_out is NULL");
    for (int i = 0; i < a->n_tensors; ++i)
        if (a->first_item[i + 1] > a->first_item[i] &&
            (!m_out[i] || !v_out[i] || !aligned(m_out[i], 4) || !aligned(v_out[i], 4)))
            return report(CGTP_ERR_ARG, "m_out or v_out of tensor %d is NULL or misaligned", i);
    for (int t0 = 0; t0 < a->n_tensors; t0 += kStatesMax) {
        const int t1 = t0 + kStatesMax < a->n_tensors ? t0 + kStatesMax : a->n_tensors;
        const int64_t i0 = a->first_item[t0], n = a->first_item[t1] - i0;
        if (n == 0) continue;
        Outs outs{};
        for (int i = t0; i < t1; ++i) {
            outs.m[i - t0] = m_out[i];
            outs.v[i - t0] = v_out[i];
        }
        auto *kernel = past_caches(n, 10) ? k_adamw_states<true> : k_adamw_states<false>;
        hipLaunchKernelGGL(kernel, dim3((unsigned)n), dim3(kThreads), 0,
                           static_cast<hipStream_t>(stream), static_cast<const Tensor *>(a->table),
                           a->items + i0, t0, outs);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return hip_fail(e, "adamw states");
    }
    return CGTP_OK;
}

namespace {

int norm_blocks(const cgtp_adamw_s *a) { return a->n_items < 1 ? 1 : a->n_items < kNormBlocks ? (int)a->n_items : kNormBlocks; }
size_t norm_bytes(const cgtp_adamw_s *a) { return norm_blocks(a) > 1 ? sizeof(double) * (size_t)norm_blocks(a) : 0; }

}  // namespace

extern "C" int cgtp_adamw_grad_norm_bytes(cgtp_adamw a, size_t *bytes)
{
    cgtp::clear_error();
    if (!a) return report(CGTP_ERR_ARG, "handle is NULL");
    if (!bytes) return report(CGTP_ERR_ARG, "bytes is NULL");
    *bytes = norm_bytes(a);
    return CGTP_OK;
}

extern "C" int cgtp_adamw_grad_norm(cgtp_adamw a, double max_norm, const float *grad_scale, float *norm, float *scale,
                                    void *workspace, size_t ws_bytes, void *stream)
{
    cgtp::clear_error();
    const int st = check_handle(a);
    if (st != CGTP_OK) return st;
    if (!(max_norm > 0)) return report(CGTP_ERR_ARG, "max_norm %g", max_norm);
    if (!norm && !scale) return report(CGTP_ERR_ARG, "norm and scale are both NULL");
    if (!aligned(norm, 4) || !aligned(scale, 4) || !aligned(grad_scale, 4))
        return report(CGTP_ERR_ARG, "norm, scale or grad_scale is not 4-byte aligned");
    const size_t need = norm_bytes(a);
    if (need > 0 && !workspace) return report(CGTP_ERR_WORKSPACE, "no workspace, %zu bytes needed", need);
    if (!aligned(workspace, 256)) return report(CGTP_ERR_ARG, "workspace %p is not 256-byte aligned", workspace);
    if (ws_bytes < need) return report(CGTP_ERR_WORKSPACE, "workspace of %zu bytes, %zu needed", ws_bytes, need);
    auto *kernel = a->grad_dtype == CGTP_BF16 ? k_grad_norm<bf16_t> : k_grad_norm<float>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)norm_blocks(a)), dim3(kThreads), 0, static_cast<hipStream_t>(stream),
                       static_cast<const Tensor *>(a->table), a->items, a->n_items, static_cast<double *>(workspace),
                       a->counters, max_norm, grad_scale, norm, scale);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? CGTP_OK : hip_fail(e, "gradient norm");
}

extern "C" int cgtp_adamw_destroy(cgtp_adamw a)
{
    cgtp::clear_error();
    if (!a) return CGTP_OK;
    hipError_t e = hipDeviceSynchronize();
    if (a->table) {
        const hipError_t f = hipFree(a->table);
        if (e == hipSuccess) e = f;
    }
    delete a;
    return e == hipSuccess ? CGTP_OK : hip_fail(e, "adamw destroy");
}
