// Launches of the wide products and of adapters with them (rows_wide.h).
#include "rows_wide.h"

namespace cgtp {

namespace {

using namespace rows;

template <typename T, bool WNK, int NP, int XP, bool FUSED, bool WHOLE, bool LINES, Extra EX = kBare>
hipError_t launch(const RowOrder &o, const RowProduct &p, hipStream_t s)
{
    const int64_t tiles = XP > 0 && !FUSED ? (o.n + kRows - 1) / kRows : o.n / kRows + o.G + 1;
    const WideGrid g = wide_grid(tiles, p.N);
    hipLaunchKernelGGL((k_row_wide<T, WNK, NP, XP, FUSED, WHOLE, LINES, EX, false, false>), g.grid, dim3(kThreads), 0, s, o, p,
                       g.splits);
    return hipGetLastError();
}

template <typename T, int NP, bool WHOLE, bool LINES>
hipError_t with_pairs(const RowOrder &o, const RowProduct &p, hipStream_t s)
{
    if constexpr (sizeof(T) == 2)
        if (p.slope_z) return launch<T, true, NP, 0, false, WHOLE, LINES, kGradZ>(o, p, s);
    if (!p.h && !p.a)
        return p.w_nk ? launch<T, true, NP, 0, false, WHOLE, LINES>(o, p, s)
                      : launch<T, false, NP, 0, false, WHOLE, LINES>(o, p, s);
    constexpr int X = kExtPairs<T>;
    const bool half = kNarrow<T> * narrow_width(p.r) <= X * kU;
    if (p.a)
        return half ? launch<T, false, NP, X / 2, true, WHOLE, LINES>(o, p, s)
                    : launch<T, false, NP, X, true, WHOLE, LINES>(o, p, s);
    return half ? launch<T, false, NP, X / 2, false, WHOLE, LINES>(o, p, s)
                : launch<T, false, NP, X, false, WHOLE, LINES>(o, p, s);
}

template <typename T, bool WHOLE, bool LINES>
hipError_t with_rows(const RowOrder &o, const RowProduct &p, hipStream_t s)
{
    constexpr int M = kPairs<T>;
    if (p.K <= M / 4 * 2 * kU) return with_pairs<T, M / 4, WHOLE, LINES>(o, p, s);
    if (p.K <= M / 2 * 2 * kU) return with_pairs<T, M / 2, WHOLE, LINES>(o, p, s);
    return with_pairs<T, M, WHOLE, LINES>(o, p, s);
}

template <typename T> hipError_t pick(const RowOrder &o, const RowProduct &p, hipStream_t s)
{
    if (by_lines<T>(p.out, p.out_stride, p.N)) return with_rows<T, true, true>(o, p, s);
    if (by_fours<T>(p.out, p.out_stride, p.N)) return with_rows<T, true, false>(o, p, s);
    return with_rows<T, false, false>(o, p, s);
}

template <typename T> bool takes(const RowProduct &p)
{
    if (p.narrow || p.N <= kCols || p.K > 2 * kPairs<T> * kU) return false;
    if (!p.h && !p.a) return p.w_group != 0 && (!p.w_nk || p.K >= kU);
    return !p.w_nk && kNarrow<T> * narrow_width(p.r) <= 2 * kExtPairs<T> * kU;
}

}  // namespace

// z, where it is kept, lies on lines as the results do, or both on whole ones.
template <typename T> bool layer_takes(const RowProduct &p)
{
    const bool z_fits = !p.z || (p.z_stride == p.out_stride && (reinterpret_cast<uintptr_t>(p.z) - reinterpret_cast<uintptr_t>(p.out)) % 128 == 0) ||
                        (by_lines<T>(p.out, p.out_stride, p.N) && by_lines<T>(p.z, p.z_stride, p.N));
    return p.N >= kCols && p.K <= 2 * kPairs<T> * kU && !p.w_nk && z_fits;
}

bool layer_wide_takes(int dtype, const RowProduct &p) { return dtype == CGTP_BF16 ? layer_takes<bf16_t>(p) : layer_takes<float>(p); }

hipError_t launch_layer_wide(int dtype, const RowOrder &o, const RowProduct &p, hipStream_t s)
{
    return dtype == CGTP_BF16 ? launch_layer_wide_bf16(o, p, s) : launch_layer_wide_f32(o, p, s);
}

bool row_wide_takes(int dtype, const RowProduct &p)
{
    return dtype == CGTP_BF16 ? takes<bf16_t>(p) : takes<float>(p);
}

// Tiles of one adapter each.
bool adapter_wide_takes(int dtype, const RowOrder &o, const RowProduct &p)
{
    return p.a && !p.h_out && own_tiles(o) && row_wide_takes(dtype, p);
}

hipError_t launch_row_wide(int dtype, const RowOrder &o, const RowProduct &p, hipStream_t s)
{
    return dtype == CGTP_BF16 ? pick<bf16_t>(o, p, s) : pick<float>(o, p, s);
}

}  // namespace cgtp
