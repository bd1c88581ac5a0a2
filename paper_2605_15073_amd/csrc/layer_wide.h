// Launches of layers with short inputs and wide outputs (rows_wide.h), of which each type has a source of its own.
#ifndef CGTP_LAYER_WIDE_H
#define CGTP_LAYER_WIDE_H

#include "rows_wide.h"

namespace cgtp {
namespace rows {

template <typename T, int NP, bool WHOLE, bool LINES, bool Z, bool RES>
hipError_t launch_wide(const RowOrder &o, const RowProduct &p, hipStream_t s)
{
    const int64_t per = tiles_per_xcd(o.n / kRows + o.G + 1);
    const WideGrid g = wide_grid(p.xcd_tiles > 0 ? kTileXcds * per : o.n / kRows + o.G + 1, p.N);
    RowProduct by_xcd = p;
    if (p.xcd_tiles > 0) by_xcd.xcd_tiles = per;
    hipLaunchKernelGGL((k_row_wide<T, false, NP, 0, false, WHOLE, LINES, kLayer, Z, RES>), g.grid, dim3(kThreads), 0, s, o, by_xcd,
                       g.splits);
    return hipGetLastError();
}

template <typename T, bool WHOLE, bool LINES, bool Z, bool RES>
hipError_t with_rows(const RowOrder &o, const RowProduct &p, hipStream_t s)
{
    constexpr int M = kPairs<T>;
    if (p.K <= M / 4 * 2 * kU) return launch_wide<T, M / 4, WHOLE, LINES, Z, RES>(o, p, s);
    if (p.K <= M / 2 * 2 * kU) return launch_wide<T, M / 2, WHOLE, LINES, Z, RES>(o, p, s);
    return launch_wide<T, M, WHOLE, LINES, Z, RES>(o, p, s);
}

template <typename T, bool WHOLE, bool LINES> hipError_t with_extras(const RowOrder &o, const RowProduct &p, hipStream_t s)
{
    if (p.z) return p.residual ? with_rows<T, WHOLE, LINES, true, true>(o, p, s) : with_rows<T, WHOLE, LINES, true, false>(o, p, s);
    return p.residual ? with_rows<T, WHOLE, LINES, false, true>(o, p, s) : with_rows<T, WHOLE, LINES, false, false>(o, p, s);
}

template <typename T> hipError_t launch_wide_layer(const RowOrder &o, const RowProduct &p, hipStream_t s)
{
    if (by_lines<T>(p.out, p.out_stride, p.N) && (!p.z || by_lines<T>(p.z, p.z_stride, p.N))) return with_extras<T, true, true>(o, p, s);
    if (by_fours<T>(p.out, p.out_stride, p.N)) return with_extras<T, true, false>(o, p, s);
    return with_extras<T, false, false>(o, p, s);
}

}  // namespace rows
}  // namespace cgtp

#endif
