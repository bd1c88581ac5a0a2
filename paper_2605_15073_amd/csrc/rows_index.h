// Index arithmetic of the row products: the grid of their tiles, and which weights a thread of the wide ones
// (rows_wide.hip) loads. Plain integers, shared by the kernels and compiled by themselves in a host test.
#pragma once

#include <cstdint>

#ifndef CGTP_HD
#ifdef __HIPCC__
#define CGTP_HD __host__ __device__
#else
#define CGTP_HD
#endif
#endif

namespace cgtp {
namespace rows {

// Workgroups of a launch for `tiles` tiles: one dimension holds fewer than 2^32 threads, so that they are cut over
// x and z; tile x + z * (size in x), which may lie past the last one.
struct TileGrid {
    unsigned x, z;
};
CGTP_HD constexpr TileGrid tile_grid(int64_t tiles)
{
    constexpr int64_t most = 1 << 23;
    const int64_t x = tiles < most ? tiles : most;
    return {(unsigned)x, (unsigned)((tiles + x - 1) / x)};
}
CGTP_HD constexpr int64_t tile_at(unsigned x, unsigned z, unsigned size_x) { return x + (int64_t)z * size_x; }

constexpr int kWideThreads = 256;
constexpr int kWideCols = 64;  // columns of a tile

// Rounds in which the threads load a tile's units, and the unit of a thread: the last one again past the end
// (loads are not under a condition; such a thread stages none).
CGTP_HD constexpr int wide_rounds(int units) { return (units + kWideThreads - 1) / kWideThreads; }
CGTP_HD constexpr int wide_unit(int thread, int round, int units)
{
    const int u = thread + kWideThreads * round;
    return u < units ? u : units - 1;
}

// The first column of tile ct of N >= kWideCols: the last tile ends with the rows.
CGTP_HD constexpr int wide_first_col(int ct, int N)
{
    return ct * kWideCols + kWideCols <= N ? ct * kWideCols : N - kWideCols;
}

// Where the load of eight values from k on starts in a row of K >= 8.
CGTP_HD constexpr int start8(int k, int K) { return k + 8 <= K ? k : K - 8; }

}  // namespace rows
}  // namespace cgtp
