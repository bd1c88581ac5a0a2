"""CPU test of the index arithmetic of the row products (csrc/rows_index.h): every weight that a thread can load lies
inside its group's weights, every unit of a tile is some thread's, and every tile some workgroup's."""
from __future__ import annotations

import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(__file__)), "paper_2605_15073_amd", "csrc")

PROGRAM = r"""
#include "rows_index.h"
#include <cstdio>
#include <vector>
using namespace cgtp::rows;

static long long bad = 0, loads = 0;
static void fail(const char *what, int pairs, int K, int N, int ct, int thread)
{
    if (++bad <= 5) std::printf("%s: pairs %d K %d N %d tile %d thread %d\n", what, pairs, K, N, ct, thread);
}

int main()
{
    // [N][K] weights: pairs of k-groups as the kernel is built for, K that it takes with them
    for (int pairs : {1, 2, 4, 8})
        for (int K = 8; K <= 16 * pairs; ++K)
            for (int N : {65, 66, 127, 128, 129, 200, 896})
                for (int ct = 0; ct < (N + kWideCols - 1) / kWideCols; ++ct) {
                    const int KG = 2 * pairs, units = kWideCols * KG;
                    std::vector<int> staged((size_t)units, 0);
                    for (int thread = 0; thread < kWideThreads; ++thread)
                        for (int i = 0; i < wide_rounds(units); ++i) {
                            ++loads;
                            const int unit = wide_unit(thread, i, units), col = wide_first_col(ct, N) + unit / KG;
                            const int k = unit % KG * 8 < K ? unit % KG * 8 : 0, at = start8(k, K);
                            if (unit < 0 || unit >= units) fail("unit", pairs, K, N, ct, thread);
                            else if (unit == thread + kWideThreads * i) ++staged[(size_t)unit];
                            if (col < 0 || col >= N || at < 0 || at + 8 > K) fail("load", pairs, K, N, ct, thread);
                        }
                    for (int n : staged)
                        if (n != 1) fail("staged", pairs, K, N, ct, n);
                }
    // [K][N] weights: units of `wide` columns, of every number of k-groups
    for (int wide : {2, 4})
        for (int groups = 2; groups <= 28; groups += 2)
            for (int N : {65, 66, 127, 128, 129, 200, 896})
                for (int ct = 0; ct < (N + kWideCols - 1) / kWideCols; ++ct) {
                    const int units = kWideCols / wide * groups;
                    for (int thread = 0; thread < kWideThreads; ++thread)
                        for (int i = 0; i < wide_rounds(units); ++i) {
                            ++loads;
                            const int unit = wide_unit(thread, i, units);
                            const int col = wide_first_col(ct, N) + wide * (unit % (kWideCols / wide));
                            if (unit / (kWideCols / wide) >= groups) fail("group", groups, 0, N, ct, thread);
                            if (col < 0 || col + wide > N) fail("columns", groups, 0, N, ct, thread);
                        }
                }
    // grids: every tile is some workgroup's, and no dimension has 2^32 threads
    for (long long tiles : {1ll, 2ll, 1000ll, (1ll << 23) - 1, 1ll << 23, (1ll << 23) + 1, 1ll << 24, (1ll << 24) + 4097, 67112961ll}) {
        const TileGrid g = tile_grid(tiles);
        if ((long long)g.x * kWideThreads >= 1ll << 32 || g.z > 65535) fail("grid", 0, 0, 0, 0, (int)g.z);
        if (tile_at(0, 0, g.x) != 0 || tile_at(0, g.z - 1, g.x) >= tiles || tile_at(g.x - 1, g.z - 1, g.x) + 1 < tiles ||
            (g.z > 1 && tile_at(0, 1, g.x) != tile_at(g.x - 1, 0, g.x) + 1))
            fail("tiles", 0, 0, 0, 0, (int)g.z);
    }
    std::printf("%lld loads, %lld faults\n", loads, bad);
    return bad != 0;
}
"""


@pytest.mark.skipif(shutil.which("g++") is None, reason="no host compiler")
def test_wide_loads_stay_inside(tmp_path):
    src, exe = tmp_path / "index.cpp", tmp_path / "index"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    run = subprocess.run([str(exe)], capture_output=True, text=True, timeout=120)
    assert run.returncode == 0, run.stdout
