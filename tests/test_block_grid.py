"""The grid of a block norm's forward pass, compiled by itself: a workgroup for every row (or rows of a wave each), and less than 2^32 threads in a
dimension, however many tokens the call takes."""
import subprocess

from paper_2309_03824_amd import build

SOURCE = r'''
#include <cstdio>
#include "block_plan.hpp"
int main()
{
    long long rows;
    int threads;
    while (scanf("%lld %d", &rows, &threads) == 2) {
        const lrd::RowsGrid g = lrd::rows_grid(rows, threads);
        printf("%u %u\n", g.x, g.y);
    }
}
'''


def test_every_row_has_a_workgroup_and_no_dimension_2_32_threads(tmp_path):
    (tmp_path / "grid.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", build.CSRC, str(tmp_path / "grid.cpp"), "-o", str(tmp_path / "grid")], check=True)
    cases = []
    for T in [1, 2, 5, 8192, 2**22 - 1, 2**22, 2**22 + 1, 2**23 + 3, 2**24 - 1, 2**24, 2**24 + 1, 2**26 - 1, 2**26, 2**26 + 5, 2**31 - 2, 2**31 - 1]:
        cases += [(-(-T // 4), 256), (T, 256), (T, 512), (T, 1024)]
    out = subprocess.run([str(tmp_path / "grid")], input="".join("%d %d\n" % c for c in cases), capture_output=True, text=True, check=True).stdout.split()
    for (rows, threads), x, y in zip(cases, map(int, out[::2]), map(int, out[1::2])):
        assert x * threads < 2**32 and y < 2**16, (rows, threads, x, y)
        assert rows <= x * y < rows + y, (rows, threads, x, y)         # none without a workgroup, and less than one to spare in each row of the grid
        assert y == 1 or rows * threads >= 2**32, (rows, threads, x, y)
