"""How a block norm's backward deals rows to workgroups, compiled by itself: every row in one unit, no unit across two rows of the
gate, and partial rows inside the workspace."""
import random
import subprocess

import pytest

from paper_2309_03824_amd import build

SOURCE = r'''
#include <cstdio>
#include "block_plan.hpp"
int main()
{
    long long T, d, g;
    while (scanf("%lld %lld %lld", &T, &d, &g) == 3) {
        const lrd::BlockNormPlan p = lrd::block_norm_plan(T, d, g);
        printf("%lld %lld %lld %lld %lld %d %lld %lld\n", (long long)p.gate_rows, (long long)p.units, (long long)p.parts, (long long)p.part_rows,
               (long long)p.workgroups, (int)p.by_slot, (long long)lrd::block_norm_most_workgroups(T), (long long)lrd::block_norm_most_units(T));
    }
}
'''


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    at = tmp_path_factory.mktemp("plan")
    (at / "plan.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", build.CSRC, str(at / "plan.cpp"), "-o", str(at / "plan")], check=True)

    def ask(cases):
        text = "".join("%d %d %d\n" % c for c in cases)
        out = subprocess.run([str(at / "plan")], input=text, capture_output=True, text=True, check=True).stdout
        return [tuple(int(v) for v in line.split()) for line in out.splitlines()]
    return ask


def test_every_row_is_dealt_once(plan):
    rng = random.Random(5)
    cases = [(T, d, g) for T in list(range(1, 40)) + [511, 512, 513, 4100, 8192, 100001] for d in (64, 513, 1024, 1025, 3000, 16384) for g in (0, 1, 2, 15, 16, 17, 18, 512, T - 1, T, T + 1)]
    cases += [(int(2 ** (rng.random() * 17)) + 1, rng.choice((8, 4096)), int(2 ** (rng.random() * 17))) for _ in range(300)]
    for (T, d, g), (rows, units, parts, part_rows, workgroups, by_slot, most_w, most_u) in zip(cases, plan(cases)):
        what = (T, d, g)
        assert rows == (g if 0 < g < T else T), what
        groups = -(-T // rows)
        assert units == groups * parts and 1 <= workgroups <= min(units, most_w), what
        assert parts == 1 or units <= most_u, what
        assert not by_slot or (parts == 1 and part_rows == rows), what
        seen = 0
        for u in range(units):
            group, part = divmod(u, parts)
            r0 = group * rows + part * part_rows
            r1 = min(r0 + part_rows, min((group + 1) * rows, T))
            if r1 > r0:
                assert r0 == seen, what
                assert r0 // rows == (r1 - 1) // rows, what
                seen = r1
        assert seen == T, what


def test_the_largest_counts_of_tokens(plan):
    for (T, d, g), p in zip([(2 ** 31 - 1, 1024, 0), (2 ** 31 - 1, 8192, 1), (2 ** 31 - 1, 64, 4096), (2 ** 31 - 1, 64, 17)],
                            plan([(2 ** 31 - 1, 1024, 0), (2 ** 31 - 1, 8192, 1), (2 ** 31 - 1, 64, 4096), (2 ** 31 - 1, 64, 17)])):
        assert p[4] in (256, 512) and (p[2] == 1 or p[1] <= p[7]) and p[2] * p[3] >= p[0], (T, d, g, p)
