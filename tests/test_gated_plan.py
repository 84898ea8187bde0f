"""Which kernel a gated pair takes, compiled by itself: no launch of 2^32 threads or more, whatever the sizes, and the choice at ordinary ones."""
import random
import subprocess

import pytest

from paper_2309_03824_amd import build

SOURCE = r'''
#include <cstdio>
#include "gated_plan.hpp"
int main()
{
    long long T, out, r;
    int padded, bf16;
    while (scanf("%lld %lld %lld %d %d", &T, &out, &r, &padded, &bf16) == 5) printf("%d\n", (int)lrd::gated_route(T, out, r, padded, bf16, 1 << 22));
}
'''
DIRECT_16, DIRECT_32, WIDE, DEEP, TILES = range(5)


@pytest.fixture(scope="module")
def route(tmp_path_factory):
    at = tmp_path_factory.mktemp("plan")
    (at / "plan.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", build.CSRC, str(at / "plan.cpp"), "-o", str(at / "plan")], check=True)

    def ask(cases):
        out = subprocess.run([str(at / "plan")], input="".join("%d %d %d %d %d\n" % c for c in cases), capture_output=True, text=True, check=True).stdout
        return [int(v) for v in out.split()]
    return ask


def up(a, b):
    return -(-a // b)


def test_no_launch_has_2_32_threads(route):
    rng = random.Random(2)
    cases = [(T, out, r, p, 1) for T in (2**30 + 1, 2**31 - 128, 2**31 - 1) for out in (1, 8, 9, 64, 65, 128, 129, 2**24 - 1, 2**24 - 8) for r in (8, 512, 520) for p in (0, 1)]
    cases += [(int(2 ** (rng.random() * 31)), int(2 ** (rng.random() * 24)), int(2 ** (rng.random() * 13)) // 8 * 8 + 8, rng.randrange(2), rng.randrange(2)) for _ in range(2000)]
    seen = set()
    for (T, out, r, padded, bf16), how in zip(cases, route(cases)):
        threads = {DIRECT_16: up(T, 16) * up(out, 16) * 512, DIRECT_32: up(T, 32) * up(out, 32) * 256, WIDE: up(T, 128) * up(out, 64) * 256,
                   DEEP: up(T, 128) * up(out, 128) * 512, TILES: 0}[how]
        assert threads < 2**32, (T, out, r, padded, bf16, how)
        assert bf16 or how in (DIRECT_16, DIRECT_32, TILES)
        seen.add(how)
    assert len(seen) == 5


def test_the_choice_at_ordinary_sizes(route):
    cases = [((1, 4096, 256, 0, 1), DIRECT_16), ((64, 4096, 256, 0, 1), DIRECT_32), ((256, 4096, 256, 0, 1), WIDE), ((512, 1024, 256, 0, 1), DIRECT_32), ((8192, 4096, 256, 0, 1), WIDE),
             ((8192, 4096, 1024, 0, 1), DEEP), ((8192, 2730, 256, 0, 1), DEEP), ((8192, 2730, 256, 1, 1), DEEP), ((8192, 4096, 257, 0, 1), TILES), ((512, 2048, 256, 0, 0), DIRECT_32),
             ((1024, 2048, 256, 0, 0), TILES), ((8192, 4194304, 8, 0, 1), WIDE), ((8192, 4194312, 8, 0, 1), DEEP)]
    assert route([c for c, _ in cases]) == [how for _, how in cases]
