"""hb_quantize_rows: the choice of lanes by size, compiled for the host."""
import os
import random
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2512_02371_amd", "csrc")
PROGRAM = r"""
#include <cstdio>
#include "quantize_plan.hpp"
int main() {
    int M, K;
    while (scanf("%d %d", &M, &K) == 2) {
        const int lanes = hb::quantize_lanes(M, K);
        printf("%d %lld %d\n", lanes, (long long)hb::quantize_workgroups(M, lanes), hb::quantize_threads(lanes));
    }
}
"""
MOST_M, MOST_K = (1 << 24) - 1, (1 << 31) - (1 << 17)


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    folder = tmp_path_factory.mktemp("quantize")
    (folder / "plan.cpp").write_text(PROGRAM)
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-Wall", "-I", CSRC, str(folder / "plan.cpp"), "-o", str(folder / "plan")])

    def ask(calls):
        out = subprocess.run([str(folder / "plan")], input="\n".join("%d %d" % c for c in calls), capture_output=True, text=True, check=True).stdout
        return [tuple(map(int, l.split())) for l in out.splitlines()]
    return ask


def test_every_size_that_is_taken_can_be_launched(plan):
    """As many rows and values as include/hb.h allows: fewer than 2^32 lanes in a launch, and each row has its lanes."""
    rng = random.Random(1)
    edges_m = [1, 2, 63, 64, 1023, 1024, (1 << 22) - 1, 1 << 22, (1 << 22) + 1, 1 << 23, MOST_M]
    edges_k = [1, 8, 128, 129, 256, 257, 512, 513, 4096, 4097, 16384, 16385, 16392, 1 << 20, MOST_K]
    calls = [(m, k) for m in edges_m for k in edges_k] + [(max(1, int(MOST_M ** rng.random())), max(1, int(MOST_K ** rng.random()))) for _ in range(20000)]
    seen = set()
    for (M, K), (lanes, workgroups, threads) in zip(calls, plan(calls)):
        seen.add(lanes)
        assert lanes in (8, 16, 32, 64, 256, 1024) and threads == max(lanes, 256), (M, K)
        assert workgroups * threads < 1 << 32, (M, K, lanes)
        rows = threads // lanes
        assert (workgroups - 1) * rows < M <= workgroups * rows, (M, K)
    assert len(seen) == 6
