"""The GPU tests of hb_linear's forms take every kernel that its choice by size can take: a change of the cost model cannot leave one untested."""
import random
import subprocess

import os
import pytest

from lineartest import FORMS, ROWS, instance

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2512_02371_amd", "csrc")
PROGRAM = r"""
#include <cstdio>
#include <initializer_list>
#include "linear_plan.hpp"
int main() {
    int M, N, K, rows;
    while (scanf("%d %d %d %d", &M, &N, &K, &rows) == 4) {
        const hb::LinPlan p = hb::linear_plan(M, N, K, (hb::LinRows)rows);
        printf("%d %d %d\n", p.kernel, p.parts, p.steps);
    }
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("forms")
    (d / "plan.cpp").write_text(PROGRAM)
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-I", CSRC, str(d / "plan.cpp"), "-o", str(d / "plan")])

    def run(calls):
        text = "\n".join("%d %d %d %d" % (M, N, K, ROWS.index(rows)) for M, N, K, rows in calls)
        out = subprocess.run([str(d / "plan")], input=text, capture_output=True, text=True, check=True).stdout
        return [tuple(map(int, l.split())) for l in out.splitlines()]
    return run


def taken(calls, plans):
    return {instance(kernel, call[3]) + (parts > 1,) for call, (kernel, parts, _) in zip(calls, plans)}


def test_every_form_is_tested(plan):
    rng = random.Random(1)
    size = lambda most: max(1, int(most ** rng.random()))
    calls = []
    for _ in range(200000):
        M, N, K, rows = size(1 << 20), size(1 << 14), size(1 << 14), rng.choice(ROWS)
        if M * max(N, K) <= 1 << 27:
            calls.append((M, N, (K + 7) // 8 * 8 if rows == "copied" else K, rows))
    reached, tested = taken(calls, plan(calls)), taken(FORMS, plan(FORMS))
    assert len(reached) >= 20 and reached <= tested, sorted(reached - tested)
    assert all(rows != "copied" or K % 8 == 0 for _, _, K, rows in FORMS)


def test_steps_of_every_kind(plan):
    """One step, an even and an odd number, with and without a tail of K, in every kernel of tiles."""
    kinds = {}
    for (M, N, K, rows), (kernel, parts, steps) in zip(FORMS, plan(FORMS)):
        kinds.setdefault(instance(kernel, rows), set()).add((min(steps, 2), K % 64 != 0))
    for key in ((3, "copied"), (3, "even"), (3, "odd"), (4, "even"), (5, "copied"), (5, "odd"), (6, "copied")):
        assert any(s == 2 and tail for s, tail in kinds[key]), (key, kinds[key])
    for key in ((3, "copied"), (3, "even"), (3, "odd"), (4, "even"), (4, "odd"), (5, "copied")):
        assert any(s == 1 for s, _ in kinds[key]), (key, kinds[key])
