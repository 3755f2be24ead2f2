"""The GPU tests of hb_attention's forms take every kernel that its choice by size can take."""
import random
import subprocess

import os

from attentiontest import FORMS, instance

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2512_02371_amd", "csrc")
PROGRAM = r"""
#include <cstdio>
#include <initializer_list>
#include "attention_plan.hpp"
int main() {
    int B, Lq, Lk, Hq, Hkv, D;
    while (scanf("%d %d %d %d %d %d", &B, &Lq, &Lk, &Hq, &Hkv, &D) == 6) {
        const hb::AttentionPlan p = hb::attention_plan(B, Lq, Lk, Hq, Hkv, D);
        printf("%d %d\n", p.parts, p.groups);
    }
}
"""


def test_every_form_is_tested(tmp_path):
    (tmp_path / "plan.cpp").write_text(PROGRAM)
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-I", CSRC, str(tmp_path / "plan.cpp"), "-o", str(tmp_path / "plan")])

    def taken(calls):
        out = subprocess.run([str(tmp_path / "plan")], input="\n".join("%d %d %d %d %d %d" % c for c in calls), capture_output=True, text=True, check=True).stdout
        return {instance(*map(int, l.split()), c[1], *c[3:]) for c, l in zip(calls, out.splitlines())}
    rng = random.Random(1)
    size = lambda most: max(1, int(most ** rng.random()))
    calls = []
    for _ in range(60000):
        Hkv = size(32)
        calls.append((size(64), size(1 << 13), size(1 << 15), Hkv * size(16), Hkv, 8 * rng.randint(1, 16)))
    reached, tested = taken(calls), taken(FORMS)
    assert len(reached) >= 20 and reached <= tested, sorted(reached - tested)
