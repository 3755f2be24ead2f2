"""The choices of hb_linear and hb_attention by size, compiled for the host: what they promise whatever the sizes."""
import random
import subprocess

import os
import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2512_02371_amd", "csrc")
PROGRAM = r"""
#include <cstdio>
#include <initializer_list>
#include "linear_plan.hpp"
#include "attention_plan.hpp"
using namespace hb;
int main() {
    char what;
    while (scanf(" %c", &what) == 1) {
        if (what == 'l') {
            int M, N, K;
            if (scanf("%d %d %d", &M, &N, &K) != 3) return 1;
            const size_t size = linear_workspace(M, N, K);
            for (LinRows rows : {kLinCopied, kLinEven, kLinOdd}) {
                const LinPlan p = linear_plan(M, N, K, rows);
                printf("%d %d %d %zu ", p.kernel, p.parts, p.steps, size);
            }
        } else {
            int B, Lq, Lk, Hq, Hkv, D;
            if (scanf("%d %d %d %d %d %d", &B, &Lq, &Lk, &Hq, &Hkv, &D) != 6) return 1;
            printf("%d %zu", attention_plan(B, Lq, Lk, Hq, Hkv, D).parts, attention_workspace(B, Lq, Lk, Hq, Hkv, D));
        }
        printf("\n");
    }
}
"""


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    d = tmp_path_factory.mktemp("plans")
    (d / "plans.cpp").write_text(PROGRAM)
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-Wall", "-I", CSRC, str(d / "plans.cpp"), "-o", str(d / "plans")])

    def run(lines):
        out = subprocess.run([str(d / "plans")], input="\n".join(lines), capture_output=True, text=True, check=True).stdout
        return [list(map(int, l.split())) for l in out.splitlines()]
    return run


def test_linear(ask):
    rng = random.Random(1)
    size = lambda most: max(1, int(most ** rng.random()))
    shapes = [(size(1 << 21), size(1 << 15), size(1 << 15)) for _ in range(3000)] + [(1, 1, 1), ((1 << 31) - 1, 1, 1), (1, (1 << 31) - 1, 1), (1, 1, 1 << 21), (1 << 30, 1 << 20, 64)]
    for (M, N, K), got in zip(shapes, ask(f"l {M} {N} {K}" for M, N, K in shapes)):
        steps = (K + 63) // 64
        for i in range(3):
            kernel, parts, per, need = got[4 * i:4 * i + 4]
            assert 0 <= kernel <= 6 and parts >= 1 and (parts - 1) * per < steps <= parts * per, (M, N, K)        # no part is empty, none is missing
            assert kernel >= 3 or M <= (16, 32, 64)[kernel]
            assert kernel != 6 or (i == 0 and parts == 1)
            assert parts == 1 or parts * M * N * 4 <= need <= 1 << 28, (M, N, K, parts, need)
            assert need % 256 == 0


def test_attention(ask):
    rng = random.Random(2)
    size = lambda most: max(1, int(most ** rng.random()))
    shapes = []
    for _ in range(3000):
        Hkv = size(32)
        shapes.append((size(64), size(1 << 14), size(1 << 17), Hkv * size(16), Hkv, 8 * rng.randint(1, 16)))
    shapes += [(1, 1, 1, 1, 1, 8), (1, 1, (1 << 31) - 1, 1, 1, 128), (1, (1 << 31) - 256, 1, 1, 1, 64)]
    for s, (parts, need) in zip(shapes, ask("a " + " ".join(map(str, s)) for s in shapes)):
        B, Lq, Lk, Hq, Hkv, D = s
        assert 1 <= parts <= 64 and parts <= (Lk + 63) // 64
        assert need == (0 if parts == 1 else (parts * B * Hq * Lq * (D + 2) * 4 + 255) // 256 * 256), s
        assert need <= 1 << 29
