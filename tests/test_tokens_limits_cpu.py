"""The token operators at the ends of their ranges: what a kernel's 32-bit arithmetic cannot hold is refused before anything touches the device."""
import ctypes
import os
import subprocess

import pytest

from paper_2512_02371_amd import hb

P = ctypes.c_void_p(0x1000)                               # never dereferenced
ROOM = ctypes.c_void_p(0x10000)
UNSUPPORTED = hb.HB_ERR_UNSUPPORTED
MOST = 0x7fffff00                                         # 2^31 - 256: a tile, or three of keys, past the end still fit


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(hb.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return hb.load()


def attention(lib, fn, B=1, Lq=1, Lk=1, Hq=1, Hkv=1, D=8, mask=None):
    # strides of 0 (broadcast): a long row of keys takes no memory
    return getattr(lib, fn)(P, P, P, P, B, Lq, Lk, Hq, Hkv, D, *[0] * 12, 1.0, None, mask, 0, ROOM, 1 << 40, None)


@pytest.mark.parametrize("fn", ["hb_attention", "hb_attention_valu"])
@pytest.mark.parametrize("Lk", [MOST + 1, (1 << 31) - 192, (1 << 31) - 64, (1 << 31) - 1])
@pytest.mark.parametrize("mask", [None, P])
def test_more_keys_than_tile_numbers_hold(lib, fn, Lk, mask):
    assert attention(lib, fn, Lk=Lk, mask=mask) == UNSUPPORTED
    assert lib.hb_attention_workspace_size(1, 1, Lk, 1, 1, 8) == 0


def test_attention_launches_of_2_to_the_32_threads(lib):
    # 256 threads a workgroup, one for each key head of a short sequence
    assert attention(lib, "hb_attention", B=1 << 24) == UNSUPPORTED
    assert attention(lib, "hb_attention", B=1 << 21, Hq=8, Hkv=8) == UNSUPPORTED
    assert attention(lib, "hb_attention", B=(1 << 31) - 1, Hq=64, Hkv=64) == UNSUPPORTED
    # the twin: four rows a workgroup
    assert attention(lib, "hb_attention_valu", B=1 << 26) == UNSUPPORTED
    assert attention(lib, "hb_attention_valu", B=1 << 20, Hq=64, Hkv=1) == UNSUPPORTED
    assert attention(lib, "hb_attention_valu", B=(1 << 31) - 1, Hq=64, Hkv=64, Lq=1 << 20) == UNSUPPORTED
    # products of sizes beyond 64 bits
    assert attention(lib, "hb_attention", B=1 << 30, Lq=1 << 30, Hq=1 << 10, Hkv=1 << 10) == UNSUPPORTED
    assert attention(lib, "hb_attention_valu", B=1 << 30, Lq=1 << 30, Hq=1 << 10, Hkv=1 << 10) == UNSUPPORTED
    assert lib.hb_attention_workspace_size(1 << 30, 1 << 30, 1 << 20, 1 << 10, 1 << 10, 64) == 0


@pytest.mark.parametrize("interleaved", [0, 1])
def test_rope_launches_of_2_to_the_32_threads(lib, interleaved):
    def call(x, B, L, D, pairs, strides=0):
        return lib.hb_rope_axes(x, x, P, P, B, L, 1, D, strides, strides, strides, strides, strides, strides, 0, 0, (ctypes.c_int32 * 1)(pairs), 1, interleaved, None)
    assert call(P, 1 << 16, 1 << 16, 16, 8) == UNSUPPORTED                                       # a thread or two for each token
    assert call(P, 1 << 14, 1 << 14, 32, 16, 1) == UNSUPPORTED                                   # odd strides: a thread for each pair
    assert call(P, (1 << 31) - 1, (1 << 31) - 1, 65536, 8) == UNSUPPORTED                        # the product passes 64 bits


@pytest.mark.parametrize("fn", ["hb_linear", "hb_linear_valu"])
@pytest.mark.parametrize("M", [MOST + 1, (1 << 31) - 1])
def test_linear_rows_within_a_tile_of_2_to_the_31(lib, fn, M):
    for N, K in ((1, 1), (64, 64), (300, 300)):
        assert getattr(lib, fn)(P, P, None, None, P, 0, 0, M, N, K, K, K, N, N, None, 0, None) == UNSUPPORTED


def test_linear_launches_of_2_to_the_32_threads(lib):
    assert lib.hb_linear_valu(P, P, None, None, P, 0, 0, 1 << 30, 64, 64, 64, 64, 64, 64, None, 0, None) == UNSUPPORTED
    assert lib.hb_linear(P, P, None, None, P, 0, 0, 1 << 30, 1 << 20, 64, 64, 64, 1 << 20, 1 << 20, None, 0, None) == UNSUPPORTED


PROGRAM = r"""
#include <cstdio>
#include <initializer_list>
#include "linear_plan.hpp"
int main() {
    int M, N, K;
    while (scanf("%d %d %d", &M, &N, &K) == 3) {
        for (hb::LinRows rows : {hb::kLinCopied, hb::kLinEven, hb::kLinOdd}) printf("%d ", hb::linear_plan(M, N, K, rows).kernel);
        printf("\n");
    }
}
"""


def test_linear_takes_a_kernel_whose_launch_holds_the_rows(tmp_path):
    """Feature maps of up to 2^31 - 256 pixels and 64 channels: outputs and threads of a workgroup of the chosen kernel."""
    (tmp_path / "plan.cpp").write_text(PROGRAM)
    csrc = os.path.join(os.path.dirname(hb.LIB_PATH), "csrc")
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-I", csrc, str(tmp_path / "plan.cpp"), "-o", str(tmp_path / "plan")])
    shapes = [(M, N, K) for M in (1 << 28, (1 << 29) - 64, 1 << 29, 1 << 30, MOST) for N in (1, 16, 64) for K in (1, 64, 65, 128, 200, 1024)]
    out = subprocess.run([str(tmp_path / "plan")], input="\n".join("%d %d %d" % s for s in shapes), capture_output=True, text=True, check=True).stdout
    workgroup = {3: (64, 64, 512), 4: (128, 64, 256), 5: (128, 128, 512)}
    for (M, N, K), kernels in zip(shapes, out.splitlines()):
        for kernel in map(int, kernels.split()):
            m, n, size = workgroup[kernel]
            assert -(-M // m) * -(-N // n) * size < 1 << 32, (M, N, K, kernel)


@pytest.mark.parametrize("H", [(1 << 31) - (1 << 20) + 1, (1 << 31) - 1])
def test_rope_heads_that_the_loop_cannot_count(lib, H):
    """A thread goes on by four times the threads of a token at most (2^20): beyond 2^31 - 2^20 heads that passed 32 bits, and the place became negative."""
    sections = (ctypes.c_int32 * 1)(1)
    for stride in (0, 1, 8):
        assert lib.hb_rope_axes(P, P, P, P, 1, 1, H, 2, 0, 0, stride, 0, 0, stride, 0, 0, sections, 1, 0, None) == UNSUPPORTED


@pytest.mark.parametrize("n", [1 << 31, (1 << 32) + 1, (1 << 40) + 64])
def test_sizes_beyond_an_int_are_not_cut_off(lib, n):
    """A size goes to the library as an int: what does not fit must not arrive as its low 32 bits."""
    for f, args in ((hb.hb_linear_workspace_size, (64, 512, 8192)), (hb.hb_attention_workspace_size, (1, 1, 16384, 8, 1, 128))):
        assert f(*args) > 0
        for i in range(len(args)):
            with pytest.raises(AssertionError):
                f(*args[:i], n, *args[i + 1:])
