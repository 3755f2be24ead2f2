"""The token operators at the ends of their ranges: what a kernel's 32-bit arithmetic cannot hold is refused before anything touches the device."""
import ctypes
import os

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


@pytest.mark.parametrize("fn", ["hb_linear", "hb_linear_valu"])
@pytest.mark.parametrize("M", [MOST + 1, (1 << 31) - 1])
def test_linear_rows_within_a_tile_of_2_to_the_31(lib, fn, M):
    for N, K in ((1, 1), (64, 64), (300, 300)):
        assert getattr(lib, fn)(P, P, None, None, P, 0, 0, M, N, K, K, K, N, N, None, 0, None) == UNSUPPORTED
