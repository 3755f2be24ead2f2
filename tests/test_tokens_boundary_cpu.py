"""The token operators' argument checks, which come before anything touches the device."""
import ctypes
import os

import numpy as np
import pytest

from paper_2512_02371_amd import hb

P, ODD, EIGHT = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1001), ctypes.c_void_p(0x1008)     # never dereferenced
INVALID, UNSUPPORTED, WORKSPACE = hb.HB_ERR_INVALID_ARG, hb.HB_ERR_UNSUPPORTED, hb.HB_ERR_WORKSPACE


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(hb.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return hb.load()


@pytest.mark.parametrize("fn", ["hb_linear", "hb_linear_valu"])
def test_linear(lib, fn):
    ok = dict(x=P, w=P, bias=None, residual=None, out=P, type=0, act=0, M=8, N=16, K=32, xp=32, wp=32, rp=16, op=16, ws=None, n=0)
    call = lambda **kw: getattr(lib, fn)(*{**ok, **kw}.values(), None)
    for bad in (dict(x=None), dict(w=None), dict(out=None), dict(M=0), dict(N=-1), dict(K=0), dict(xp=31), dict(wp=31), dict(op=15), dict(residual=P, rp=15), dict(type=2),
                dict(type=-1), dict(act=5), dict(act=-1), dict(x=ODD), dict(w=ODD), dict(bias=ODD), dict(out=ODD), dict(residual=ODD), dict(type=1, out=ctypes.c_void_p(0x1002)),
                dict(type=1, residual=ctypes.c_void_p(0x1002))):
        assert call(**bad) == INVALID, bad
    for bad in (dict(xp=hb.HB_LINEAR_MAX_PITCH + 1), dict(wp=hb.HB_LINEAR_MAX_PITCH + 1), dict(op=hb.HB_LINEAR_MAX_PITCH + 1), dict(residual=P, rp=hb.HB_LINEAR_MAX_PITCH + 1)):
        assert call(**bad) == UNSUPPORTED, bad
    assert lib.hb_linear_workspace_size(0, 1, 1) == lib.hb_linear_workspace_size(1, -1, 1) == lib.hb_linear_workspace_size(1, 1, 0) == 0


def test_linear_workspace(lib):
    shapes = [(1, 64, 8192), (64, 512, 8192), (100, 64, 5000), (512, 512, 8192), (8192, 8192, 2048)]
    for M, N, K in shapes:
        need = lib.hb_linear_workspace_size(M, N, K)
        args = [P, P, None, None, P, 0, 0, M, N, K, K, K, N, N]
        if need:
            assert need <= 1 << 28
            for ws, n in ((None, need), (ctypes.c_void_p(0x10000), need - 1), (ctypes.c_void_p(0x10010), need)):
                assert lib.hb_linear(*args, ws, n, None) == WORKSPACE


@pytest.mark.parametrize("fn", ["hb_attention", "hb_attention_valu"])
def test_attention(lib, fn):
    ok = dict(q=P, k=P, v=P, out=P, B=2, Lq=3, Lk=5, Hq=4, Hkv=2, D=64, qb=768, qt=256, qh=64, kb=640, kt=128, kh=64, vb=640, vt=128, vh=64, ob=768, ot=256, oh=64,
              scale=1.0, len=None, mask=None, pitch=0, ws=None, n=0)
    call = lambda **kw: getattr(lib, fn)(*{**ok, **kw}.values(), None)
    for bad in (dict(q=None), dict(k=None), dict(v=None), dict(out=None), dict(B=0), dict(Lq=0), dict(Lk=-1), dict(Hq=0), dict(Hkv=0), dict(D=0), dict(Hq=5), dict(q=EIGHT), dict(k=EIGHT),
                dict(v=EIGHT), dict(out=EIGHT), dict(qt=260), dict(kt=-8), dict(vh=4), dict(ob=1), dict(scale=float("nan")), dict(scale=float("-inf")), dict(len=ODD), dict(mask=P, pitch=-1)):
        assert call(**bad) == INVALID, bad
    for bad in (dict(D=60), dict(D=136), dict(kt=(1 << 20) + 8), dict(vt=(1 << 20) + 8)):
        assert call(**bad) == UNSUPPORTED, bad
    assert lib.hb_attention_workspace_size(0, 1, 1, 1, 1, 64) == lib.hb_attention_workspace_size(1, 1, 1, 3, 2, 64) == lib.hb_attention_workspace_size(1, 1, 0, 1, 1, 64) == 0


def test_attention_workspace(lib):
    for B, Lq, Lk, Hq, Hkv, D in ((1, 1, 16384, 8, 1, 128), (4, 1, 16384, 32, 8, 128), (1, 3, 5000, 2, 2, 64), (2, 4096, 4096, 16, 16, 64)):
        need = lib.hb_attention_workspace_size(B, Lq, Lk, Hq, Hkv, D)
        tq, tk = Hq * D, Hkv * D
        args = [P, P, P, P, B, Lq, Lk, Hq, Hkv, D, Lq * tq, tq, D, Lk * tk, tk, D, Lk * tk, tk, D, Lq * tq, tq, D, 1.0, None, None, 0]
        if need:
            assert need <= 1 << 28
            for ws, n in ((None, need), (ctypes.c_void_p(0x10000), need - 1), (ctypes.c_void_p(0x10010), need)):
                assert lib.hb_attention(*args, ws, n, None) == WORKSPACE


def test_rope(lib):
    def call(sections=(4, 4), **kw):
        ok = dict(x=P, out=P, pos=P, freq=P, B=2, L=3, H=4, D=16, xb=192, xt=64, xh=16, ob=192, ot=64, oh=16, pb=6, pt=2)
        a = np.array(sections, dtype=np.int32)
        s = kw.pop("ptr", a.ctypes.data_as(ctypes.c_void_p))
        return lib.hb_rope_axes(*{**ok, **kw}.values(), s, kw.get("axes", len(sections)), 0, None) if "axes" not in kw else \
            lib.hb_rope_axes(*{**ok, **{k: v for k, v in kw.items() if k != "axes"}}.values(), s, kw["axes"], 0, None)
    for bad in (dict(x=None), dict(out=None), dict(pos=None), dict(freq=None), dict(ptr=None), dict(B=0), dict(L=0), dict(H=0), dict(D=1), dict(axes=0), dict(x=ODD), dict(out=ODD),
                dict(pos=ctypes.c_void_p(0x1002)), dict(freq=ctypes.c_void_p(0x1002)), dict(xb=-1), dict(pt=-1), dict(sections=(5, 4)), dict(sections=(-1, 4)), dict(sections=(0, 0)),
                dict(sections=(1 << 30, 1 << 30, 1 << 30, 1 << 30))):
        assert call(**bad) == INVALID, bad
    assert call(sections=(1, 1, 1, 1, 1)) == UNSUPPORTED and call(D=65538) == UNSUPPORTED


def test_symbols_and_constants(lib):
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "hb.h")).read()
    for name, v in hb.HB_ACTS.items():
        assert f"HB_ACT_{name.upper()} = {v}" in text
    assert "HB_ATTENTION_MAX_D 128" in text and hb.HB_ATTENTION_MAX_D == 128 and "HB_ROPE_MAX_AXES 4" in text and hb.HB_ROPE_MAX_AXES == 4
    assert "HB_LINEAR_MAX_PITCH (1 << 21)" in text and hb.HB_LINEAR_MAX_PITCH == 1 << 21
