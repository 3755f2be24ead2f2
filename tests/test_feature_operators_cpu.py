"""hb_group_norm, hb_quantize_rows and hb_linear_i8 on the host: their argument checks, which come before anything touches the device, and the oracle's
functions against closed forms and loops over their definitions."""
import ctypes
import math
import os
import re
from fractions import Fraction

import numpy as np
import pytest

import oracle
from paper_2512_02371_amd import hb

P, ODD, TWO = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1001), ctypes.c_void_p(0x1002)       # never dereferenced
INVALID, UNSUPPORTED, WORKSPACE = hb.HB_ERR_INVALID_ARG, hb.HB_ERR_UNSUPPORTED, hb.HB_ERR_WORKSPACE


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(hb.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return hb.load()


def test_the_integer_product_has_one_wrapper():
    """One shape, in one header: what test_matrix_builtins_appear_only_in_the_wrappers asks of the floating-point products."""
    package = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2512_02371_amd")
    assert os.listdir(os.path.join(package, "wrappers")) == ["mfma_i8.hpp"]
    text = re.sub(r"//[^\n]*", "", open(os.path.join(package, "wrappers", "mfma_i8.hpp")).read())
    assert re.findall(r"__builtin_amdgcn_\w+", text) == ["__builtin_amdgcn_mfma_i32_16x16x64_i8"] and "asm" not in text
    for name in os.listdir(os.path.join(package, "csrc")):
        text = re.sub(r"//[^\n]*", "", open(os.path.join(package, "csrc", name)).read())
        assert ("mfma16x16x64i8" in text) == (name == "linear_tiles.hpp"), name


def test_group_norm_arguments(lib):
    ok = dict(x=P, xt=0, w=None, b=None, out=P, ot=0, act=0, eps=1e-5, N=2, P=16, C=32, G=4, xi=512, xp=32, oi=512, op=32, ws=None, n=0)
    call = lambda **kw: lib.hb_group_norm(*{**ok, **kw}.values(), None)
    for bad in (dict(x=None), dict(out=None), dict(N=0), dict(P=0), dict(C=0), dict(G=0), dict(N=-1), dict(P=-5), dict(G=5), dict(G=33), dict(xt=2), dict(ot=-1), dict(act=5), dict(act=-1), dict(eps=0.0),
                dict(eps=-1e-5), dict(eps=float("nan")), dict(eps=float("inf")), dict(xp=31), dict(op=31), dict(xi=31), dict(oi=31), dict(xi=-512), dict(x=ODD), dict(out=ODD), dict(w=ODD),
                dict(b=ODD), dict(xt=1, x=TWO), dict(ot=1, out=TWO)):
        assert call(**bad) == INVALID, bad
    for bad in (dict(C=8192, G=1, xp=8192, op=8192, xi=8192 * 16, oi=8192 * 16), dict(C=1 << 30, G=1 << 29, N=2, P=1, xi=1 << 30, oi=1 << 30), dict(P=1 << 30, xi=1 << 40, oi=1 << 40)):
        assert call(**bad) == UNSUPPORTED, bad
    assert lib.hb_group_norm_workspace_size(0, 1, 1, 1) == lib.hb_group_norm_workspace_size(1, 0, 8, 2) == lib.hb_group_norm_workspace_size(1, 1, 8, 3) == lib.hb_group_norm_workspace_size(1, 1, 8, 0) == 0


def test_quantize_arguments(lib):
    ok = dict(x=P, q=P, s=P, M=4, K=32, xp=32, qp=32)
    call = lambda **kw: lib.hb_quantize_rows(*{**ok, **kw}.values(), None)
    for bad in (dict(x=None), dict(q=None), dict(s=None), dict(M=0), dict(K=0), dict(M=-1), dict(xp=31), dict(qp=31), dict(x=ODD), dict(s=TWO)):
        assert call(**bad) == INVALID, bad
    assert call(M=1 << 24) == UNSUPPORTED


@pytest.mark.parametrize("fn", ["hb_linear_i8", "hb_linear_i8_valu"])
def test_linear_i8_arguments(lib, fn):
    ok = dict(x=P, w=P, xs=P, ws=P, bias=None, residual=None, out=P, type=0, act=0, M=8, N=16, K=32, xp=32, wp=32, rp=16, op=16, wk=None, n=0)
    call = lambda **kw: getattr(lib, fn)(*{**ok, **kw}.values(), None)
    for bad in (dict(x=None), dict(w=None), dict(xs=None), dict(ws=None), dict(out=None), dict(M=0), dict(N=-1), dict(K=0), dict(xp=31), dict(wp=31), dict(op=15), dict(residual=P, rp=15), dict(type=2),
                dict(type=-1), dict(act=5), dict(act=-1), dict(xs=TWO), dict(ws=TWO), dict(bias=ODD), dict(out=ODD), dict(residual=ODD), dict(type=1, out=TWO), dict(type=1, residual=TWO)):
        assert call(**bad) == INVALID, bad
    big = hb.HB_LINEAR_MAX_PITCH + 1
    for bad in (dict(xp=big), dict(wp=big), dict(op=big), dict(residual=P, rp=big), dict(K=hb.HB_LINEAR_I8_MAX_K + 1, xp=1 << 20, wp=1 << 20), dict(M=0x7fffff01)):
        assert call(**bad) == UNSUPPORTED, bad
    assert lib.hb_linear_i8_workspace_size(0, 1, 1) == lib.hb_linear_i8_workspace_size(1, -1, 1) == lib.hb_linear_i8_workspace_size(1, 1, 0) == 0


def test_group_norm_oracle_against_loops():
    rng = np.random.default_rng(1)
    x, w, b = rng.normal(size=(2, 5, 6)) + 3.0, rng.normal(size=6), rng.normal(size=6)
    got = oracle.group_norm(x, 3, w, b, 1e-3, "silu")
    for n in range(2):
        for g in range(3):
            v = [x[n, p, c] for p in range(5) for c in (2 * g, 2 * g + 1)]
            mean = math.fsum(v) / 10
            var = math.fsum((t - mean) ** 2 for t in v) / 10
            for p in range(5):
                for c in (2 * g, 2 * g + 1):
                    y = (x[n, p, c] - mean) / math.sqrt(var + 1e-3) * w[c] + b[c]
                    assert abs(got[n, p, c] - y / (1 + math.exp(-y))) < 1e-13
    one = oracle.group_norm(x, 6, eps=1e-12)                                       # a channel of its own each
    assert np.allclose(one.mean(axis=1), 0, atol=1e-12) and np.allclose(one.var(axis=1), 1, atol=1e-6)
    assert np.array_equal(oracle.group_norm(np.full((1, 4, 4), 5.0), 2, bias=np.arange(4.0)), np.broadcast_to(np.arange(4.0), (1, 4, 4)))


def test_quantize_oracle_against_fractions():
    rng = np.random.default_rng(2)
    x = np.concatenate([rng.normal(size=(6, 40)), rng.normal(size=(3, 40)) * 1e-6, rng.normal(size=(3, 40)) * 1e4]).astype(np.float16)
    x[2] = 0
    x[3] = np.arange(40) - 20
    x[4, :39], x[4, 39] = np.arange(39), 254
    q, scale = oracle.quantize_rows(x)
    for m in range(len(x)):
        v = [Fraction(float(t)) for t in x[m]]
        top = max(abs(t) for t in v)
        assert scale[m] == float(top / 127)
        for k, t in enumerate(v):
            assert q[m, k] == (round(127 * t / top) if top else 0)                 # of a fraction: to even
    x[1, 3], x[0, 0] = np.nan, -np.inf
    q, scale = oracle.quantize_rows(x)
    assert np.isnan(scale[:2]).all() and not q[:2].any()


def test_quotients_are_never_nearer_to_a_half_than_an_fp32_quotient_is_off():
    """What lets fp32 give the integer of the exact quotient: for every largest value of a binade and every value that is not below half a step, 127 x / top is a half or at least 2^(e - 20)
    from one, 2^e the quotient's own binade."""
    for top in [1024, 1025, 1365, 1536, 1793, 2046, 2047]:
        for shift in range(9):                                                     # x shift binades below
            x = np.arange(1024, 2048, dtype=np.int64)                              # x / 2^shift
            twice = 2 * 127 * x - 0
            den = top << shift                                                     # the quotient is 127 x / den
            odd = 2 * (127 * x // den) + 1                                         # the half above its whole part
            away = np.abs(twice - odd * den)
            quotient = 127 * x / den
            e = np.floor(np.log2(quotient))
            away = away / (2.0 * den)
            keep = (quotient >= 0.25) & (quotient <= 127.0)
            assert ((away[keep] == 0) | (away[keep] >= 2.0 ** (e[keep] - 20))).all()


def test_linear_i8_oracle_against_loops():
    rng = np.random.default_rng(3)
    x, w = rng.integers(-128, 128, size=(3, 9)).astype(np.int8), rng.integers(-128, 128, size=(4, 9)).astype(np.int8)
    xs, ws, b, r = rng.random(3).astype(np.float32), rng.random(4).astype(np.float32), rng.normal(size=4), rng.normal(size=(3, 4))
    got = oracle.linear_i8(x, w, xs, ws, b, r, "relu")
    for m in range(3):
        for n in range(4):
            s = sum(int(x[m, k]) * int(w[n, k]) for k in range(9))
            assert abs(got[m, n] - (max(s * float(xs[m]) * float(ws[n]) + b[n], 0.0) + r[m, n])) < 1e-9
