"""The activations of hb_linear and its twin, value by value: fp32 output, relative bounds out to where results are 1e-15 of their argument.

The bounds were derived before the test first ran.  An exponent whose constant and products are rounded n times is off by n 2^-24 of itself, and
the exponential by that times the exponent: 3 roundings of v^2 / 2 for gelu, 5 of 2 z for gelu_tanh, 2 of v for silu (powers of two above them below).
What is left, the polynomial of gelu's tail (1e-7) with its eight steps, reciprocal, exponential and products of an ulp each, is below 2^-20.
Results below the smallest normal number may be zero."""
import numpy as np
import pytest
from scipy.special import erfc

from paper_2512_02371_amd import hb

pytestmark = pytest.mark.gpu
BOTH = pytest.mark.parametrize("fn", ["hb_linear", "hb_linear_valu"])


def exact(v, act):
    """The activation, and what its exponent amounts to."""
    if act == "gelu":
        return 0.5 * v * erfc(-v / np.sqrt(2.0)), v * v / 2.0
    z = 2.0 * np.sqrt(2.0 / np.pi) * (v + 0.044715 * v ** 3) if act == "gelu_tanh" else v
    return v / (1.0 + np.exp(-z)), np.abs(z)


def check(got, v, act):
    want, exponent = exact(v, act)
    roundings = {"gelu": 4, "gelu_tanh": 8, "silu": 4}[act]
    bound = (2.0 ** -20 + roundings * 2.0 ** -24 * exponent) * np.abs(want) + 2.0 ** -126
    err = np.abs(got.double().cpu().numpy() - want)
    bad = ~(err <= bound)
    assert not bad.any(), (act, int(bad.sum()), "first at", v[bad][0], "relative error", (err / np.abs(want))[bad][0])


@BOTH
@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("form", ["rows", "one row", "split"])
def test_every_value(fn, act, form):
    import torch
    n = 4001
    v = torch.linspace(-8.0, 8.0, n, dtype=torch.float64).half()
    one = torch.ones((1, 1), dtype=torch.float16)
    x, w = (v[:, None], one) if form == "rows" else (one, v[:, None])
    if form == "split":                                   # a sum over 8192 of which one term is not 0
        x, w = torch.zeros((1, 8192), dtype=torch.float16), torch.zeros((64, 8192), dtype=torch.float16)
        x[0, 5000], v = 1.0, v[:: n // 63][:64]
        w[:len(v), 5000] = v
    x, w = x.cuda(), w.cuda()
    size = hb.hb_linear_workspace_size(x.shape[0], w.shape[0], x.shape[1])
    assert (size > 0) == (form == "split")
    ws = torch.empty(size, dtype=torch.uint8, device="cuda:0") if size else None
    out = torch.empty((x.shape[0], w.shape[0]), dtype=torch.float32, device="cuda:0")
    print(fn, act, form, flush=True)
    getattr(hb, fn)(x, w, out, ws, act=act)
    check(out.reshape(-1)[:len(v)], v.double().numpy(), act)
