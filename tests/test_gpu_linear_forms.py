"""hb_linear in every form that its choice by size takes, against fp64: rows between NaN, results between canaries, residuals in place and beside."""
import pytest

from lineartest import FORMS
from paper_2512_02371_amd import hb
from tokentest import F16, TINY

pytestmark = pytest.mark.gpu

ACTS = {"none": lambda t: t, "relu": lambda t: t.clamp(min=0.0), "gelu": lambda t: 0.5 * t * (-t * 0.5 ** 0.5).erfc(), "silu": lambda t: t * t.sigmoid()}


def window(torch, t, pad, lead, fill):
    """t as a view of a larger buffer of `fill`: `pad` elements behind every row, `lead` in front of the first."""
    rows, width = t.shape
    buf = torch.full((lead + rows * (width + pad) + 64,), fill, dtype=t.dtype, device="cuda")
    view = buf.as_strided((rows, width), (width + pad, 1), lead)
    view.copy_(t)
    return buf, view


@pytest.mark.parametrize("M,N,K,rows", FORMS)
def test_form(M, N, K, rows):
    import torch
    gen = torch.Generator("cuda").manual_seed(M + N + K)
    normal = lambda *s: torch.randn(s, generator=gen, device="cuda", dtype=torch.float32)
    x, w, bias = normal(M, K).half(), (normal(N, K) * K ** -0.5).half(), normal(N).half()
    lead, xpad, wpad = {"copied": (8, 8, 16), "even": (2, 2 + K % 2, 4 + K % 2), "odd": (1, 1 + K % 2, 2 - K % 2)}[rows]
    xv, wv = window(torch, x, xpad, lead, float("nan"))[1], window(torch, w, wpad, lead, float("nan"))[1]
    product = torch.mm(x.double(), w.double().t().contiguous())
    size = torch.mm(x.abs().double(), w.abs().double().t().contiguous()) + bias.double().abs()
    room = hb.hb_linear_workspace_size(M, N, K)
    ws = torch.full((room,), 0xff, dtype=torch.uint8, device="cuda") if room else None
    for act, f32, residual in (("gelu", False, None), ("silu", True, "in place"), ("relu", False, "in place"), ("none", True, "beside"), ("none", False, "beside")):
        kind = torch.float32 if f32 else torch.float16
        r = normal(M, N).to(kind) if residual else torch.full((M, N), 7.0, dtype=kind, device="cuda")
        pad, first = {"gelu": (0, 0), "silu": (3, 1), "relu": (8, 8), "none": (5, 3)}[act]
        buf, out = window(torch, r, pad, first, 7.0)
        beside = window(torch, r, 7, 1, float("nan"))[1] if residual == "beside" else None
        print(M, N, K, rows, act, f32, residual, "workspace", room, flush=True)
        hb.hb_linear(xv, wv, out, ws, bias, out if residual == "in place" else beside, act)
        want = ACTS[act](product + bias.double())
        bound = (K + 8) * 2.0 ** -23 * size * 1.13 + (0.0 if act in ("none", "relu") else 2.0 ** -20 * size)
        if residual:
            want = want + r.double()
            bound = bound + 2.0 ** -22 * (size + r.double().abs())
        bound = bound + (2.0 ** -22 * want.abs() if f32 else F16 * want.abs() + TINY)
        wrong = ~((out.double() - want).abs() <= bound)
        assert not wrong.any(), (act, f32, residual, int(wrong.sum()), wrong.nonzero()[0].tolist())
        out.fill_(7.0)
        assert bool((buf == 7.0).all()), "wrote beside its output"
