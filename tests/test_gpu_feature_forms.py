"""hb_group_norm and hb_linear_i8 in every form that their choices by size take, against fp64: inputs between other values, results between canaries, in place and beside."""
import pytest

from featureforms import I8_FORMS, NORM_FORMS
from paper_2512_02371_amd import hb
from tokentest import F16, TINY

pytestmark = pytest.mark.gpu

ACTS = {"none": lambda t: t, "relu": lambda t: t.clamp(min=0.0), "gelu": lambda t: 0.5 * t * (-t * 0.5 ** 0.5).erfc(), "silu": lambda t: t * t.sigmoid()}


@pytest.mark.parametrize("N,P,C,groups,f32,dense", NORM_FORMS)
def test_group_norm(N, P, C, groups, f32, dense):
    import torch
    gen = torch.Generator("cuda").manual_seed(N + P + C)
    normal = lambda *s: torch.randn(s, generator=gen, device="cuda")
    kind = torch.float32 if f32 else torch.float16
    act = sorted(ACTS)[(N + P + C + groups) % 4]
    out_kind = (torch.float16, torch.float32)[(P + C) % 2]
    pad, lead, gap = (0, 8, 0) if dense else (3, 1, 5)

    def window(t, pad, lead, gap, fill):
        strides = (P * (C + pad) + gap, C + pad, 1)
        buf = torch.full((lead + N * strides[0] + 64,), fill, dtype=t.dtype, device="cuda")
        view = buf.as_strided((N, P, C), strides, lead)
        view.copy_(t)
        return buf, view

    x = (normal(N, P, C) * (0.5 + torch.rand(C, generator=gen, device="cuda")) + normal(C)).to(kind)
    w, b = (1.0 + 0.2 * normal(C)).half(), (0.2 * normal(C)).half()
    xv = window(x, pad, lead, gap, float("nan"))[1]
    buf, out = window(torch.full((N, P, C), 7.0, dtype=out_kind, device="cuda"), pad, lead, gap, 7.0)
    size = hb.hb_group_norm_workspace_size(N, P, C, groups)
    ws = torch.full((size,), 0xff, dtype=torch.uint8, device="cuda") if size else None
    print(N, P, C, groups, f32, dense, act, out_kind, flush=True)
    hb.hb_group_norm(xv, out, groups, w, b, 1e-5, act, ws)
    # the definition, and the bounds of normtest.norm_bound
    v = x.double().reshape(N, P, groups, C // groups)
    mean = v.mean(dim=(1, 3), keepdim=True)
    d = v - mean
    var = (d * d).mean(dim=(1, 3), keepdim=True)
    rstd = 1.0 / (var + 1e-5).sqrt()
    H = 300 + P * (C // groups) / 256
    dm = 2.0 ** -23 * mean.abs() + H * 2.0 ** -24 * d.abs().mean(dim=(1, 3), keepdim=True)
    off = ((H + 8) * 2.0 ** -24 * var + dm ** 2) * rstd ** 2
    flat = lambda t: t.expand(v.shape).reshape(N, P, C)
    want = ACTS[act](flat(d * rstd) * w.double() + b.double())
    part = flat((d * rstd).abs()) * w.double().abs()
    e = flat(dm * rstd) * w.double().abs() + part * (flat(off) + 6 * 2.0 ** -24) + 2.0 ** -23 * (part + b.double().abs())
    e = 1.13 * e + (0.0 if act in ("none", "relu") else 2.0 ** -20 * (part + b.double().abs()))
    e = e + (2.0 ** -23 * want.abs() if out_kind == torch.float32 else F16 * want.abs() + TINY)
    wrong = ~((out.double() - want).abs() <= e)
    assert not wrong.any(), (int(wrong.sum()), wrong.nonzero()[0].tolist())
    if kind == out_kind:                                              # in place, the same bits
        other = window(x, pad, lead, gap, float("nan"))[1]
        hb.hb_group_norm(other, other, groups, w, b, 1e-5, act, ws)
        assert torch.equal(other, out)
    out.fill_(7.0)
    assert bool((buf == 7.0).all()), "wrote beside its output"


@pytest.mark.parametrize("M,N,K,rows", I8_FORMS)
def test_linear_i8(M, N, K, rows):
    import torch
    gen = torch.Generator("cuda").manual_seed(M + N + K)
    integers = lambda *s: torch.randint(-128, 128, s, generator=gen, device="cuda", dtype=torch.int8)
    x, w, xs = integers(M, K), integers(N, K), torch.rand(M, generator=gen, device="cuda") * 0.02 + 0.005
    ws, bias = (torch.rand(N, generator=gen, device="cuda") * 0.02 + 0.005) * K ** -0.5, torch.randn(N, generator=gen, device="cuda").half()

    def window(t, pad, lead, fill):
        rows, width = t.shape
        buf = torch.full((lead + rows * (width + pad) + 64,), fill, dtype=t.dtype, device="cuda")
        view = buf.as_strided((rows, width), (width + pad, 1), lead)
        view.copy_(t)
        return buf, view

    lead, xpad, wpad = {"copied": (16, 16, 32), "even": (4, 4 + -K % 4, 8 + -K % 4), "odd": (1, 1 + K % 2, 2 - K % 2)}[rows]
    xv, wv = window(x, xpad, lead, 101)[1], window(w, wpad, lead, -99)[1]
    size = torch.mm(x.double(), w.double().t().contiguous()) * xs.double()[:, None] * ws.double()
    room = hb.hb_linear_i8_workspace_size(M, N, K)
    scratch = torch.full((room,), 0xff, dtype=torch.uint8, device="cuda") if room else None
    for act, f32, residual in (("gelu", False, None), ("silu", True, "in place"), ("relu", False, "in place"), ("none", True, "beside"), ("none", False, "beside")):
        kind = torch.float32 if f32 else torch.float16
        r = torch.randn((M, N), generator=gen, device="cuda").to(kind) if residual else torch.full((M, N), 7.0, dtype=kind, device="cuda")
        pad, first = {"gelu": (0, 0), "silu": (3, 1), "relu": (8, 8), "none": (5, 3)}[act]
        buf, out = window(r, pad, first, 7.0)
        beside = window(r, 7, 1, float("nan"))[1] if residual == "beside" else None
        print(M, N, K, rows, act, f32, residual, "workspace", room, flush=True)
        hb.hb_linear_i8(xv, wv, xs, ws, out, scratch, bias, out if residual == "in place" else beside, act)
        want, part = ACTS[act](size + bias.double()), size.abs() + bias.double().abs()
        bound = 4 * 2.0 ** -24 * part * 1.13 + (0.0 if act in ("none", "relu") else 2.0 ** -20 * part)
        if residual:
            want = want + r.double()
            bound = bound + 2.0 ** -23 * (part + r.double().abs())
        bound = bound + (2.0 ** -23 * want.abs() if f32 else F16 * want.abs() + TINY)
        wrong = ~((out.double() - want).abs() <= bound)
        assert not wrong.any(), (act, f32, residual, int(wrong.sum()), wrong.nonzero()[0].tolist())
        out.fill_(7.0)
        assert bool((buf == 7.0).all()), "wrote beside its output"
