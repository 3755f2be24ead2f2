"""hb_group_norm with groups in the registers of a workgroup, every kernel and every number of vectors that matters: values that are alike everywhere, and first vectors whose mean is far from
that of the others, which the one-pass variance has to make up for."""
import pytest

from normslabs import NORM_SLABS, slab_bound
from paper_2512_02371_amd import hb

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("N,P,C,groups,f32,dense,first", NORM_SLABS)
def test_alike_and_first_vectors_far_from_the_others(N, P, C, groups, f32, dense, first):
    import torch
    gen = torch.Generator("cuda").manual_seed(N + P + C)
    normal = lambda *s: torch.randn(s, generator=gen, device="cuda")
    kind = torch.float32 if f32 else torch.float16
    pad, gap = (0, 0) if dense else (3, 5)

    def window(fill, kind):
        strides = (P * (C + pad) + gap, C + pad, 1)
        buf = torch.full((N * strides[0] + 64,), fill, dtype=kind, device="cuda")
        return buf, buf.as_strided((N, P, C), strides)

    weight, bias = (1.0 + 0.2 * normal(C)).half(), (0.2 * normal(C)).half()
    size = hb.hb_group_norm_workspace_size(N, P, C, groups)
    ws = torch.full((size,), 0xff, dtype=torch.uint8, device="cuda") if size else None
    for far, act in ((0.0, "silu"), (50.0, "none")):
        x = normal(N, P, C) * (0.5 + torch.rand(C, generator=gen, device="cuda")) + normal(C)
        x[:, :first] += far
        x = x.to(kind)
        xv = window(float("nan"), kind)[1]
        xv.copy_(x)
        v = x.double()
        parts = v.reshape(N, P, groups, C // groups)
        d = parts - parts.mean(dim=(1, 3), keepdim=True)
        y = (d / ((d * d).mean(dim=(1, 3), keepdim=True) + 1e-5).sqrt()).reshape(N, P, C) * weight.double() + bias.double()
        want = y * y.sigmoid() if act == "silu" else y
        for out_kind in (torch.float16, torch.float32):
            buf, out = window(7.0, out_kind)
            print(N, P, C, groups, f32, dense, far, out_kind, flush=True)
            hb.hb_group_norm(xv, out, groups, weight, bias, 1e-5, act, ws)
            wrong = ~((out.double() - want).abs() <= slab_bound(v, groups, first, weight.double(), bias.double(), act, want, out_kind == torch.float32))
            assert not wrong.any(), (far, out_kind, int(wrong.sum()), wrong.nonzero()[0].tolist())
            out.fill_(7.0)
            assert bool((buf == 7.0).all()), "wrote beside its output"
