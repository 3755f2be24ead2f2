"""hb_linear and hb_attention at the sizes whose kernels smaller ones do not reach: the largest tile with several tiles a workgroup and edges
on every side, and workgroups whose waves share the keys in two groups, with ragged, masked and empty rows."""
import numpy as np
import pytest

from paper_2512_02371_amd import hb
from test_gpu_attention import run as attention
from tokentest import F16, TINY

pytestmark = pytest.mark.gpu

ACTS = {"none": lambda t: t, "relu": lambda t: t.clamp(min=0.0), "gelu": lambda t: 0.5 * t * (1.0 + (t * 0.5 ** 0.5).erf()),
        "gelu_tanh": lambda t: 0.5 * t * (1.0 + ((2.0 / np.pi) ** 0.5 * (t + 0.044715 * t ** 3)).tanh()), "silu": lambda t: t * t.sigmoid()}


@pytest.mark.parametrize("M,N,K", [(4090, 4072, 4104), (4090, 8184, 4104), (4096, 4096, 4096), (2049, 8190, 4160)])
def test_linear(M, N, K):
    import torch
    gen = torch.Generator("cuda").manual_seed(M + N)
    normal = lambda *s: torch.randn(s, generator=gen, device="cuda", dtype=torch.float32)
    x, w, bias = normal(M, K).half(), (normal(N, K) * K ** -0.5).half(), normal(N).half()
    product = x.double() @ w.double().t().contiguous()
    size = x.float().abs().double() @ w.float().abs().double().t().contiguous() + bias.double().abs()
    room = hb.hb_linear_workspace_size(M, N, K)
    ws = torch.full((room,), 0xff, dtype=torch.uint8, device="cuda") if room else None
    for i, (act, fn) in enumerate(ACTS.items()):
        for f32 in (False, True):
            kind = torch.float32 if f32 else torch.float16
            residual = normal(M, N).to(kind) if i % 2 == 0 else None
            pitch = N + 8 * (i % 3) + i // 3                           # the last ones at odd elements
            buf = torch.full((M * pitch + 8,), 7.0, dtype=kind, device="cuda")
            out = buf.as_strided((M, N), (pitch, 1))
            print(M, N, K, act, f32, residual is not None, pitch, flush=True)
            hb.hb_linear(x, w, out, ws, bias, residual, act)
            want = fn(product + bias.double())
            bound = (K + 8) * 2.0 ** -23 * size * 1.13 + (0.0 if act in ("none", "relu") else 2.0 ** -20 * size)
            if residual is not None:
                want = want + residual.double()
                bound = bound + 2.0 ** -22 * (size + residual.double().abs())
            bound = bound + (2.0 ** -22 * want.abs() if f32 else F16 * want.abs() + TINY)
            wrong = ~((out.double() - want).abs() <= bound)
            assert not wrong.any(), (act, f32, int(wrong.sum()), wrong.nonzero()[0].tolist())
            out.fill_(7.0)
            assert bool((buf == 7.0).all()), "wrote beside its output"


@pytest.mark.parametrize("B,Lq,Lk,Hq,Hkv,D", [(2, 1000, 600, 10, 10, 64), (1, 1030, 515, 8, 2, 128), (3, 677, 517, 12, 3, 128), (2, 900, 300, 8, 4, 96), (2, 900, 300, 8, 4, 72)])
def test_attention_in_two_groups(B, Lq, Lk, Hq, Hkv, D):
    rng = np.random.default_rng(Lq + D)
    mask = rng.random((B, Lk)) < 0.5
    mask[0, :128] = False                                             # the first tile of either group
    lens = [Lk, 65, 0][:B]                                            # two tiles, or none
    attention("hb_attention", B, Lq, Lk, Hq, Hkv, D, vmean=0.5)
    attention("hb_attention", B, Lq, Lk, Hq, Hkv, D, lens=lens, hidden=(np.nan, np.nan), vmean=0.5)
    attention("hb_attention", B, Lq, Lk, Hq, Hkv, D, lens=[64, 128, 1][:B], mask=mask, hidden=(np.inf, np.nan))
    mask[:] = False
    mask[0, 70] = True                                                # one key, of the second group
    attention("hb_attention", B, Lq, Lk, Hq, Hkv, D, mask=mask, hidden=(np.nan, np.inf))


@pytest.mark.parametrize("B,Lq,Lk,Hq,Hkv,D", [(5, 130, 200, 3, 3, 64), (8, 200, 130, 2, 2, 64), (3, 1, 700, 5, 5, 64), (9, 2, 900, 6, 3, 128), (17, 140, 70, 1, 1, 40)])
def test_ragged_batches_in_every_order_of_heads(B, Lq, Lk, Hq, Hkv, D):
    rng = np.random.default_rng(B)
    lens = [int(n) for n in rng.integers(0, Lk + 1, size=B)]
    attention("hb_attention", B, Lq, Lk, Hq, Hkv, D, lens=lens, hidden=(np.nan, np.nan), vmean=0.5)
