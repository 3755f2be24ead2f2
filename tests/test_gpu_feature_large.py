"""hb_group_norm, hb_quantize_rows and hb_linear_i8 on more than 2^32 elements, at the start, around 2^31 and 2^32, and at the end."""
import pytest

from paper_2512_02371_amd import hb
from tokentest import F16, TINY

pytestmark = pytest.mark.gpu


def filled(torch, shape, seed):
    """fp16 values of a normal distribution, made a part at a time."""
    t = torch.empty(shape, dtype=torch.float16, device="cuda")
    gen = torch.Generator("cuda").manual_seed(seed)
    flat = t.view(-1)
    for i in range(0, flat.numel(), 1 << 28):
        n = min(1 << 28, flat.numel() - i)
        flat[i:i + n] = torch.randn(n, generator=gen, device="cuda", dtype=torch.float16)
    return t


def test_group_norm():
    import torch
    P, C, groups = 70_000_001, 64, 8
    x = filled(torch, (1, P, C), 1)
    out = torch.empty_like(x)
    ws = torch.empty(hb.hb_group_norm_workspace_size(1, P, C, groups), dtype=torch.uint8, device="cuda")
    hb.hb_group_norm(x, out, groups, None, None, 1e-5, "relu", ws)
    total, squares = torch.zeros(groups, dtype=torch.float64, device="cuda"), torch.zeros(groups, dtype=torch.float64, device="cuda")
    for p in range(0, P, 1 << 21):
        v = x[0, p:p + (1 << 21)].double().view(-1, groups, C // groups)
        total += v.sum(dim=(0, 2))
        squares += (v * v).sum(dim=(0, 2))                            # means are next to zero
    mean = total / (P * (C // groups))
    rstd = 1.0 / (squares / (P * (C // groups)) - mean ** 2 + 1e-5).sqrt()
    for p in (0, (1 << 25) - 3000, (1 << 26) - 3000, P - 6000):         # element 2^31 and 2^32 among them
        v = x[0, p:p + 6000].double().view(-1, groups, C // groups)
        want = ((v - mean[:, None]) * rstd[:, None]).clamp(min=0.0).view(-1, C)
        # the statistics of four billion values in chunks of a few thousand: 1e-5 of a deviation
        wrong = ~((out[0, p:p + 6000].double() - want).abs() <= F16 * want + 1e-5 * (1.0 + want) + TINY)
        assert not wrong.any(), (p, wrong.nonzero()[0].tolist())


def test_quantize():
    import torch
    M, K = 270_000, 16384
    x = filled(torch, (M, K), 2)
    q, scale = torch.full((M, K), 99, dtype=torch.int8, device="cuda"), torch.empty(M, device="cuda")
    hb.hb_quantize_rows(x, q, scale)
    for m in range(0, M, 4096):
        v = x[m:m + 4096].float()
        top = v.abs().amax(dim=1)
        assert torch.equal(scale[m:m + 4096], (top.double() / 127.0).float()), m         # divided in fp32 by a number, torch multiplies by its inverse
        assert torch.equal(q[m:m + 4096], torch.round(127.0 * v / top[:, None]).to(torch.int8)), m


def test_linear_i8():
    import torch
    M, N, K = 2_200_000, 48, 2048
    gen = torch.Generator("cuda").manual_seed(3)
    x = torch.randint(-128, 128, (M, K), generator=gen, device="cuda", dtype=torch.int8)
    w = torch.randint(-128, 128, (N, K), generator=gen, device="cuda", dtype=torch.int8)
    xs, ws = torch.rand(M, generator=gen, device="cuda"), torch.rand(N, generator=gen, device="cuda") * 1e-4
    out = torch.empty((M, N), dtype=torch.float32, device="cuda")
    size = hb.hb_linear_i8_workspace_size(M, N, K)
    hb.hb_linear_i8(x, w, xs, ws, out, torch.empty(size, dtype=torch.uint8, device="cuda") if size else None)
    for m in (0, (1 << 20) - 2000, (1 << 21) - 2000, M - 4000):         # element 2^31 and 2^32 among them
        want = torch.mm(x[m:m + 4000].double(), w.double().t().contiguous()) * xs[m:m + 4000].double()[:, None] * ws.double()
        assert ((out[m:m + 4000].double() - want).abs() <= 2.0 ** -22 * want.abs()).all(), m
