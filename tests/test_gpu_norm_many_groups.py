"""hb_group_norm of so many groups or tokens that a launch has not a wave, or a workgroup's lanes, for each."""
import pytest

from paper_2512_02371_amd import hb
from tokentest import F16, TINY

pytestmark = pytest.mark.gpu


def fill(torch, x, value):
    """`value` for every image, a part of them at a time."""
    for n in range(0, x.shape[0], 1 << 16):
        x[n:n + (1 << 16)] = value


def test_a_channel_a_group_in_many_images_that_stream():
    """16401 images of 29 pixels of 4092 channels, 2^26 groups and more whose rows are read twice: in place, all images the same but for some."""
    import torch
    N, P, C = 16401, 29, 4092
    assert N * C >= 1 << 26 and hb.hb_group_norm_workspace_size(N, P, C, C) > 0
    gen = torch.Generator("cuda").manual_seed(1)
    made = torch.randn((5, P, C), generator=gen, device="cuda").half()
    x = torch.empty((N, P, C), dtype=torch.float16, device="cuda")
    fill(torch, x, made[0])
    at = [1, 8000, N - 2, N - 1]
    x[at] = made[1:]
    ws = torch.empty(hb.hb_group_norm_workspace_size(N, P, C, C), dtype=torch.uint8, device="cuda")
    print(N, P, C, flush=True)
    hb.hb_group_norm(x, x, C, act="relu", workspace=ws)
    torch.cuda.synchronize()
    v = made.double()
    d = v - v.mean(dim=1, keepdim=True)
    rstd = 1.0 / ((d * d).mean(dim=1, keepdim=True) + 1e-5).sqrt()
    want = (d * rstd).clamp(min=0.0)
    # 29 values to a group: means and variances are off by 40 roundings at most
    wrong = ~((x[[0] + at].double() - want).abs() <= F16 * want + 40 * 2.0 ** -24 * (1.0 + v.mean(dim=1, keepdim=True).abs() * rstd + (d * rstd).abs()) + TINY)
    assert not wrong.any(), wrong.nonzero()[0].tolist()
    first = x[0].clone()
    x[at] = first
    for n in range(0, N, 1 << 11):
        assert bool((x[n:n + (1 << 11)] == first).all()), n
