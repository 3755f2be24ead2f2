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


@pytest.mark.parametrize("N,C,groups,kind", [((1 << 24) + 5, 1032, 1, "float16"), ((1 << 27) + 11, 66, 2, "float32")], ids=["a token a workgroup", "eight tokens a workgroup"])
def test_tokens_of_more_lanes_than_a_launch_has(N, C, groups, kind):
    """256 lanes a workgroup, 2^32 and more in all: 35 GB, in place, all tokens the same but for some around the end of what one launch takes."""
    import torch
    kind = getattr(torch, kind)
    torch.cuda.empty_cache()
    gen = torch.Generator("cuda").manual_seed(2)
    x = torch.empty((N, 1, C), dtype=kind, device="cuda")
    end = ((1 << 32) - 1) // 256 * (8 if groups == 2 else 1)
    at = [1, N // 2, end - 2, end - 1, end, end + 1, N - 2, N - 1]
    made = torch.randn((9, 1, C), generator=gen, device="cuda").to(kind)
    fill(torch, x, made[0])
    x[at] = made[1:]
    weight = (1.0 + 0.2 * torch.randn(C, generator=gen, device="cuda")).half()
    assert hb.hb_group_norm_workspace_size(N, 1, C, groups) == 0
    print(N, C, groups, kind, flush=True)
    hb.hb_group_norm(x, x, groups, weight)
    torch.cuda.synchronize()
    v = made.double().view(9, groups, C // groups)
    d = v - v.mean(dim=2, keepdim=True)
    rstd = 1.0 / ((d * d).mean(dim=2, keepdim=True) + 1e-5).sqrt()
    scaled = weight.double().view(groups, C // groups)
    want = d * rstd * scaled
    # a value passes 20 additions at most (8 of its lane, 3 or 4 of lanes and 6 between them): the mean is off by 2^-23 of itself and 20 2^-24 of the mean difference, the variance by 28 2^-24,
    # and six roundings make the result
    bound = 40 * 2.0 ** -24 * (1.0 + v.mean(dim=2, keepdim=True).abs() * rstd + (d * rstd).abs()) * scaled.abs() + (F16 * want.abs() + TINY if kind == torch.float16 else 0.0)
    wrong = ~((x[[0] + at].double().view(want.shape) - want).abs() <= bound)
    assert not wrong.any(), wrong.nonzero()[0].tolist()
    first = x[0].clone()
    x[at] = first
    for n in range(0, N, 1 << 20):
        assert bool((x[n:n + (1 << 20)] == first).all()), n
    del x
    torch.cuda.empty_cache()
