"""hb_group_norm against the fp64 oracle: channels and pixels around every vector and tile edge, types, activations, strides, images in place and far
apart, groups that are constant or far from zero, NaN that stays in its group, what lies beside the tensors, and what is refused."""
import numpy as np
import pytest

import oracle
from normtest import norm_bound, pixels
from paper_2512_02371_amd import hb
from tokentest import check, normal, untouched

pytestmark = pytest.mark.gpu


def data(seed, N, P, C, kind):
    rng = np.random.default_rng(seed)
    x = rng.normal(size=(N, P, C)) * (0.5 + rng.random(C)) + rng.normal(size=C)
    return x.astype(kind), (1.0 + 0.2 * rng.normal(size=C)).astype(np.float16), (0.2 * rng.normal(size=C)).astype(np.float16)


def workspace(torch, N, P, C, groups):
    size = hb.hb_group_norm_workspace_size(N, P, C, groups)
    return torch.full((size,), 0xff, dtype=torch.uint8, device="cuda:0") if size else None


def run(N, P, C, groups, act="none", weight=True, bias=True, kinds=(np.float16, np.float16), x_at=(0, 0, 0), out_at=(0, 0, 0), eps=1e-5, seed=1, x=None, in_place=False):
    import torch
    made, w, b = data(seed, N, P, C, kinds[0])
    x = made if x is None else x
    w, b = w if weight else None, b if bias else None
    buf, dx = pixels(torch, x, *x_at, fill=7.0 if in_place else float("nan"))
    obuf, out = (buf, dx) if in_place else pixels(torch, np.full((N, P, C), 7.0, kinds[1]), *out_at, fill=7.0)
    up = lambda t: None if t is None else torch.from_numpy(t).cuda()
    print(N, P, C, groups, act, weight, bias, kinds, x_at, out_at, in_place, flush=True)
    hb.hb_group_norm(dx, out, groups, up(w), up(b), eps, act, workspace(torch, N, P, C, groups))
    torch.cuda.synchronize()
    want = oracle.group_norm(x, groups, w, b, eps, act)
    check(out, want, norm_bound(x, groups, w, b, eps, act, want, kinds[1] is np.float32), f"{N} x {P} x {C} in {groups}")
    assert untouched(torch, obuf, out, 7.0), "wrote beside its output"


@pytest.mark.parametrize("N,P,C,groups", [(1, 1, 1, 1), (1, 1, 8, 1), (1, 2, 1, 1), (2, 1, 64, 32), (3, 1, 1000, 1), (1, 3, 5, 5), (1, 7, 3, 1), (2, 9, 6, 2), (1, 64, 512, 32),
                                          (2, 17, 20, 4), (5, 33, 40, 10), (1, 100, 36, 12), (2, 50, 24, 3), (1, 257, 15, 3), (4, 8, 7, 7), (1, 1000, 64, 32),
                                          (2, 300, 320, 32), (3, 65, 96, 32), (1, 31, 1079, 13), (2, 5, 2048, 8), (1, 4, 4096, 1), (1, 3, 8192, 2), (40, 2, 16, 4), (300, 1, 8, 8),
                                          (7, 12, 130, 13), (1, 1023, 72, 9), (2, 129, 44, 4)])
@pytest.mark.parametrize("kinds", [(np.float16, np.float16), (np.float32, np.float32)], ids=["fp16", "fp32"])
def test_sizes(N, P, C, groups, kinds):
    run(N, P, C, groups, "silu", kinds=kinds)


@pytest.mark.parametrize("N,P,C,groups", [(1, 16384, 64, 32), (2, 4096, 320, 32), (1, 70001, 24, 3), (1, 30000, 9, 3), (1, 100000, 4, 1), (3, 5000, 128, 1), (2, 1500, 1024, 4), (1, 9000, 130, 2),
                                          (1, 5, 12288, 3), (1, 700, 4096, 1), (1, 131072, 16, 8), (9, 2048, 64, 32), (1, 40000, 36, 3), (1, 65536, 8, 1)])
def test_larger_sizes(N, P, C, groups):
    run(N, P, C, groups, "gelu")
    run(N, P, C, groups, "none", False, False, (np.float32, np.float16))


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("kinds", [(a, b) for a in (np.float16, np.float32) for b in (np.float16, np.float32)])
def test_epilogues(act, kinds):
    for weight in (False, True):
        for bias in (False, True):
            run(2, 40, 48, 6, act, weight, bias, kinds)
            run(1, 33, 30, 5, act, weight, bias, kinds)
    run(1, 20000, 48, 6, act, True, True, kinds)
    run(1, 20001, 30, 2, act, True, True, kinds)


# pad, lead, gap of x and of out
@pytest.mark.parametrize("x_at,out_at", [((8, 0, 0), (0, 0, 0)), ((0, 8, 0), (8, 0, 16)), ((1, 0, 0), (3, 1, 5)), ((0, 3, 1), (0, 1, 0)), ((24, 16, 8), (7, 5, 3)), ((2, 2, 2), (2, 2, 2))])
@pytest.mark.parametrize("N,P,C,groups", [(2, 50, 64, 8), (3, 41, 36, 4), (2, 30, 15, 5), (1, 20000, 64, 4), (2, 9001, 35, 1)])
def test_strides_and_addresses(N, P, C, groups, x_at, out_at):
    run(N, P, C, groups, "relu", x_at=x_at, out_at=out_at)
    run(N, P, C, groups, "relu", kinds=(np.float32, np.float16), x_at=x_at, out_at=out_at)


@pytest.mark.parametrize("N,P,C,groups", [(2, 50, 64, 8), (3, 41, 36, 4), (2, 30, 15, 5), (1, 30000, 64, 4), (2, 9001, 35, 1)])
@pytest.mark.parametrize("kind", [np.float16, np.float32])
def test_in_place(N, P, C, groups, kind):
    run(N, P, C, groups, "silu", kinds=(kind, kind), in_place=True)
    run(N, P, C, groups, "silu", kinds=(kind, kind), x_at=(5, 3, 1), in_place=True)


@pytest.mark.parametrize("P", [60, 30000])
def test_pixels_before_images(P):
    """P x N x C in memory: the image stride is the smaller one."""
    import torch
    N, C, groups = 3, 40, 4
    x, w, b = data(3, N, P, C, np.float16)
    dx = torch.from_numpy(np.ascontiguousarray(x.transpose(1, 0, 2))).cuda().transpose(0, 1)
    out = torch.empty((P, N, C), dtype=torch.float16, device="cuda:0").transpose(0, 1)
    hb.hb_group_norm(dx, out, groups, torch.from_numpy(w).cuda(), torch.from_numpy(b).cuda(), 1e-5, "none", workspace(torch, N, P, C, groups))
    want = oracle.group_norm(x, groups, w, b)
    check(out, want, norm_bound(x, groups, w, b, 1e-5, "none", want, False), "pixels before images")


def test_maps_with_rows():
    import torch
    x, w, b = data(4, 2, 6 * 7, 64, np.float16)
    dx = torch.from_numpy(x).cuda().view(2, 6, 7, 64)
    out = hb.hb_group_norm(dx, torch.empty_like(dx), 8, torch.from_numpy(w).cuda(), torch.from_numpy(b).cuda())
    flat = hb.hb_group_norm(dx.view(2, 42, 64), torch.empty_like(dx).view(2, 42, 64), 8, torch.from_numpy(w).cuda(), torch.from_numpy(b).cuda())
    assert torch.equal(out.view(2, 42, 64), flat)
    column = dx[:, :, 2:3]                                            # one pixel of each row: pixels 7 apart
    got = hb.hb_group_norm(column, torch.empty((2, 6, 1, 64), dtype=torch.float16, device="cuda:0"), 8)
    want = oracle.group_norm(x.reshape(2, 6, 7, 64)[:, :, 2], 8)
    check(got[:, :, 0], want, norm_bound(x.reshape(2, 6, 7, 64)[:, :, 2], 8, None, None, 1e-5, "none", want, False), "a column")
    row = hb.hb_group_norm(dx[:, 1:2, 1:5], torch.empty((2, 1, 4, 64), dtype=torch.float16, device="cuda:0"), 8)
    assert torch.isfinite(row).all()
    with pytest.raises(AssertionError):
        hb.hb_group_norm(dx[:, :, 1:5], torch.empty((2, 6, 4, 64), dtype=torch.float16, device="cuda:0"), 8)      # a window: pixels at two distances


@pytest.mark.parametrize("N,P,C,groups", [(2, 64, 64, 8), (1, 37, 30, 6), (1, 20000, 64, 8), (1, 20011, 30, 2)])
@pytest.mark.parametrize("kind", [np.float16, np.float32])
def test_means_far_from_zero_and_constants(N, P, C, groups, kind):
    rng = np.random.default_rng(5)
    x = rng.normal(size=(N, P, C)) + 1000.0
    run(N, P, C, groups, kinds=(kind, np.float32), x=x.astype(kind))
    x[:, :1] = 0.0                                                    # a first pixel that is a thousand deviations away
    run(N, P, C, groups, kinds=(kind, np.float32), x=x.astype(kind))
    x = np.broadcast_to(rng.normal(size=(N, 1, groups, 1)) * 300.0, (N, P, groups, C // groups)).reshape(N, P, C).astype(kind)
    run(N, P, C, groups, kinds=(kind, np.float32), x=x)
    run(N, P, C, groups, kinds=(kind, np.float32), x=np.zeros((N, P, C), kind))
    run(N, P, C, groups, kinds=(kind, np.float32), x=(rng.normal(size=(N, P, C)) * 1e-7).astype(kind), eps=1e-12)


@pytest.mark.parametrize("P", [50, 30000])
@pytest.mark.parametrize("C,groups", [(64, 8), (30, 6)])
def test_nan_and_infinity_stay_in_their_group(P, C, groups):
    import torch
    N, D = 3, C // groups
    x, w, b = data(6, N, P, C, np.float16)
    clean = oracle.group_norm(x, groups, w, b, act="relu")
    x[0, P // 2, D], x[2, P - 1, C - 1], x[1, 0, 0] = np.nan, np.inf, -np.inf
    out = torch.empty((N, P, C), dtype=torch.float16, device="cuda:0")
    hb.hb_group_norm(torch.from_numpy(x).cuda(), out, groups, torch.from_numpy(w).cuda(), torch.from_numpy(b).cuda(), 1e-5, "relu", workspace(torch, N, P, C, groups))
    got = out.float().cpu().numpy().reshape(N, P, groups, D)
    hit = np.zeros((N, groups), bool)
    hit[0, 1] = hit[2, groups - 1] = hit[1, 0] = True
    clean = clean.reshape(N, P, groups, D)
    for n in range(N):
        for g in range(groups):
            if hit[n, g]:
                assert np.isnan(got[n, :, g]).all()
            else:
                assert np.abs(got[n, :, g] - clean[n, :, g]).max() < 1e-2


def test_offsets_beyond_32_bits():
    import torch
    N, P, C, pixel = 2, 1100, 40, 1 << 21
    pool = torch.zeros(N * P * pixel, dtype=torch.float16, device="cuda:0")       # 9.2 GB: pixels 4 MB apart
    x, w, b = data(7, N, P, C, np.float16)
    dx = pool.as_strided((N, P, C), (P * pixel, pixel, 1))
    dx.copy_(torch.from_numpy(x))
    out = pool.as_strided((N, P, C), (P * pixel, pixel, 1), 1 << 20)
    hb.hb_group_norm(dx, out, 4, torch.from_numpy(w).cuda(), torch.from_numpy(b).cuda(), 1e-5, "none", workspace(torch, N, P, C, 4))
    want = oracle.group_norm(x, 4, w, b)
    check(out, want, norm_bound(x, 4, w, b, 1e-5, "none", want, False), "pixels far apart")


def test_repeats_bit_for_bit_on_any_stream():
    import torch
    for N, P, C, groups in ((2, 64, 64, 8), (1, 50000, 64, 32), (3, 9001, 35, 5)):
        x = torch.from_numpy(data(8, N, P, C, np.float16)[0]).cuda()
        outs = []
        for _ in range(3):
            s = torch.cuda.Stream()
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                outs.append(hb.hb_group_norm(x, torch.empty((N, P, C), dtype=torch.float32, device="cuda:0"), groups, act="silu", workspace=workspace(torch, N, P, C, groups)))
            s.synchronize()
        assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


def test_images_alone_and_together_are_the_same():
    import torch
    for P, C, groups in ((64, 64, 8), (40000, 64, 32), (1001, 35, 5), (1, 96, 3)):
        x = torch.from_numpy(data(9, 4, P, C, np.float16)[0]).cuda()
        ws = workspace(torch, 4, P, C, groups)
        all_of = hb.hb_group_norm(x, torch.empty_like(x), groups, workspace=ws)
        for n in range(4):
            one = hb.hb_group_norm(x[n:n + 1], torch.empty_like(x[:1]), groups, workspace=workspace(torch, 1, P, C, groups))
            a, b = one[0].float(), all_of[n].float()                   # sums in another order: a rounding may go the other way
            assert (a - b).abs().max() <= 2.0 ** -10 * a.abs().max()


def test_refusals():
    import torch
    f16 = lambda *s: torch.zeros(s, dtype=torch.float16, device="cuda:0")
    ok = dict(x=f16(2, 4, 8), out=f16(2, 4, 8), groups=2)
    for bad in (dict(x=f16(2, 4, 7)), dict(out=f16(2, 3, 8)), dict(x=f16(2, 4, 8).double()), dict(x=f16(2, 4, 8).cpu()), dict(weight=f16(7)), dict(bias=f16(8).float()),
                dict(weight=f16(8).cpu()), dict(x=f16(2, 8, 4).transpose(1, 2)), dict(x=f16(4, 8), out=f16(4, 8)), dict(workspace=f16(8)), dict(out=f16(2, 4, 8).to(torch.bfloat16))):
        with pytest.raises(AssertionError):
            hb.hb_group_norm(**{**ok, **bad})
    with pytest.raises(KeyError):
        hb.hb_group_norm(**ok, act="swish")
    for bad in (dict(groups=3), dict(groups=0), dict(groups=16), dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")),
                dict(out=f16(64).as_strided((2, 4, 8), (16, 4, 1))), dict(x=f16(8).expand(2, 4, 8))):
        with pytest.raises(hb.HbError) as e:
            hb.hb_group_norm(**{**ok, **bad})
        assert e.value.code == hb.HB_ERR_INVALID_ARG, bad
    N, P, C, groups = 1, 1 << 16, 64, 1
    if hb.hb_group_norm_workspace_size(N, P, C, groups):
        for ws in (None, torch.empty(16, dtype=torch.uint8, device="cuda:0")):
            with pytest.raises(hb.HbError) as e:
                hb.hb_group_norm(f16(N, P, C), f16(N, P, C), groups, workspace=ws)
            assert e.value.code == hb.HB_ERR_WORKSPACE
