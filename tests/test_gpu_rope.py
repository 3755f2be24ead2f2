"""hb_rope_axes against the fp64 oracle: one to four axes, both pairings, partial rotation, strides, in place, far positions."""
import numpy as np
import pytest

import oracle
from paper_2512_02371_amd import hb
from tokentest import F16, TINY, check, inside, normal, untouched

pytestmark = pytest.mark.gpu


def bound(x, want, sections, interleaved):
    P = sum(sections)
    size = np.zeros(x.shape)
    a = np.abs(x.astype(np.float64))
    u, v = (slice(0, 2 * P, 2), slice(1, 2 * P, 2)) if interleaved else (slice(0, P), slice(P, 2 * P))
    size[..., u] = size[..., v] = a[..., u] + a[..., v]
    return np.where(size > 0, F16 * np.abs(want) + TINY, 0.0) + 1e-5 * size


def frequencies(sections):
    return np.concatenate([10000.0 ** (-np.arange(n) / max(n, 1)) for n in sections]).astype(np.float32)


def run(B, L, H, D, sections, interleaved, pads=(0, 0), leads=(0, 0), low=-100, high=5000, in_place=False, order="blhd", shared=False, seed=1):
    import torch
    x = normal(seed, (B, L, H, D))
    pos = np.random.default_rng(seed).integers(low, high, size=(1 if shared else B, L, len(sections))).astype(np.int32)
    freq = frequencies(sections)
    axes = ["blhd".index(c) for c in order]
    back = [order.index(c) for c in "blhd"]

    def place(a, pad, lead, fill):
        buf, t = inside(torch, a.transpose(axes), pad, lead, fill)
        return buf, t.permute(back)

    _, dx = place(x, pads[0], leads[0], float("nan"))
    buf, out = place(x if in_place else np.full(x.shape, 7.0, np.float16), pads[1], leads[1], 7.0)
    dpos = torch.from_numpy(pos).cuda().expand(B, L, len(sections))
    print("hb_rope_axes", B, L, H, D, sections, interleaved, pads, leads, in_place, order, shared, flush=True)
    hb.hb_rope_axes(out if in_place else dx, out, dpos, torch.from_numpy(freq).cuda(), sections, interleaved)
    torch.cuda.synchronize()
    want = oracle.rope_axes(x, np.broadcast_to(pos, (B, L, len(sections))), freq, sections, interleaved)
    check(out, want, bound(x, want, sections, interleaved), "hb_rope_axes")
    assert untouched(torch, buf, out, 7.0)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("B,L,H,D,sections", [(1, 1, 1, 2, [1]), (1, 1, 1, 64, [32]), (2, 5, 3, 64, [16, 16]), (3, 7, 2, 128, [16, 24, 24]), (1, 9, 4, 80, [20, 20]),
                                              (2, 33, 1, 96, [16, 16, 16]), (1, 17, 5, 40, [7, 6, 7]), (2, 4, 40, 128, [22, 21, 21]), (1, 300, 16, 64, [8, 8]),
                                              (1, 6, 2, 10, [1, 0, 2]), (2, 3, 2, 72, [9, 9, 9, 9]), (1, 5, 3, 7, [3]), (4, 100, 8, 32, [16]), (1, 3, 2, 256, [64, 64])])
def test_shapes(interleaved, B, L, H, D, sections):
    run(B, L, H, D, sections, interleaved)
    run(B, L, H, D, sections, interleaved, in_place=True)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("pads,leads", [((8, 0), (8, 0)), ((0, 8), (0, 8)), ((1, 3), (0, 0)), ((0, 0), (1, 2)), ((5, 0), (0, 3)), ((4, 4), (4, 4)), ((2, 2), (2, 2))])
def test_strides_and_addresses(interleaved, pads, leads):
    for order in ("blhd", "bhld", "lbhd", "hbld"):
        run(2, 11, 3, 64, [16, 16], interleaved, pads, leads, order=order)
        run(2, 11, 3, 48, [8, 8], interleaved, pads, leads, order=order, shared=True)
        run(2, 11, 3, 48, [8, 8], interleaved, pads, leads, order=order, in_place=True)


@pytest.mark.parametrize("low,high", [(0, 1 << 20), ((1 << 24) - 1000, (1 << 24) + 1000), (-(1 << 31), (1 << 31) - 1), ((1 << 31) - 50, (1 << 31) - 1)])
def test_far_positions(low, high):
    for interleaved in (False, True):
        run(2, 200, 2, 64, [16, 16], interleaved, low=low, high=high)


def test_negated_frequencies_turn_back_and_are_the_gradient():
    import torch
    x = torch.from_numpy(normal(3, (2, 30, 4, 64))).cuda()
    g = torch.from_numpy(normal(4, (2, 30, 4, 64))).cuda()
    pos = torch.randint(0, 90, (2, 30, 2), dtype=torch.int32).cuda()
    freq = torch.from_numpy(frequencies([16, 16])).cuda()
    y = hb.hb_rope_axes(x, torch.empty_like(x), pos, freq, [16, 16])
    back = hb.hb_rope_axes(y, torch.empty_like(x), pos, -freq, [16, 16])
    assert (back.float() - x.float()).abs().max() <= 4 * 2.0 ** -11 * 4.5          # two roundings of a pair of up to 4.5
    gx = hb.hb_rope_axes(g, torch.empty_like(x), pos, -freq, [16, 16])
    # <g, R x> = <R^T g, x>, and the difference quotient of a map that is linear is the map itself
    a, b = (g.double() * y.double()).sum(), (gx.double() * x.double()).sum()
    assert abs(a - b) <= 2.0 ** -10 * (g.double().abs() * x.double().abs()).sum() * 2


def test_a_grid_of_tokens_beyond_one_launch_dimension():
    import torch
    B, L, H, D = 1, 70000, 1, 16
    x = normal(5, (B, L, H, D))
    pos = np.stack(np.divmod(np.arange(L), 300), axis=-1)[None].astype(np.int32)
    freq = frequencies([4, 4])
    out = torch.empty((B, L, H, D), dtype=torch.float16, device="cuda:0")
    hb.hb_rope_axes(torch.from_numpy(x).cuda(), out, torch.from_numpy(pos).cuda(), torch.from_numpy(freq).cuda(), (4, 4))
    want = oracle.rope_axes(x, pos, freq, [4, 4], False)
    check(out, want, bound(x, want, [4, 4], False), "many tokens")


def test_refusals():
    import torch
    x = torch.zeros((2, 3, 4, 16), dtype=torch.float16, device="cuda:0")
    pos = torch.zeros((2, 3, 2), dtype=torch.int32, device="cuda:0")
    freq = torch.zeros(8, dtype=torch.float32, device="cuda:0")
    ok = dict(x=x, out=torch.empty_like(x), positions=pos, freq=freq, sections=[4, 4])
    for bad in (dict(out=x[:, :2]), dict(x=x.float()), dict(positions=pos.long()), dict(positions=pos[..., :1]), dict(freq=freq[:7]), dict(freq=freq.double()),
                dict(sections=[4, 3]), dict(sections=[8]), dict(x=x.cpu()), dict(x=x.transpose(2, 3))):
        with pytest.raises(AssertionError):
            hb.hb_rope_axes(**{**ok, **bad})
    for sections, code in (([9, -1], hb.HB_ERR_INVALID_ARG), ([4, 5], hb.HB_ERR_INVALID_ARG), ([0, 0], hb.HB_ERR_INVALID_ARG), ([1, 1, 1, 1, 1], hb.HB_ERR_UNSUPPORTED)):
        with pytest.raises(hb.HbError) as e:
            hb.hb_rope_axes(x, ok["out"], torch.zeros((2, 3, len(sections)), dtype=torch.int32, device="cuda:0"), torch.zeros(sum(sections), device="cuda:0"), sections)
        assert e.value.code == code
