"""hb_attention and its twin against the fp64 oracle: lengths from none to long, grouped heads, every head size, ragged and masked keys,
rows that see nothing, what stands behind a mask, strides and orders, and what is refused."""
import numpy as np
import pytest

import oracle
from paper_2512_02371_amd import hb
from tokentest import attention_bound, check, inside, normal, untouched

pytestmark = pytest.mark.gpu
BOTH = pytest.mark.parametrize("fn", ["hb_attention", "hb_attention_valu"])


def call(fn, q, k, v, out, scale, key_len=None, key_mask=None):
    import torch
    B, Lq, Hq, D = q.shape
    size = hb.hb_attention_workspace_size(B, Lq, k.shape[1], Hq, k.shape[2], D)
    ws = torch.full((size,), 0xff, dtype=torch.uint8, device="cuda:0") if size else None
    print(fn, tuple(q.shape), tuple(k.shape), q.stride(), k.stride(), flush=True)
    return getattr(hb, fn)(q, k, v, out, scale, ws, key_len, key_mask)


def run(fn, B, Lq, Lk, Hq, Hkv, D, lens=None, mask=None, scale=None, qstd=1.0, vmean=0.0, pads=(0, 0, 0), order="blhd", hidden=None, seed=1):
    import torch
    scale = D ** -0.5 if scale is None else scale
    q, k, v = normal(seed, (B, Lq, Hq, D), qstd), normal(seed + 1, (B, Lk, Hkv, D)), normal(seed + 2, (B, Lk, Hkv, D)) + np.float16(vmean)
    if hidden is not None:                                            # what keys that are not visible hold
        for b in range(B):
            for j in range(Lk):
                if (lens is not None and j >= lens[b]) or (mask is not None and not mask[b, j]):
                    k[b, j], v[b, j] = hidden
    axes = ["blhd".index(c) for c in order]
    back = [order.index(c) for c in "blhd"]

    def place(a, pad, fill):
        buf, t = inside(torch, a.transpose(axes), pad, 8, fill)
        return buf, t.permute(back)

    dq, dk, dv = (place(a, p, float("nan"))[1] for a, p in ((q, pads[0]), (k, pads[1]), (v, pads[1])))
    buf, out = place(np.full(q.shape, 7.0, np.float16), pads[2], 7.0)
    dl = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda:0")
    dm = None
    if mask is not None:
        dm = torch.ones((B, Lk + 5), dtype=torch.uint8, device="cuda:0")[:, :Lk]
        dm.copy_(torch.from_numpy(mask))
    call(fn, dq, dk, dv, out, scale, dl, dm)
    torch.cuda.synchronize()
    want = oracle.attention(q, k, v, scale, lens, mask)
    check(out, want, attention_bound(q, k, v, scale, lens, mask, want), f"{fn} {B} {Lq} {Lk} {Hq} {Hkv} {D}")
    assert untouched(torch, buf, out, 7.0)


@BOTH
@pytest.mark.parametrize("D", [8, 16, 24, 32, 40, 56, 64, 72, 80, 96, 104, 112, 128])
def test_head_sizes(fn, D):
    run(fn, 2, 70, 90, 4, 2, D)
    run(fn, 2, 1, 90, 4, 2, D)


@BOTH
@pytest.mark.parametrize("Lq", [1, 2, 15, 17, 32, 33, 64, 100, 129, 257])
@pytest.mark.parametrize("Lk", [1, 2, 31, 32, 33, 63, 64, 65, 77, 128, 200])
def test_lengths(fn, Lq, Lk):
    run(fn, 1, Lq, Lk, 2, 1, 64, vmean=1.0)


@pytest.mark.parametrize("B,Lq,Lk,Hq,Hkv,D", [(1, 1, 5000, 1, 1, 64), (2, 1, 4097, 8, 1, 128), (3, 2, 3001, 8, 2, 80), (1, 5, 8200, 4, 4, 40), (2, 600, 700, 3, 3, 64),
                                              (1, 1030, 515, 8, 2, 128), (2, 300, 1100, 6, 1, 96), (1, 33, 2500, 32, 4, 64), (20, 1, 300, 16, 2, 128), (1, 513, 65, 16, 16, 32)])
def test_longer(B, Lq, Lk, Hq, Hkv, D):
    run("hb_attention", B, Lq, Lk, Hq, Hkv, D)
    lens = [int(n) for n in np.random.default_rng(B + Lk).integers(0, Lk + 1, size=B)]
    run("hb_attention", B, Lq, Lk, Hq, Hkv, D, lens=lens, vmean=0.5)


@BOTH
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (3, 3), (4, 1), (6, 2), (8, 8), (5, 1), (64, 4), (16, 1)])
def test_grouped_heads(fn, Hq, Hkv):
    for Lq in (1, 3, 40):
        run(fn, 2, Lq, 70, Hq, Hkv, 64)


@BOTH
@pytest.mark.parametrize("Lq", [1, 7, 150])
def test_masks(fn, Lq):
    rng = np.random.default_rng(7)
    Lk = 300
    lens = [0, 1, 64, 65, 299, 300, -5, 1000]
    B = len(lens)
    mask = rng.random((B, Lk)) < 0.5
    for D in (64, 128):
        run(fn, B, Lq, Lk, 2, 1, D, lens=lens)
        run(fn, B, Lq, Lk, 2, 1, D, mask=mask)
        run(fn, B, Lq, Lk, 2, 1, D, lens=lens, mask=mask)
    mask[:] = False
    mask[1, 0] = mask[2, 299] = mask[3, 150] = True                   # one key, or none
    mask[4, 128:192] = True                                           # whole blocks hidden in front and behind
    mask[5, 100:] = True
    run(fn, B, Lq, Lk, 2, 1, 64, mask=mask)
    run(fn, B, Lq, Lk, 2, 1, 64, mask=mask, lens=[300, 1, 299, 150, 130, 100, 0, 300])


@BOTH
@pytest.mark.parametrize("hidden", [(np.nan, np.nan), (np.inf, np.inf), (-np.inf, np.nan), (65504.0, -65504.0)])
def test_what_is_hidden_has_no_influence(fn, hidden):
    rng = np.random.default_rng(8)
    for Lq in (1, 80):
        run(fn, 3, Lq, 140, 2, 1, 64, lens=[0, 77, 139], hidden=hidden)
        run(fn, 3, Lq, 140, 2, 1, 72, mask=rng.random((3, 140)) < 0.4, hidden=hidden)


@BOTH
def test_no_keys_at_all(fn):
    import torch
    for Lq in (1, 50):
        q = torch.randn((2, Lq, 4, 64), device="cuda:0").half()
        k = torch.empty((2, 0, 2, 64), dtype=torch.float16, device="cuda:0")
        out = torch.full_like(q, 7.0)
        call(fn, q, k, k, out, 1.0)
        assert not out.any()


@BOTH
def test_large_scores_and_single_winners(fn):
    # scores up to some hundreds: one key takes all, the maximum moves from block to block
    for Lq in (1, 64):
        run(fn, 2, Lq, 333, 2, 2, 64, scale=1.0, qstd=8.0)
        run(fn, 1, Lq, 200, 1, 1, 128, scale=-0.5)
        run(fn, 1, Lq, 200, 1, 1, 64, scale=0.0, vmean=1.0)


@BOTH
def test_extreme_scores(fn):
    """Scores beyond what exp() holds in fp32, in growing and in falling order, and infinite ones."""
    import torch
    for Lq in (1, 40):
        q = torch.full((1, Lq, 1, 64), 100.0, dtype=torch.float16, device="cuda:0")
        k = torch.linspace(-100, 100, 500, device="cuda:0").half()[None, :, None, None].expand(1, 500, 1, 64).contiguous()
        v = torch.randn((1, 500, 1, 64), device="cuda:0").half()
        for kk, best in ((k, 499), (k.flip(1).contiguous(), 0)):
            out = call(fn, q, kk, v, torch.empty_like(q), 1.0)
            assert torch.equal(out, v[:, best:best + 1].expand_as(out))
        low = torch.full_like(k, -65504.0)                            # all of them the type's lowest value
        out = call(fn, q, low, v, torch.empty_like(q), 1.0)
        assert (out.float() - v.float().mean(dim=1, keepdim=True)).abs().max() < 2e-3
        q[:, Lq - 1] = float("nan")                                   # a query that is no number has no result, its neighbours have theirs
        out = call(fn, q, k, v, torch.empty_like(q), 1.0)
        assert torch.isnan(out[:, Lq - 1]).all()
        assert torch.equal(out[:, :Lq - 1], v[:, 499:].expand(1, Lq - 1, 1, 64))


@BOTH
@pytest.mark.parametrize("order", ["blhd", "bhld", "lbhd", "hlbd"])
@pytest.mark.parametrize("pads", [(0, 0, 0), (8, 16, 24)])
def test_strides_and_orders(fn, order, pads):
    for Lq, D in ((1, 64), (50, 64), (50, 80)):
        run(fn, 3, Lq, 90, 4, 2, D, pads=pads, order=order, lens=[90, 50, 33])


def test_keys_and_values_beside_each_other_and_broadcast():
    import torch
    states = torch.randn((2, 100, 2, 3, 64), device="cuda:0").half()
    q = torch.randn((2, 40, 3, 64), device="cuda:0").half()
    k, v = states[:, :, 0], states[:, :, 1]
    a = call("hb_attention", q, k, v, torch.empty_like(q), 0.125)
    b = call("hb_attention", q, k.contiguous(), v.contiguous(), torch.empty_like(q), 0.125)
    assert torch.equal(a, b)
    one = k[:1].contiguous()
    a = call("hb_attention", q, one.expand(2, -1, -1, -1), one.expand(2, -1, -1, -1), torch.empty_like(q), 0.125)
    b = call("hb_attention", q, one.repeat(2, 1, 1, 1), one.repeat(2, 1, 1, 1), torch.empty_like(q), 0.125)
    assert torch.equal(a, b)


def test_offsets_beyond_32_bits():
    import torch
    Lk, token = 3000, 1 << 20                                         # 2 MB from key to key
    pool = torch.zeros(Lk * token, dtype=torch.float16, device="cuda:0")
    k, v = pool.as_strided((1, Lk, 1, 64), (0, token, 64, 1)), pool.as_strided((1, Lk, 1, 64), (0, token, 64, 1), 64)
    kn, vn = normal(1, (1, Lk, 1, 64)), normal(2, (1, Lk, 1, 64))
    k.copy_(torch.from_numpy(kn))
    v.copy_(torch.from_numpy(vn))
    for Lq in (1, 70):
        qn = normal(3, (1, Lq, 1, 64))
        q = torch.from_numpy(qn).cuda()
        out = call("hb_attention", q, k, v, torch.empty_like(q), 0.125)
        want = oracle.attention(qn, kn, vn, 0.125)
        check(out, want, attention_bound(qn, kn, vn, 0.125, None, None, want), "keys far apart")


@BOTH
def test_repeats_bit_for_bit_on_any_stream(fn):
    import torch
    for Lq, Lk in ((1, 5000), (90, 300)):
        q, k = torch.randn((2, Lq, 4, 64), device="cuda:0").half(), torch.randn((2, Lk, 2, 64), device="cuda:0").half()
        torch.cuda.synchronize()
        outs = []
        for _ in range(3):
            s = torch.cuda.Stream()
            with torch.cuda.stream(s):
                outs.append(call(fn, q, k, k, torch.empty_like(q), 0.2))
            s.synchronize()
        assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


def test_refusals():
    import torch
    f16 = lambda *s: torch.zeros(s, dtype=torch.float16, device="cuda:0")
    ok = dict(q=f16(2, 3, 4, 64), k=f16(2, 5, 2, 64), v=f16(2, 5, 2, 64), out=f16(2, 3, 4, 64), scale=1.0)
    for bad in (dict(k=f16(1, 5, 2, 64)), dict(k=f16(2, 5, 2, 32)), dict(v=f16(2, 6, 2, 64)), dict(out=f16(2, 3, 4, 32)), dict(q=f16(2, 3, 4, 64).float()),
                dict(key_len=torch.zeros(2, dtype=torch.int64, device="cuda:0")), dict(key_len=torch.zeros(3, dtype=torch.int32, device="cuda:0")),
                dict(key_mask=torch.zeros((2, 4), dtype=torch.uint8, device="cuda:0")), dict(key_mask=torch.zeros((2, 5), device="cuda:0")), dict(q=ok["q"].transpose(2, 3))):
        with pytest.raises(AssertionError):
            hb.hb_attention(**{**ok, **bad})

    def code(**kw):
        with pytest.raises(hb.HbError) as e:
            hb.hb_attention(**{**ok, **kw})
        return e.value.code
    assert code(k=f16(2, 5, 3, 64), v=f16(2, 5, 3, 64)) == hb.HB_ERR_INVALID_ARG                  # 4 heads over 3
    assert code(q=f16(2, 3, 4, 60), k=f16(2, 5, 2, 60), v=f16(2, 5, 2, 60), out=f16(2, 3, 4, 60)) in (hb.HB_ERR_UNSUPPORTED, hb.HB_ERR_INVALID_ARG)
    assert code(q=f16(2, 3, 4, 136), k=f16(2, 5, 2, 136), v=f16(2, 5, 2, 136), out=f16(2, 3, 4, 136)) == hb.HB_ERR_UNSUPPORTED
    assert code(scale=float("nan")) == hb.HB_ERR_INVALID_ARG and code(scale=float("inf")) == hb.HB_ERR_INVALID_ARG
    assert code(k=f16(2, 5, 2, 72)[..., 4:68]) == hb.HB_ERR_INVALID_ARG                           # an address between 16 bytes
    assert code(k=f16(2, 5, 2 * 68).as_strided((2, 5, 2, 64), (680, 136, 68, 1))) == hb.HB_ERR_INVALID_ARG
