"""hb_linear and its twin against the fp64 oracle: sizes around every tile edge, one row, odd pitches and addresses, rows between NaN,
results between canaries, the activations, both output types, the residual in place, and what is refused."""
import numpy as np
import pytest

import oracle
from paper_2512_02371_amd import hb
from tokentest import check, inside, linear_bound, normal, untouched

pytestmark = pytest.mark.gpu
BOTH = pytest.mark.parametrize("fn", ["hb_linear", "hb_linear_valu"])


def run(fn, M, N, K, act="none", bias=True, residual=False, f32=False, pads=(0, 0, 0, 0), leads=(0, 0, 0, 0), seed=1, in_place=False):
    import torch
    x, w = normal(seed, (M, K)), normal(seed + 1, (N, K), K ** -0.5)
    b = normal(seed + 2, (N,)) if bias else None
    kind = np.float32 if f32 else np.float16
    r = normal(seed + 3, (M, N)).astype(kind) if residual or in_place else None
    _, dx = inside(torch, x, pads[0], leads[0])
    _, dw = inside(torch, w, pads[1], leads[1])
    db = None if b is None else inside(torch, b[None], 0, leads[1] % 8)[1][0]
    dr = None if r is None else inside(torch, r, pads[2], leads[2])[1]
    buf, out = inside(torch, r if in_place else np.full((M, N), 7.0, kind), pads[3], leads[3], 7.0)
    if in_place:
        dr = out
    size = hb.hb_linear_workspace_size(M, N, K)
    ws = torch.full((size,), 0xff, dtype=torch.uint8, device="cuda:0") if size else None
    print(fn, M, N, K, act, bias, residual, f32, pads, leads, in_place, flush=True)
    getattr(hb, fn)(dx, dw, out, ws, db, dr, act)
    torch.cuda.synchronize()
    want = oracle.linear(x, w, b, r, act)
    check(out, want, linear_bound(x, w, b, r, act, want, f32), f"{fn} {M} x {N} x {K}")
    assert untouched(torch, buf, out, 7.0), "wrote beside its output"


@BOTH
@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (1, 16, 8), (1, 17, 65), (2, 64, 64), (15, 33, 31), (16, 16, 32), (17, 128, 40), (33, 100, 129), (63, 65, 64),
                                   (64, 64, 128), (65, 129, 72), (127, 255, 136), (128, 128, 192), (129, 127, 63), (200, 300, 96), (255, 257, 256),
                                   (256, 256, 64), (257, 513, 200), (300, 64, 1), (5, 1000, 7), (1000, 8, 16), (640, 384, 320)])
def test_sizes(fn, M, N, K):
    run(fn, M, N, K, "gelu", True, True)


@pytest.mark.parametrize("M,N,K", [(1, 4096, 1024), (1, 64, 8192), (3, 1000, 4097), (16, 2048, 512), (31, 333, 2048), (48, 96, 3000), (64, 512, 8192), (100, 64, 5000),
                                   (2048, 64, 64), (5000, 48, 80), (1030, 1026, 520), (700, 2049, 1001), (4100, 256, 144), (513, 769, 2056)])
def test_larger_sizes(M, N, K):
    run("hb_linear", M, N, K, "silu", True, True, True)
    run("hb_linear", M, N, K, "none", False, False, False)


@BOTH
@pytest.mark.parametrize("act", ["none", "relu", "gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("f32", [False, True])
def test_epilogues(fn, act, f32):
    for bias in (False, True):
        for residual in (False, True):
            run(fn, 70, 90, 50, act, bias, residual, f32)
            run(fn, 3, 90, 56, act, bias, residual, f32)
    run(fn, 70, 90, 64, act, True, True, f32, in_place=True)
    run(fn, 1, 90, 512, act, True, True, f32, in_place=True)


@BOTH
@pytest.mark.parametrize("pads,leads", [((8, 0, 0, 0), (0, 0, 0, 0)), ((0, 8, 8, 16), (8, 8, 8, 8)), ((1, 0, 3, 5), (0, 0, 0, 0)), ((0, 3, 0, 0), (1, 1, 1, 1)),
                                        ((4, 4, 4, 4), (4, 2, 6, 2)), ((7, 9, 11, 13), (3, 5, 7, 1))])
@pytest.mark.parametrize("M,N,K", [(1, 100, 96), (20, 72, 64), (140, 136, 128), (300, 260, 72), (131, 67, 59)])
def test_pitches_and_addresses(fn, pads, leads, M, N, K):
    run(fn, M, N, K, "relu", True, True, False, pads, leads)
    run(fn, M, N, K, "relu", True, True, True, pads, leads)


@BOTH
def test_infinities_stay_in_their_row_and_column(fn):
    import torch
    M, N, K = 150, 140, 75
    x, w = normal(5, (M, K)), normal(6, (N, K), K ** -0.5)
    x[7, 3], x[149, 74] = np.inf, np.nan
    want = oracle.linear(np.where(np.isfinite(x), x, 0), w)
    out = torch.empty((M, N), dtype=torch.float16, device="cuda:0")
    size = hb.hb_linear_workspace_size(M, N, K)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda:0") if size else None
    getattr(hb, fn)(torch.from_numpy(x).cuda(), torch.from_numpy(w).cuda(), out, ws)
    got = out.float().cpu().numpy()
    rows = np.ones(M, bool)
    rows[[7, 149]] = False
    assert np.isfinite(got[rows]).all() and np.isnan(got[149]).all() and (np.isinf(got[7]) | np.isnan(got[7])).all()
    assert np.abs(got[rows] - want[rows]).max() < 2e-2
    out32 = torch.empty((M, N), dtype=torch.float32, device="cuda:0")
    big = torch.full((M, K), 60000.0, dtype=torch.float16, device="cuda:0")
    getattr(hb, fn)(big, torch.ones((N, K), dtype=torch.float16, device="cuda:0"), out, ws)
    assert torch.isinf(out).all()                                     # beyond fp16
    getattr(hb, fn)(big, torch.ones((N, K), dtype=torch.float16, device="cuda:0"), out32, ws)
    assert (out32 == 60000.0 * K - K * (60000.0 - float(np.float16(60000.0)))).all()


def test_offsets_beyond_32_bits():
    import torch
    M, N, K, pitch = 1100, 40, 72, 2 << 20
    pool = torch.zeros(M * pitch, dtype=torch.float16, device="cuda:0")           # 4.6 GB: rows 2^22 bytes apart
    x = pool.as_strided((M, K), (pitch, 1))
    xs, w = normal(8, (M, K)), normal(9, (N, K), K ** -0.5)
    x.copy_(torch.from_numpy(xs))
    out = torch.empty(M * pitch // 2, dtype=torch.float32, device="cuda:0").as_strided((M, N), (pitch // 2, 1))
    size = hb.hb_linear_workspace_size(M, N, K)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda:0") if size else None
    hb.hb_linear(x, torch.from_numpy(w).cuda(), out, ws)
    want = oracle.linear(xs, w)
    check(out, want, linear_bound(xs, w, None, None, "none", want, True), "rows far apart")


@BOTH
def test_repeats_bit_for_bit_on_any_stream(fn):
    import torch
    for M, N, K in ((1, 512, 4096), (40, 200, 3000), (300, 500, 256)):
        x, w = torch.from_numpy(normal(1, (M, K))).cuda(), torch.from_numpy(normal(2, (N, K))).cuda()
        size = hb.hb_linear_workspace_size(M, N, K)
        outs = []
        for _ in range(3):
            s = torch.cuda.Stream()
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                ws = torch.full((size,), 0x7f, dtype=torch.uint8, device="cuda:0") if size else None
                outs.append(getattr(hb, fn)(x, w, torch.empty((M, N), dtype=torch.float32, device="cuda:0"), ws))
            s.synchronize()
        assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


def test_refusals():
    import torch
    f16 = lambda *s: torch.zeros(s, dtype=torch.float16, device="cuda:0")
    ok = dict(x=f16(4, 8), w=f16(6, 8), out=f16(4, 6), act="none")
    for bad in (dict(x=f16(4, 7)), dict(w=f16(6, 9)), dict(out=f16(4, 5)), dict(out=f16(4, 6).double()), dict(x=f16(4, 8).float()), dict(bias=f16(5)),
                dict(bias=f16(6).float()), dict(residual=f16(4, 5)), dict(residual=f16(4, 6).float()), dict(x=f16(8, 4).t()), dict(x=f16(4, 8).cpu())):
        with pytest.raises(AssertionError):
            hb.hb_linear(**{**ok, **bad})
    with pytest.raises(KeyError):
        hb.hb_linear(**{**ok, "act": "swish"})
    with pytest.raises(hb.HbError) as e:                              # overlapping rows
        hb.hb_linear(**{**ok, "x": f16(64).as_strided((4, 8), (4, 1))})
    assert e.value.code == hb.HB_ERR_INVALID_ARG
    M, N, K = 64, 512, 8192
    if hb.hb_linear_workspace_size(M, N, K):
        for ws in (None, torch.empty(16, dtype=torch.uint8, device="cuda:0")):
            with pytest.raises(hb.HbError) as e:
                hb.hb_linear(f16(M, K), f16(N, K), f16(M, N), ws)
            assert e.value.code == hb.HB_ERR_WORKSPACE
