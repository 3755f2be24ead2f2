"""hb_linear_i8 and its twin against the oracle, whose sums are integers: sizes around every tile edge, one row, odd pitches and addresses, rows between
other values, results between canaries, the activations, both output types, the residual in place, the largest sums, and what is refused."""
import numpy as np
import pytest

import oracle
from normtest import bytes_rows, i8_bound
from paper_2512_02371_amd import hb
from tokentest import check, inside, normal, untouched

pytestmark = pytest.mark.gpu
BOTH = pytest.mark.parametrize("fn", ["hb_linear_i8", "hb_linear_i8_valu"])


def workspace(torch, M, N, K):
    size = hb.hb_linear_i8_workspace_size(M, N, K)
    return torch.full((size,), 0xff, dtype=torch.uint8, device="cuda:0") if size else None


def run(fn, M, N, K, act="none", bias=True, residual=False, f32=False, pads=(0, 0, 0, 0), leads=(0, 0, 0, 0), seed=1, in_place=False):
    import torch
    x, xs = bytes_rows(seed, (M, K))
    w, ws = bytes_rows(seed + 1, (N, K))
    ws = (ws * np.float32(K ** -0.5)).astype(np.float32)
    b = normal(seed + 2, (N,)) if bias else None
    kind = np.float32 if f32 else np.float16
    r = normal(seed + 3, (M, N)).astype(kind) if residual or in_place else None
    _, dx = inside(torch, x, pads[0], leads[0], 101)
    _, dw = inside(torch, w, pads[1], leads[1], -99)
    up = lambda t: torch.from_numpy(t).cuda()
    dr = None if r is None else inside(torch, r, pads[2], leads[2])[1]
    buf, out = inside(torch, r if in_place else np.full((M, N), 7.0, kind), pads[3], leads[3], 7.0)
    if in_place:
        dr = out
    print(fn, M, N, K, act, bias, residual, f32, pads, leads, in_place, flush=True)
    getattr(hb, fn)(dx, dw, up(xs), up(ws), out, workspace(torch, M, N, K), None if b is None else up(b), dr, act)
    torch.cuda.synchronize()
    want = oracle.linear_i8(x, w, xs, ws, b, r, act)
    check(out, want, i8_bound(x, w, xs, ws, b, r, act, want, f32), f"{fn} {M} x {N} x {K}")
    assert untouched(torch, buf, out, 7.0), "wrote beside its output"


@BOTH
@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (1, 16, 8), (1, 17, 65), (2, 64, 64), (15, 33, 31), (16, 16, 32), (17, 128, 40), (33, 100, 129), (63, 65, 64),
                                   (64, 64, 128), (65, 129, 72), (127, 255, 136), (128, 128, 192), (129, 127, 63), (200, 300, 96), (255, 257, 256),
                                   (256, 256, 64), (257, 513, 200), (300, 64, 1), (5, 1000, 7), (1000, 8, 16), (640, 384, 320), (70, 70, 144), (70, 70, 143), (70, 70, 145), (3, 40, 15), (3, 40, 17)])
def test_sizes(fn, M, N, K):
    run(fn, M, N, K, "gelu", True, True)


@pytest.mark.parametrize("M,N,K", [(1, 4096, 1024), (1, 64, 8192), (3, 1000, 4097), (16, 2048, 512), (31, 333, 2048), (48, 96, 3000), (64, 512, 8192), (100, 64, 5000),
                                   (2048, 64, 64), (5000, 48, 80), (1030, 1026, 528), (700, 2049, 1001), (4100, 256, 144), (513, 769, 2064), (1, 8, 100000), (40, 72, 131071)])
def test_larger_sizes(M, N, K):
    run("hb_linear_i8", M, N, K, "silu", True, True, True)
    run("hb_linear_i8", M, N, K, "none", False, False, False)


@BOTH
@pytest.mark.parametrize("act", ["none", "relu", "gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("f32", [False, True])
def test_epilogues(fn, act, f32):
    for bias in (False, True):
        for residual in (False, True):
            run(fn, 70, 90, 50, act, bias, residual, f32)
            run(fn, 3, 90, 64, act, bias, residual, f32)
    run(fn, 70, 90, 64, act, True, True, f32, in_place=True)
    run(fn, 1, 90, 512, act, True, True, f32, in_place=True)


@BOTH
@pytest.mark.parametrize("pads,leads", [((16, 0, 0, 0), (0, 0, 0, 0)), ((0, 16, 8, 16), (16, 16, 8, 8)), ((1, 0, 3, 5), (0, 0, 0, 0)), ((0, 3, 0, 0), (1, 1, 1, 1)),
                                        ((4, 4, 4, 4), (4, 2, 6, 2)), ((7, 9, 11, 13), (3, 5, 7, 1)), ((0, 0, 0, 0), (8, 0, 0, 0)), ((2, 6, 0, 0), (2, 12, 0, 0))])
@pytest.mark.parametrize("M,N,K", [(1, 100, 96), (20, 72, 64), (140, 136, 128), (300, 260, 72), (131, 67, 59), (50, 40, 1000)])
def test_pitches_and_addresses(fn, pads, leads, M, N, K):
    run(fn, M, N, K, "relu", True, True, False, pads, leads)
    run(fn, M, N, K, "relu", True, True, True, pads, leads)


@BOTH
def test_largest_sums(fn):
    """-128 times -128, as many as the limit lets; and all but one that cancel."""
    import torch
    K = hb.HB_LINEAR_I8_MAX_K
    for M, N in ((1, 3), (40, 20), (70, 70)):
        x = torch.full((M, K), -128, dtype=torch.int8, device="cuda:0")
        w = torch.full((N, K), -128, dtype=torch.int8, device="cuda:0")
        w[1::2] = 127
        w[2, ::2] = 127
        one = lambda n: torch.ones(n, device="cuda:0")
        out = getattr(hb, fn)(x, w, one(M), one(N), torch.empty((M, N), dtype=torch.float32, device="cuda:0"), workspace(torch, M, N, K))
        want = (w.double().sum(dim=1) * -128.0).float().expand(M, N)
        assert torch.equal(out, want)


@BOTH
def test_scales_stay_in_their_row_and_column(fn):
    import torch
    for M, N, K in ((150, 140, 80), (3, 140, 75), (300, 70, 2048)):
        x, xs = bytes_rows(5, (M, K))
        w, ws = bytes_rows(6, (N, K))
        xs[M - 1], xs[1], ws[7], xs[0] = np.nan, 0.0, np.inf, -xs[0]
        w[9] = 0
        up = lambda t: torch.from_numpy(t).cuda()
        got = getattr(hb, fn)(up(x), up(w), up(xs), up(ws), torch.empty((M, N), dtype=torch.float32, device="cuda:0"), workspace(torch, M, N, K)).cpu().numpy()
        with np.errstate(invalid="ignore"):
            want = oracle.linear_i8(x, w, xs, ws)
        assert np.array_equal(np.isnan(got), np.isnan(want)) and np.isnan(want[M - 1]).all()
        assert np.array_equal(np.isinf(got), np.isinf(want)) and not want[1, 8:].any() and not got[1, 8:].any()
        fine = np.isfinite(want)
        assert (np.abs(got[fine] - want[fine]) <= 2.0 ** -21 * np.abs(want[fine])).all()


def test_offsets_beyond_32_bits():
    import torch
    M, N, K, pitch = 2100, 40, 80, 1 << 21
    pool = torch.zeros(M * pitch, dtype=torch.int8, device="cuda:0")              # 4.4 GB: rows 2^21 bytes apart
    dx = pool.as_strided((M, K), (pitch, 1))
    x, xs = bytes_rows(8, (M, K))
    w, ws = bytes_rows(9, (N, K))
    dx.copy_(torch.from_numpy(x))
    out = torch.empty(M * pitch // 2, dtype=torch.float32, device="cuda:0").as_strided((M, N), (pitch // 2, 1))
    up = lambda t: torch.from_numpy(t).cuda()
    hb.hb_linear_i8(dx, up(w), up(xs), up(ws), out, workspace(torch, M, N, K))
    want = oracle.linear_i8(x, w, xs, ws)
    check(out, want, i8_bound(x, w, xs, ws, None, None, "none", want, True), "rows far apart")


@BOTH
def test_repeats_bit_for_bit_on_any_stream(fn):
    import torch
    for M, N, K in ((1, 512, 4096), (40, 200, 3000), (300, 500, 256)):
        x, xs = (torch.from_numpy(t).cuda() for t in bytes_rows(1, (M, K)))
        w, ws = (torch.from_numpy(t).cuda() for t in bytes_rows(2, (N, K)))
        outs = []
        for _ in range(3):
            s = torch.cuda.Stream()
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                outs.append(getattr(hb, fn)(x, w, xs, ws, torch.empty((M, N), dtype=torch.float32, device="cuda:0"), workspace(torch, M, N, K)))
            s.synchronize()
        assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


def test_equals_its_twin_bit_for_bit():
    """The sums are integers: the order in which they are added is not in the result (fp32 output, no exponential)."""
    import torch
    for M, N, K in ((1, 300, 4000), (40, 200, 3000), (300, 500, 256), (130, 70, 9001), (1000, 1000, 1024)):
        x, xs = (torch.from_numpy(t).cuda() for t in bytes_rows(3, (M, K)))
        w, ws = (torch.from_numpy(t).cuda() for t in bytes_rows(4, (N, K)))
        a, b = (f(x, w, xs, ws, torch.empty((M, N), dtype=torch.float32, device="cuda:0"), workspace(torch, M, N, K)) for f in (hb.hb_linear_i8, hb.hb_linear_i8_valu))
        assert torch.equal(a, b)


def test_refusals():
    import torch
    i8 = lambda *s: torch.zeros(s, dtype=torch.int8, device="cuda:0")
    f16, f32 = (lambda *s: torch.zeros(s, dtype=torch.float16, device="cuda:0")), (lambda *s: torch.zeros(s, device="cuda:0"))
    ok = dict(x=i8(4, 16), w=i8(6, 16), x_scale=f32(4), w_scale=f32(6), out=f16(4, 6))
    for bad in (dict(x=i8(4, 15)), dict(w=i8(6, 17)), dict(out=f16(4, 5)), dict(out=f16(4, 6).double()), dict(x=f16(4, 16)), dict(w=i8(6, 16).to(torch.uint8)), dict(x_scale=f32(5)),
                dict(x_scale=f16(4)), dict(w_scale=f32(5)), dict(w_scale=f32(6, 2)[:, 0]), dict(bias=f16(5)), dict(bias=f32(6)), dict(residual=f16(4, 5)), dict(residual=f32(4, 6)), dict(x=i8(16, 4).t()),
                dict(x=i8(4, 16).cpu()), dict(x_scale=f32(4).cpu()), dict(bias=f16(6).cpu())):
        with pytest.raises(AssertionError):
            hb.hb_linear_i8(**{**ok, **bad})
    with pytest.raises(KeyError):
        hb.hb_linear_i8(**ok, act="swish")
    with pytest.raises(hb.HbError) as e:                              # overlapping rows
        hb.hb_linear_i8(**{**ok, "x": i8(64).as_strided((4, 16), (8, 1))})
    assert e.value.code == hb.HB_ERR_INVALID_ARG
    with pytest.raises(hb.HbError) as e:
        hb.hb_linear_i8(**{**ok, "x": i8(4, 131072), "w": i8(6, 131072)})
    assert e.value.code == hb.HB_ERR_UNSUPPORTED
    M, N, K = 64, 512, 16384
    if hb.hb_linear_i8_workspace_size(M, N, K):
        for ws in (None, torch.empty(16, dtype=torch.uint8, device="cuda:0")):
            with pytest.raises(hb.HbError) as e:
                hb.hb_linear_i8(i8(M, K), i8(N, K), f32(M), f32(N), f16(M, N), ws)
            assert e.value.code == hb.HB_ERR_WORKSPACE
