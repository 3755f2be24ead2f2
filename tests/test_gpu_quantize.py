"""hb_quantize_rows against the oracle, integer for integer: sizes around every vector and tile edge, strides, ties, zeros, subnormals, NaN and infinities."""
import numpy as np
import pytest

import oracle
from paper_2512_02371_amd import hb
from tokentest import inside, normal, untouched

pytestmark = pytest.mark.gpu


def run(x, x_at=(0, 0), q_at=(0, 0)):
    import torch
    M, K = x.shape
    _, dx = inside(torch, x, *x_at)
    buf, q = inside(torch, np.full((M, K), 77, np.int8), *q_at, fill=77)
    sbuf = torch.full((M + 16,), 7.0, dtype=torch.float32, device="cuda:0")
    print(M, K, x_at, q_at, flush=True)
    hb.hb_quantize_rows(dx, q, sbuf[8:8 + M])
    torch.cuda.synchronize()
    want, scale = oracle.quantize_rows(x)
    got = q.cpu().numpy()
    bad = np.argwhere(got != want)
    assert not len(bad), f"{len(bad)} of {want.size}, first {bad[0]}: {got[tuple(bad[0])]} for {want[tuple(bad[0])]}"
    assert np.array_equal(sbuf[8:8 + M].cpu().numpy(), scale.astype(np.float32), equal_nan=True)
    assert untouched(torch, buf, q, 77) and (sbuf[:8] == 7.0).all() and (sbuf[8 + M:] == 7.0).all(), "wrote beside its output"


@pytest.mark.parametrize("M,K", [(1, 1), (3, 1), (1, 7), (2, 8), (5, 9), (4, 15), (7, 16), (1, 63), (9, 64), (2, 65), (3, 127), (1, 500), (2, 511), (3, 512), (5, 513), (2, 1023), (4, 1024), (3, 1079), (1, 2048),
                                 (2, 2051), (1, 4096), (6, 4095), (2, 5000), (1, 8192), (3, 8200), (1, 16384), (2, 16391), (1, 33000), (2, 70001), (700, 24), (1917, 130), (300, 1000)])
def test_sizes(M, K):
    run(normal(M * 70001 + K, (M, K)))


@pytest.mark.parametrize("x_at,q_at", [((8, 0), (0, 0)), ((0, 8), (8, 8)), ((1, 0), (0, 0)), ((0, 0), (1, 0)), ((0, 1), (0, 3)), ((3, 5), (5, 7)), ((24, 2), (16, 4)), ((2, 0), (4, 4))])
@pytest.mark.parametrize("M,K", [(1, 100), (13, 64), (6, 1001), (5, 2048), (3, 9000), (2, 40001)])
def test_strides_and_addresses(M, K, x_at, q_at):
    run(normal(3, (M, K)), x_at, q_at)


def test_ties_go_to_even():
    # of 254: x / 2 is a half for odd x; all magnitudes, both signs
    x = np.arange(-254, 255).astype(np.float16)
    run(np.stack([x, x * np.float16(2.0 ** -10), x * np.float16(64.0)]))
    # of 2032 and 508: quarters and eighths of a step
    run(np.arange(-2032, 2033).astype(np.float16)[None])
    run(np.arange(-508, 509).astype(np.float16)[None])


def test_every_value_against_many_largest():
    """All finite fp16 values up to the row's largest, for largest values over the whole range, subnormal ones among them."""
    everything = np.arange(0x7c00, dtype=np.uint16).view(np.float16)
    rng = np.random.default_rng(1)
    for top in [1, 2, 3, 127, 254, 1023, 1024, 0x7bff, 0x3c00, 0x3c01, 0x3fff, *rng.integers(4, 0x7c00, 40)]:
        run((everything[:int(top) + 1] * np.where(rng.random(int(top) + 1) < 0.5, -1, 1).astype(np.float16))[None])


def test_zeros_nan_and_infinities():
    for K in (1, 40, 1000, 3001, 20000, 50000):
        x = normal(4, (7, K))
        x[1] = 0.0
        x[2, K - 1], x[3, 0], x[4, K // 2], x[5, :] = np.nan, np.inf, -np.inf, np.nan
        x[6] = -0.0
        run(x)


def test_offsets_beyond_32_bits():
    import torch
    M, K, pitch = 1200, 72, 1 << 22
    pool = torch.zeros(M * pitch, dtype=torch.float16, device="cuda:0")           # 10 GB: rows 2^23 bytes apart
    x = normal(5, (M, K))
    dx = pool.as_strided((M, K), (pitch, 1))
    dx.copy_(torch.from_numpy(x))
    q = torch.zeros(M * pitch, dtype=torch.int8, device="cuda:0").as_strided((M, K), (pitch, 1))
    scale = torch.empty(M, dtype=torch.float32, device="cuda:0")
    hb.hb_quantize_rows(dx, q, scale)
    want, s = oracle.quantize_rows(x)
    assert np.array_equal(q.cpu().numpy(), want) and np.array_equal(scale.cpu().numpy(), s.astype(np.float32))


def test_refusals():
    import torch
    x, q, s = torch.zeros((4, 8), dtype=torch.float16, device="cuda:0"), torch.zeros((4, 8), dtype=torch.int8, device="cuda:0"), torch.zeros(4, device="cuda:0")
    for bad in ((x[:, :7], q, s), (x, q[:3], s), (x.float(), q, s), (x, q.to(torch.uint8), s), (x, q, s[:3]), (x, q, s.half()), (x.cpu(), q, s), (x, q.cpu(), s), (x, q, s.cpu()),
                (x.t(), q.t(), s), (x, q, torch.zeros((4, 2), device="cuda:0")[:, 0])):
        with pytest.raises(AssertionError):
            hb.hb_quantize_rows(*bad)
    for bad in ((x.expand(4, 8).as_strided((4, 8), (4, 1)), q, s), (x, q.as_strided((4, 8), (0, 1)), s)):
        with pytest.raises(hb.HbError) as e:
            hb.hb_quantize_rows(*bad)
        assert e.value.code == hb.HB_ERR_INVALID_ARG
