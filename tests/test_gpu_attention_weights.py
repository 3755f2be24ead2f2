"""How exact hb_attention is where the keys are split and rows are those of one wave (single tokens): like its result rounded once.

With independent errors the root mean square is sqrt(a^2 + b^2).  a: rounding the result to fp16, computed from the exact result.  Weights that are rounded
to fp16 before their product with random values add b = a (each term is off by as much as the sum is), 1.41 a in all; weights held to 2^-20 and
sums in fp32 add b < 0.01 a.  The limit of 1.1 a allows b = 0.46 a.  Sampling moves the root mean square of 2000 errors by 3 % at most."""
import numpy as np
import pytest

import oracle
from paper_2512_02371_amd import hb
from tokentest import normal

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,Lq,Lk,Hq,Hkv,D,keys", [(2, 1, 8192, 32, 8, 128, "all"), (4, 1, 5001, 16, 4, 64, "lengths"), (1, 5, 8200, 16, 16, 40, "all"), (3, 2, 3001, 16, 2, 80, "mask"),
                                                   (2, 8, 4000, 4, 4, 96, "mask"), (1, 1, 20000, 64, 2, 32, "lengths")])
def test_split_keys(B, Lq, Lk, Hq, Hkv, D, keys):
    import torch
    rng = np.random.default_rng(Lk)
    q, k, v = normal(1, (B, Lq, Hq, D)), normal(2, (B, Lk, Hkv, D)), normal(3, (B, Lk, Hkv, D))
    lens = rng.integers(Lk // 2, Lk + 1, size=B).astype(np.int32) if keys == "lengths" else None
    mask = (rng.random((B, Lk)) < 0.75).astype(np.uint8) if keys == "mask" else None
    size = hb.hb_attention_workspace_size(B, Lq, Lk, Hq, Hkv, D)
    assert size > 0 and Lq * (Hq // Hkv) <= 32, "split keys, rows of one wave"
    up = lambda a: None if a is None else torch.from_numpy(a).cuda()
    print("hb_attention", B, Lq, Lk, Hq, Hkv, D, keys, flush=True)
    dq = up(q)
    out = hb.hb_attention(dq, up(k), up(v), torch.empty_like(dq), D ** -0.5, torch.empty(size, dtype=torch.uint8, device="cuda:0"), up(lens), up(mask))
    want = oracle.attention(q, k, v, D ** -0.5, lens, mask)
    rms = lambda a: float(np.sqrt(np.mean(np.square(a))))
    once = rms(want.astype(np.float16).astype(np.float64) - want)
    got = rms(out.double().cpu().numpy() - want)
    assert want.size >= 2000 and got <= 1.1 * once, (got / once, got / rms(want))


@pytest.mark.parametrize("fn", ["hb_attention", "hb_attention_valu"])
@pytest.mark.parametrize("scale", [3.0e38, -3.0e38, 3.4028234e38])
def test_scales_near_the_largest_number(fn, scale):
    """Scores of 0 stay 0: the scale in powers of two (1.44 times as large) must not become infinite."""
    import torch
    q = torch.zeros((1, 3, 2, 64), dtype=torch.float16, device="cuda:0")
    k, v = (torch.randn((1, 100, 2, 64), device="cuda:0").half() for _ in range(2))
    out = getattr(hb, fn)(q, k, v, torch.empty_like(q), scale)
    want = v.double().mean(dim=1, keepdim=True).expand(1, 3, 2, 64)
    assert ((out.double() - want).abs() <= 2.0 ** -10 * v.double().abs().mean(dim=1, keepdim=True)).all()
