"""The example that runs the token operators together, against the fp64 oracle step by step."""
import os
import sys

import numpy as np
import pytest

import oracle

pytestmark = pytest.mark.gpu


def test_block_against_the_oracle():
    import torch
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    from image_text_block import ImageTextBlock
    B, size, S = 2, 12, 9
    block = ImageTextBlock(B, size, S, text=48, heads=4, channels=32, hidden=200, seed=3)
    pixels = torch.rand((B, size, size, 64), device="cuda").mul_(2).sub_(1).half()
    caption = torch.randn((B, S, 48), device="cuda").half()
    caption[1, 4:] = float("nan")                                     # behind the caption's end
    lengths = torch.tensor([S, 4], dtype=torch.int32, device="cuda")
    got = block(pixels, caption, lengths).double().cpu().numpy()
    again = block(pixels, caption, lengths).double().cpu().numpy()
    assert np.array_equal(got, again)
    f64 = lambda t: t.double().cpu().numpy()
    half = lambda a: a.astype(np.float16).astype(np.float64)          # what leaves a step
    bits = lambda t: t.cpu().numpy().view(np.uint16)
    w, b = {n: f64(t) for n, t in block.w.items()}, {n: f64(t) for n, t in block.b.items()}
    L, H, D = size * size, 4, 32
    x = half(oracle.linear(half(oracle.conv3x3(bits(pixels), bits(block.conv))).reshape(B * L, 64), w["in"], b["in"]))
    q = half(oracle.linear(x, w["q"], b["q"])).reshape(B, L, H, D)
    q = half(oracle.rope_axes(q, block.positions.cpu().numpy(), f64(block.freq), block.sections, False))
    with np.errstate(invalid="ignore"):
        kv = half(oracle.linear(f64(caption).reshape(B * S, 48), w["kv"], b["kv"])).reshape(B, S, 2, H, D)
    seen = half(oracle.attention(q, kv[:, :, 0], kv[:, :, 1], D ** -0.5, [S, 4])).reshape(B * L, H * D)
    x = half(oracle.linear(seen, w["out"], b["out"], x))
    x = oracle.linear(half(oracle.linear(x, w["up"], b["up"], None, "gelu")), w["down"], b["down"], x)
    # seven roundings to fp16 on the way, each at most 2^-11 of values of a few units, through matrices of norm 1 to 2
    assert np.isfinite(got).all() and np.abs(got.reshape(B * L, -1) - x).max() <= 2e-2 * max(1.0, np.abs(x).max())
    assert np.sqrt(np.mean((got.reshape(B * L, -1) - x) ** 2)) <= 2e-3 * np.sqrt(np.mean(x ** 2))
