"""Inputs and error bounds of the GPU tests of hb_group_norm and hb_linear_i8.

The bounds follow from the number formats and were derived before the tests first ran:
  - a sum of n numbers in fp32, in pieces: a term passes at most H = 300 + n / 256 additions, each off by 2^-24 of its result (pieces of at most 128
    numbers of a thread and 128 of a lane, or n / 256 numbers of a thread): H 2^-24 of the sum of magnitudes;
  - the mean: rounded, and what a sum of differences from it is off by: 2^-23 |mean| + H 2^-24 of the mean |difference|;
  - the variance: each difference is off by 2^-24 of itself, its square by 2^-22, their sum by H 2^-24; a mean that is off by e adds e^2;
  - the result before the activation: the mean's error times rstd and weight; the result's own size times half the variance's relative error and
    six roundings (difference, rstd's square root and quotient, its product with the weight, the product, the sum);
  - activations and the rounding of the output: as in tokentest.py.
"""
import numpy as np

from tokentest import F16, TINY


def norm_bound(x, groups, weight, bias, eps, act, want, f32):
    x = x.astype(np.float64)
    N, P, C = x.shape
    D = C // groups
    v = x.reshape(N, P, groups, D)
    n = P * D
    H = 300 + n / 256
    mean = v.mean(axis=(1, 3), keepdims=True)
    d = v - mean
    dm = 2.0 ** -23 * np.abs(mean) + H * 2.0 ** -24 * np.abs(d).mean(axis=(1, 3), keepdims=True)
    var = (d * d).mean(axis=(1, 3), keepdims=True)
    rstd = 1.0 / np.sqrt(var + eps)
    off = ((H + 8) * 2.0 ** -24 * var + dm ** 2) * rstd ** 2              # of var + eps, relative
    flat = lambda t: np.broadcast_to(t, v.shape).reshape(N, P, C)
    w = np.ones(C) if weight is None else np.abs(weight.astype(np.float64))
    b = np.zeros(C) if bias is None else np.abs(bias.astype(np.float64))
    size = flat(np.abs(d) * rstd) * w
    e = flat(dm * rstd) * w + size * (flat(off) + 6 * 2.0 ** -24) + 2.0 ** -23 * (size + b)
    e = 1.13 * e + (0.0 if act in ("none", "relu") else 2.0 ** -20 * (size + b))
    return e + (2.0 ** -23 * np.abs(want) if f32 else F16 * np.abs(want) + TINY)


def i8_bound(x, w, x_scale, w_scale, bias, residual, act, want, f32):
    """The sum is exact; four roundings to the activation, by 2^-24 each of at most the size of product and bias."""
    size = np.abs(x.astype(np.float64) @ w.astype(np.float64).T) * np.abs(x_scale.astype(np.float64))[:, None] * np.abs(w_scale.astype(np.float64))[None, :]
    if bias is not None:
        size = size + np.abs(bias.astype(np.float64))[None, :]
    e = 4 * 2.0 ** -24 * size * 1.13 + (0.0 if act in ("none", "relu") else 2.0 ** -20 * size)
    if residual is not None:
        e = e + 2.0 ** -23 * (size + np.abs(residual.astype(np.float64)))
    return e + (2.0 ** -23 * np.abs(want) if f32 else F16 * np.abs(want) + TINY)


def pixels(torch, array, pad=0, lead=0, gap=0, fill=float("nan"), device="cuda:0"):
    """N x P x C values in a larger buffer of `fill`: `pad` elements behind every pixel, `gap` behind every image, `lead` in front of the first."""
    t = torch.from_numpy(np.ascontiguousarray(array))
    N, P, C = t.shape
    strides = (P * (C + pad) + gap, C + pad, 1)
    buf = torch.full((lead + N * strides[0] + 64,), fill, dtype=t.dtype)
    buf.as_strided(t.shape, strides, lead).copy_(t)
    buf = buf.to(device)
    return buf, buf.as_strided(t.shape, strides, lead)


def bytes_rows(seed, shape):
    """8-bit integers of every value, and scales as of normal rows."""
    rng = np.random.default_rng(seed)
    return rng.integers(-128, 128, size=shape).astype(np.int8), (rng.random(shape[0]) * 0.02 + 0.005).astype(np.float32)
