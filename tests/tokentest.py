"""Inputs, guards and error bounds of the token operators' GPU tests.

The bounds follow from the number formats and were derived before the tests first ran:
  - one rounding to fp16: 2^-11 of the value, or 2^-25 (half the smallest subnormal); none that matters for fp32 output;
  - a sum of n products in fp32, in any order, rounded or truncated at each step: (n + 8) 2^-23 of the sum of magnitudes;
  - activations: at most 1.13 times their argument's error, and 2^-20 of the argument's size for exp, erf and the division;
  - a weight of attention: its score's error, absolute, taken twice (the score's and the maximum's), 2^-11 for its rounding to
    fp16 and 2^-25 of the largest weight where that is subnormal;
  - the rotation: 1e-5 of the pair for the angle, sin and cos (a fiftieth of fp16's rounding).
"""
import numpy as np

F16, TINY = 2.0 ** -11, 2.0 ** -25


def normal(seed, shape, std=1.0):
    return (np.random.default_rng(seed).normal(size=shape) * std).astype(np.float16)


def check(got, want, bound, what):
    got = got.double().cpu().numpy()
    assert got.shape == want.shape, what
    bad = ~(np.abs(got - want) <= bound)
    if bad.any():
        i = tuple(np.argwhere(bad)[0])
        raise AssertionError(f"{what}: {bad.sum()} of {bad.size} out of bounds, first at {i}: {got[i]} for {want[i]}, bound {np.broadcast_to(bound, want.shape)[i]}")


def linear_bound(x, w, bias, residual, act, want, f32):
    x, w = np.abs(x.astype(np.float64)), np.abs(w.astype(np.float64))
    size = x @ w.T
    if bias is not None:
        size = size + np.abs(bias.astype(np.float64))[None, :]
    e = (x.shape[1] + 8) * 2.0 ** -23 * size * 1.13 + (0.0 if act in ("none", "relu") else 2.0 ** -20 * size)
    if residual is not None:
        e = e + 2.0 ** -22 * (size + np.abs(residual.astype(np.float64)))
    return e + (2.0 ** -22 * np.abs(want) if f32 else F16 * np.abs(want) + TINY)


def attention_bound(q, k, v, scale, key_len, key_mask, want):
    """Elementwise; k and v as the kernel sees them, visible keys only."""
    q, k, v = (t.astype(np.float64) for t in (q, k, v))
    B, Lq, Hq, D = q.shape
    Lk, Hkv = k.shape[1], k.shape[2]
    out = np.full(q.shape, TINY)
    for b in range(B):
        n = Lk if key_len is None else min(max(int(key_len[b]), 0), Lk)
        seen = [j for j in range(n) if key_mask is None or key_mask[b, j]]
        if not seen:
            continue
        for h in range(Hq):
            kk, vv = k[b, seen, h // (Hq // Hkv)], v[b, seen, h // (Hq // Hkv)]
            s = scale * (q[b, :, h] @ kk.T)
            size = abs(scale) * (np.abs(q[b, :, h]) @ np.abs(kk).T)
            ds = (D + 8) * 2.0 ** -23 * size + 2.0 ** -22 * np.abs(s)
            err = 2.0 * ds.max(axis=1, keepdims=True)
            e = np.exp(s - s.max(axis=1, keepdims=True))
            total = e.sum(axis=1, keepdims=True)
            spread = (e @ np.abs(vv)) / total
            out[b, :, h] += (2.0 * err + 2.0 * F16 + (len(seen) + 8) * 2.0 ** -23) * spread + TINY * np.abs(vv).sum(axis=0) / total + F16 * np.abs(want[b, :, h])
    return out


def inside(torch, array, pad=0, lead=0, fill=float("nan"), device="cuda:0"):
    """The array's values as a view of a larger buffer of `fill`: `pad` elements behind every row, `lead` in front of the first."""
    t = torch.from_numpy(np.ascontiguousarray(array))
    rows = int(np.prod(t.shape[:-1]))
    width = t.shape[-1] + pad
    buf = torch.full((lead + rows * width + 64,), fill, dtype=t.dtype)
    view = buf[lead:lead + rows * width].view(rows, width)
    view[:, :t.shape[-1]] = t.reshape(rows, -1)
    buf = buf.to(device)
    strides = [0] * t.dim()
    strides[-1], step = 1, width
    for i in range(t.dim() - 2, -1, -1):
        strides[i], step = step, step * t.shape[i]
    return buf, buf.as_strided(t.shape, strides, lead)


def untouched(torch, buf, view, fill):
    """Whether everything of buf outside the view still holds fill."""
    seen = torch.zeros_like(buf, dtype=torch.bool)
    seen.as_strided(view.shape, view.stride(), view.storage_offset()).fill_(True)
    return bool((buf[~seen] == fill).all())
