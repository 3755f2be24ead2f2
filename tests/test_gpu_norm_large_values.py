"""hb_group_norm of fp32 values whose squares pass fp32 while those of their differences from the mean hold in it: what include/hb.h asks for, and no more.

The bounds are normtest.norm_bound's.  Means are 2e19 to 1e20, deviations 2e15: the mean's rounding is 2^-23 of it, up to 6e-3 of a deviation, and sums of 16 times the
squares (at most 2e6 values of a group) stay below 2e38.
"""
import numpy as np
import pytest

import oracle
from normtest import norm_bound, pixels
from paper_2512_02371_amd import hb

pytestmark = pytest.mark.gpu

# images, pixels, channels, groups, elements between two pixels: every way in which rows stream (vectors of one group, of two, of more; whole ones or not; few chunks and many), last rows
# that are short and fall to lanes with no row before them, and groups that stay in a workgroup
CALLS = [
    (1, 5041, 4, 1, 4), (1, 5377, 24, 3, 27), (1, 30000, 64, 32, 64), (3, 1079, 180, 12, 204), (1, 1315, 5, 1, 8), (1, 16819, 5, 1, 8), (1, 265, 39, 3, 39), (1, 519, 145, 5, 145),
    (1, 385, 27, 1, 27), (1, 515, 135, 5, 135), (1, 201, 52, 4, 52), (1, 788, 148, 4, 151), (1, 1492, 7, 1, 7), (1, 520, 135, 5, 135), (1, 2694, 1, 1, 3), (1, 34262, 1, 1, 3),
    (1, 751, 15, 5, 15), (1, 44009, 3, 3, 3), (1, 1162, 9, 3, 9), (1, 14435, 9, 3, 9), (1, 2618, 4, 4, 4), (1, 3614, 36, 12, 36), (1, 1746, 6, 2, 6), (1, 43592, 3, 1, 3),
    (2, 64, 64, 8, 64), (2, 37, 30, 6, 33), (1, 1, 9, 1, 9), (5, 9, 3, 3, 3),
]


def run(torch, x, groups, pixel, kind):
    N, P, C = x.shape
    dx = pixels(torch, x, pixel - C)[1]
    out = torch.empty((N, P, C), dtype=kind, device="cuda:0")
    size = hb.hb_group_norm_workspace_size(N, P, C, groups)
    hb.hb_group_norm(dx, out, groups, workspace=torch.full((size,), 0xff, dtype=torch.uint8, device="cuda:0") if size else None)
    return out.double().cpu().numpy()


@pytest.mark.parametrize("N,P,C,groups,pixel", CALLS)
def test_differences_that_hold_in_fp32(N, P, C, groups, pixel):
    import torch
    rng = np.random.default_rng(P + C)
    means = rng.uniform(2e19, 1e20, size=(N, 1, groups, 1)) * np.where(rng.random((N, 1, groups, 1)) < 0.5, -1.0, 1.0)
    x = (means + 2e15 * rng.normal(size=(N, P, groups, C // groups))).reshape(N, P, C).astype(np.float32)
    for kind in (torch.float32, torch.float16):
        print(N, P, C, groups, pixel, kind, flush=True)
        got, want = run(torch, x, groups, pixel, kind), oracle.group_norm(x, groups)
        assert np.isfinite(got).all(), f"{(~np.isfinite(got)).sum()} of {got.size} are not finite"
        bad = ~(np.abs(got - want) <= norm_bound(x, groups, None, None, 1e-5, "none", want, kind is torch.float32))
        assert not bad.any(), (int(bad.sum()), got[bad][0], want[bad][0])


@pytest.mark.parametrize("N,P,C,groups,pixel", CALLS)
def test_equal_values(N, P, C, groups, pixel):
    """No differences at all: whatever the mean's rounding makes of them, it is a number."""
    import torch
    x = np.broadcast_to(2.0 ** 66 * np.arange(1, groups + 1, dtype=np.float64)[:, None], (N, P, groups, C // groups)).reshape(N, P, C).astype(np.float32)
    print(N, P, C, groups, pixel, flush=True)
    assert np.isfinite(run(torch, x, groups, pixel, torch.float32)).all()
