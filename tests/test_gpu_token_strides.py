"""Strides of dimensions of size 1, which torch gives any value: they have no meaning, and no call is refused or turned elsewhere for them."""
import pytest

from paper_2512_02371_amd import hb

pytestmark = pytest.mark.gpu


def odd(t, dims, by):
    """The same tensor with other strides where its size is 1."""
    assert all(t.shape[d] == 1 for d in dims)
    return t.as_strided(t.shape, [by if d in dims else s for d, s in enumerate(t.stride())], t.storage_offset())


@pytest.mark.parametrize("fn", ["hb_attention", "hb_attention_valu"])
@pytest.mark.parametrize("by", [3, 1 << 21, (1 << 40) + 1])
@pytest.mark.parametrize("B,Lq,Lk,Hq,Hkv,dims", [(1, 5, 7, 4, 2, (0,)), (2, 1, 9, 4, 4, (1,)), (2, 6, 1, 2, 2, (1,)), (3, 4, 5, 1, 1, (2,)), (1, 1, 1, 1, 1, (0, 1, 2)), (1, 1, 6000, 1, 1, (0, 2))])
def test_attention(fn, by, B, Lq, Lk, Hq, Hkv, dims):
    import torch
    q, k, v = (torch.randn(s, device="cuda:0").half() for s in ((B, Lq, Hq, 64), (B, Lk, Hkv, 64), (B, Lk, Hkv, 64)))
    size = hb.hb_attention_workspace_size(B, Lq, Lk, Hq, Hkv, 64)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda:0") if size else None
    want = getattr(hb, fn)(q, k, v, torch.empty_like(q), 0.125, ws)
    out = torch.empty_like(q)
    other = [odd(t, [d for d in dims if t.shape[d] == 1], by) for t in (q, k, v, out)]
    print(fn, B, Lq, Lk, Hq, Hkv, by, flush=True)
    getattr(hb, fn)(*other, 0.125, ws)
    assert torch.equal(out, want)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("shape,dims", [((1, 6, 4, 64), (0,)), ((3, 1, 4, 64), (1,)), ((3, 5, 1, 64), (2,)), ((1, 1, 1, 64), (0, 1, 2))])
def test_rope(interleaved, shape, dims):
    import torch
    x = torch.randn(shape, device="cuda:0").half()
    pos = torch.randint(0, 100, shape[:2] + (1,), dtype=torch.int32, device="cuda:0")
    freq = torch.rand(32, device="cuda:0")
    want = hb.hb_rope_axes(x, torch.empty_like(x), pos, freq, [32], interleaved)
    out = torch.empty_like(x)
    print("hb_rope_axes", shape, interleaved, flush=True)
    hb.hb_rope_axes(odd(x, dims, 3), odd(out, dims, 5), pos, freq, [32], interleaved)
    assert torch.equal(out, want)


def test_rope_keeps_its_wide_accesses():
    """A million tokens of one image and one head, the strides of both odd: 2-byte accesses take twice as long (65 and 150 us)."""
    import torch
    x = torch.randn((1, 1000000, 1, 64), device="cuda:0").half()
    pos = torch.zeros((1, 1000000, 1), dtype=torch.int32, device="cuda:0")
    freq, out = torch.rand(32, device="cuda:0"), torch.empty_like(x)

    def least(a, b):
        times = []
        for _ in range(6):
            start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            start.record()
            for _ in range(5):
                hb.hb_rope_axes(a, b, pos, freq, [32])
            end.record()
            end.synchronize()
            times.append(start.elapsed_time(end))
        return min(times)
    usual, other = least(x, out), least(odd(x, (0, 2), 3), odd(out, (0, 2), 3))
    print("five calls", usual, "ms; odd strides", other, "ms", flush=True)
    assert other < 1.5 * usual


@pytest.mark.parametrize("fn", ["hb_linear", "hb_linear_valu"])
def test_linear_of_one_column(fn):
    """K = 1 and N = 1: the stride from column to column has no meaning."""
    import torch
    x, w = torch.randn((1, 200), device="cuda:0").half(), torch.randn((1, 70), device="cuda:0").half()
    want = x.t().float() @ w.float()
    out = getattr(hb, fn)(x.t(), w.t(), torch.empty((200, 70), dtype=torch.float32, device="cuda:0"))
    assert torch.equal(out, want)                         # one product each
    column, beside = (torch.full((1, 200), 7.0, device="cuda:0").t() for _ in range(2))
    getattr(hb, fn)(x.t(), w[:, :1], column, residual=beside)
    assert torch.equal(column, want[:, :1] + 7.0)
