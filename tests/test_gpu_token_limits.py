"""The token operators at the largest sizes that they take."""
import pytest

from paper_2512_02371_amd import hb

pytestmark = pytest.mark.gpu


def test_as_many_keys_as_a_call_takes():
    """2^31 - 256 times the same key (a token stride of 0), masked in between: the mean is that key's value, exactly (powers of two)."""
    import torch
    Lk = (1 << 31) - 256
    q = torch.ones((1, 1, 1, 8), dtype=torch.float16, device="cuda:0")
    k = torch.full((1, 1, 1, 8), 0.5, dtype=torch.float16, device="cuda:0").expand(1, Lk, 1, 8)
    v = torch.tensor([0.5, 1.0, -2.0, 0.25, -0.125, 4.0, 8.0, 0.0], dtype=torch.float16, device="cuda:0").reshape(1, 1, 1, 8)
    ws = torch.empty(hb.hb_attention_workspace_size(1, 1, Lk, 1, 1, 8), dtype=torch.uint8, device="cuda:0")
    mask = torch.ones((1, Lk), dtype=torch.uint8, device="cuda:0")
    mask[0, 1:: 1 << 20] = 0
    for m in (None, mask):
        print("hb_attention", Lk, m is not None, flush=True)
        out = hb.hb_attention(q, k, v.expand(1, Lk, 1, 8), torch.empty_like(q), 1.0, ws, None, m)
        torch.cuda.synchronize()
        if m is None:
            assert torch.equal(out, v)
        else:                                             # 2048 of 2^31 keys are missing in the sums and in the weights alike
            assert (out - v).abs().max() <= 2.0 ** -10 * 8.0


def test_just_under_2_to_the_32_threads():
    """2^24 - 8 workgroups of 256 threads, one for each key head: one key each, so that every query's result is its value."""
    import torch
    B, H, D = (1 << 21) - 1, 8, 8
    q = torch.ones((1, 1, H, D), dtype=torch.float16, device="cuda:0").expand(B, 1, H, D)
    v = torch.randn((B, 1, H, D), device="cuda:0").half()
    out = torch.full_like(v, 7.0)
    print("hb_attention", B, flush=True)
    hb.hb_attention(q, v, v, out, 1.0)
    torch.cuda.synchronize()
    assert torch.equal(out, v)


def test_rope_just_under_2_to_the_32_threads():
    """2^32 - 2^16 pairs at odd strides: each by itself, all of them a half turn."""
    import torch
    B, L = (1 << 16) - 1, 1 << 16
    token = 3                                             # elements from token to token: two of them turn, the third is between
    x = torch.zeros((B * L * token,), dtype=torch.float16, device="cuda:0")
    x[0::token], x[1::token], x[2::token] = 1.0, -2.0, 7.0
    view = x.as_strided((B, L, 1, 2), (L * token, token, 2, 1))
    pos = torch.ones((1, 1, 1), dtype=torch.int32, device="cuda:0").expand(B, L, 1)
    print("hb_rope_axes", B, L, flush=True)
    hb.hb_rope_axes(view, view, pos, torch.full((1,), 3.14159265, device="cuda:0"), [1])
    torch.cuda.synchronize()
    for i, want in enumerate((-1.0, 2.0, 7.0)):
        assert bool((x[i::token] == want).all()), i


def test_sizes_beyond_an_int_are_not_cut_off():
    """2^32 + 5 keys, broadcast: not a call of five keys.  2^32 + 3 rows: not a call of three."""
    import torch
    q = torch.ones((1, 2, 1, 8), dtype=torch.float16, device="cuda:0")
    k = q[:, :1].expand(1, (1 << 32) + 5, 1, 8)
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda:0")
    for fn in (hb.hb_attention, hb.hb_attention_valu):
        with pytest.raises(AssertionError):
            fn(q, k, k, torch.empty_like(q), 1.0, ws)
    x = torch.zeros(((1 << 32) + 3, 1), dtype=torch.float16, device="cuda:0")
    for fn in (hb.hb_linear, hb.hb_linear_valu):
        with pytest.raises(AssertionError):
            fn(x, x[:1], x, ws)
    pos, turns = torch.zeros((1, 1, 1), dtype=torch.int32, device="cuda:0"), x.view(-1)[: (1 << 32) + 2].view(1, (1 << 31) + 1, 1, 2)
    with pytest.raises(AssertionError):
        hb.hb_rope_axes(turns, turns, pos.expand(1, (1 << 31) + 1, 1), torch.ones(1, device="cuda:0"), [1])
