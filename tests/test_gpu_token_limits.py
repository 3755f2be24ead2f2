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
