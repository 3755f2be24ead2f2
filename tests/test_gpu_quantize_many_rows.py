"""hb_quantize_rows with more rows than a launch has lanes for at a workgroup of 1024 each."""
import pytest

from paper_2512_02371_amd import hb

pytestmark = pytest.mark.gpu


def test_rows_of_more_than_a_workgroup_holds():
    """2^22 + 3 rows of 16392 values, 206 GB in all: zeros but for a few rows."""
    import torch
    M, K = (1 << 22) + 3, 16392
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 3 * M * K + (8 << 30):
        pytest.skip("not enough free memory")
    gen = torch.Generator("cuda").manual_seed(1)
    rows = torch.tensor([0, 1, (1 << 18) - 1, 1 << 18, (1 << 21) + 5, (1 << 22) - 1, 1 << 22, M - 1], device="cuda")           # values 2^32 and 2^33 and the last launch's end among them
    values = torch.randn((len(rows), K), generator=gen, device="cuda").half()
    values[:, -1] = 9.0                                               # the largest, where no lane holds it
    x, q, scale = torch.zeros((M, K), dtype=torch.float16, device="cuda"), torch.full((M, K), 99, dtype=torch.int8, device="cuda"), torch.full((M,), 7.0, device="cuda")
    x[rows] = values
    print(M, K, flush=True)
    hb.hb_quantize_rows(x, q, scale)
    torch.cuda.synchronize()
    want = torch.zeros(M, device="cuda")
    want[rows] = (values.double().abs().amax(dim=1) / 127.0).float()
    assert torch.equal(scale, want)
    assert torch.equal(q[rows], torch.round(127.0 * values.double() / 9.0).to(torch.int8))
    q[rows] = 0
    for m in range(0, M, 1 << 16):
        assert not q[m:m + (1 << 16)].any(), m
    del x, q
    torch.cuda.empty_cache()
