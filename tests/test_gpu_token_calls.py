"""The token operators' native marshalling: what it takes gives what ctypes gives, what it does not take is left to ctypes; and a graph."""
import pytest

from paper_2512_02371_amd import hb

pytestmark = pytest.mark.gpu


def usual(torch):
    """Entry point -> (arguments of a usual call, which is its output)."""
    gen = torch.Generator(device="cuda:0").manual_seed(1)
    f16 = lambda *s: torch.randn(s, generator=gen, device="cuda:0").half()
    size = hb.hb_linear_workspace_size(40, 72, 4096)
    ws = torch.empty(max(size, 1), dtype=torch.uint8, device="cuda:0")
    q, k = f16(2, 5, 4, 64), f16(2, 3000, 2, 64)
    aws = torch.empty(max(1, hb.hb_attention_workspace_size(2, 5, 3000, 4, 2, 64)), dtype=torch.uint8, device="cuda:0")
    x = f16(2, 6, 3, 32)
    return {
        "linear": ([f16(40, 4096), f16(72, 4096), torch.zeros((40, 72), dtype=torch.float16, device="cuda:0"), ws, f16(72), f16(40, 72), "gelu"], 2),
        "rope_axes": ([x, torch.zeros_like(x), torch.randint(0, 50, (2, 6, 2), dtype=torch.int32, generator=gen, device="cuda:0"), torch.rand(12, generator=gen, device="cuda:0"),
                       [5, 7], True], 1),
        "attention": ([q, k, f16(2, 3000, 2, 64), torch.zeros_like(q), 0.125, aws, torch.tensor([2000, 3000], dtype=torch.int32, device="cuda:0"),
                       (torch.rand((2, 3000), generator=gen, device="cuda:0") < 0.7).to(torch.uint8)], 3),
    }


@pytest.mark.parametrize("name", ["linear", "rope_axes", "attention"])
def test_taken_calls_equal_ctypes(name, monkeypatch):
    import torch
    hb.load()
    args, o = usual(torch)[name]
    call, entry = getattr(hb._calls, name), getattr(hb, "hb_" + name)
    print(name, flush=True)
    torch.cuda.synchronize()
    first, busy = args[0].clone(), torch.zeros((2, 8192, 8192), dtype=torch.float16, device="cuda:0")
    args[0].zero_()
    stream = torch.cuda.Stream()                          # what the call reads is written behind products of milliseconds on its stream
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        for _ in range(3):
            torch.mm(busy[0], busy[0], out=busy[1])
        args[0].copy_(first)
        assert call(*args) is True
    stream.synchronize()
    got = args[o].clone()
    assert got.any()
    args[o].zero_()
    with monkeypatch.context() as m:
        m.setattr(hb, "_calls", None)
        assert entry(*args) is args[o]
    assert torch.equal(got, args[o])

    class Sub(torch.Tensor):
        pass
    args[o].zero_()
    for i in (0, 1, o):
        other = list(args)
        other[i] = args[i].as_subclass(Sub)
        assert call(*other) is False
        other[i] = args[i].cpu()
        assert call(*other) is False
        with pytest.raises(AssertionError):
            entry(*other)
        other[i] = args[i][:-1]                           # another shape
        assert call(*other) is False
        with pytest.raises(AssertionError):
            entry(*other)
    assert call(*args[:-1]) is False
    torch.cuda.synchronize()
    assert not args[o].any(), "a call that was not taken wrote"
    for i, v in {"linear": {6: "swish"}, "rope_axes": {4: [5, 8]}, "attention": {4: "a"}}[name].items():
        other = list(args)
        other[i] = v
        assert call(*other) is False


def test_optional_arguments_and_one_row():
    import torch
    f16 = lambda *s: torch.randn(s, device="cuda:0").half()
    wide = f16(1, 900)
    x, w, out = wide.as_strided((1, 64), (3, 1)), f16(48, 64), torch.empty((1, 48), dtype=torch.float32, device="cuda:0")
    assert hb._calls.linear(x, w, out, None, None, None, "none") is True             # any pitch: there is one row
    assert torch.allclose(out, x.float() @ w.float().t(), atol=1e-3)
    q, k = f16(1, 2, 2, 64), f16(1, 9, 1, 64)
    assert hb._calls.attention(q, k, k, torch.empty_like(q), 0.1, None, None, None) is True
    mask = torch.zeros((1, 9), dtype=torch.bool, device="cuda:0")
    mask[0, 4] = True
    out = hb.hb_attention(q, k, k, torch.empty_like(q), 0.1, None, None, mask)
    assert torch.equal(out, k[:, 4:5].expand_as(out))
    for bad in (dict(out=torch.empty_like(q)[:, :1]),):
        with pytest.raises(AssertionError):
            hb.hb_attention(q, k, k, scale=0.1, **bad)
    with pytest.raises(hb.HbError) as e:                  # the library's own errors, by either way
        hb.hb_attention(q, k, k, torch.empty_like(q), float("nan"))
    assert e.value.code == hb.HB_ERR_INVALID_ARG and str(e.value).startswith("hb_attention failed: ")


def test_replays_from_a_graph():
    """All three, captured, replayed on other inputs with eager work in between: bit for bit the eager results."""
    import torch
    gen = torch.Generator(device="cuda:0").manual_seed(2)
    new = lambda *s: torch.randn(s, generator=gen, device="cuda:0").half()
    pos = torch.stack(torch.meshgrid(torch.arange(10), torch.arange(10), indexing="ij"), -1).reshape(1, 100, 2).int().cuda().contiguous()
    freq = torch.rand(32, generator=gen, device="cuda:0")
    w, kv = new(256, 2048), new(2, 2500, 2, 4, 64)
    lws = torch.empty(max(1, hb.hb_linear_workspace_size(100, 256, 2048)), dtype=torch.uint8, device="cuda:0")
    aws = torch.empty(max(1, hb.hb_attention_workspace_size(1, 100, 2500, 4, 4, 64)), dtype=torch.uint8, device="cuda:0")

    def step(x, q, out):
        hb.hb_linear(x, w, q.view(100, 256), lws, None, None, "none")
        hb.hb_rope_axes(q, q, pos, freq, (16, 16))
        hb.hb_attention(q, kv[:1, :, 0], kv[:1, :, 1], out, 0.125, aws)

    inputs, want = [new(100, 2048) for _ in range(2)], []
    for x in inputs:
        q, out = torch.empty((1, 100, 4, 64), dtype=torch.float16, device="cuda:0"), torch.empty((1, 100, 4, 64), dtype=torch.float16, device="cuda:0")
        step(x, q, out)
        want.append(out.clone())
    static = inputs[0].clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(static, q, out)
    for rep in range(4):
        static.copy_(inputs[rep & 1])
        out.fill_(-1.0)
        torch.cuda.synchronize()
        print("replay", rep, flush=True)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[rep & 1])
