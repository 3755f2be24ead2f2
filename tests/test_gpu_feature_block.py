"""The operators around a feature map together: the example against the oracle step by step, a graph of them replayed, two calls at once, and their native marshalling."""
import os
import sys

import numpy as np
import pytest

import oracle
from paper_2512_02371_amd import hb

pytestmark = pytest.mark.gpu


def example(*args, **kw):
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    from feature_mlp_i8 import FeatureMlpI8
    return FeatureMlpI8(*args, **kw)


@pytest.mark.parametrize("images,size,width,hidden,groups", [(2, 12, 96, 200, 32), (1, 33, 128, 256, 8)])
def test_block_against_the_oracle(images, size, width, hidden, groups):
    import torch
    run = example(images, size, width, hidden, groups, seed=3)
    pixels = torch.rand((images, size, size, 64), device="cuda").mul_(2).sub_(1).half()
    got = run(pixels).double().cpu().numpy().reshape(-1, width)
    assert np.array_equal(got, run(pixels).double().cpu().numpy().reshape(-1, width))
    f64, f16 = (lambda t: t.double().cpu().numpy()), (lambda t: t.cpu().numpy())
    near = lambda t, want: np.abs(f64(t).reshape(want.shape) - want).max() <= 2.0 ** -10 * np.abs(want).max()          # a rounding is 2^-11
    # the whole: each step on what the step before left, the first two together (in place): the convolution's rounding, times the norm's 1 / deviation
    conv = oracle.conv3x3(f16(pixels).view(np.uint16), f16(run.conv).view(np.uint16)).reshape(images, size * size, 64)
    want = oracle.group_norm(conv, groups, f64(run.norms["features"][0]), f64(run.norms["features"][1]), 1e-5, "silu")
    spread = conv.reshape(images, -1, groups, 64 // groups).std(axis=(1, 3)).min()
    assert np.abs(f64(run.features).reshape(want.shape) - want).max() <= 2.0 ** -10 * np.abs(want).max() + 4 * 2.0 ** -11 * np.abs(conv).max() / spread
    assert near(run.x, oracle.linear(f64(run.features).reshape(-1, 64), f64(run.w["in"]), f64(run.b["in"])))
    want = oracle.group_norm(f64(run.x).reshape(images, -1, width), groups, f64(run.norms["tokens"][0]), f64(run.norms["tokens"][1]))
    assert near(run.normed, want)
    q, scale = oracle.quantize_rows(f16(run.normed))
    assert np.array_equal(f16(run.x8), q) and np.array_equal(f16(run.x_scale), scale.astype(np.float32))
    w = {n: (f16(a), f16(s)) for n, (a, s) in run.w8.items()}
    for n in w:
        q_w, s_w = oracle.quantize_rows(f16(run.w[n]))
        assert np.array_equal(w[n][0], q_w) and np.array_equal(w[n][1], s_w.astype(np.float32))
    assert near(run.hidden, oracle.linear_i8(q, w["up"][0], f16(run.x_scale), w["up"][1], f64(run.b["up"]), None, "gelu"))
    q, scale = oracle.quantize_rows(f16(run.hidden))
    assert np.array_equal(f16(run.h8), q)
    want = oracle.linear_i8(q, w["down"][0], f16(run.h_scale), w["down"][1], f64(run.b["down"]), f64(run.x))
    assert np.abs(got - want).max() <= 2.0 ** -10 * np.abs(want).max()
    # beside fp16 products: each product has operands of 127 steps to a row's largest value, four deviations of it, so each is off by 4 / 127 / sqrt(12) = 0.9 % of a deviation,
    # the two operands of the two products together by twice that
    apart = got - f64(run.mlp_in_fp16()).reshape(-1, width)
    assert np.sqrt((apart ** 2).mean()) <= 0.03 * np.sqrt((got ** 2).mean())


def test_replays_from_a_graph():
    """The statistics of streaming rows, a slab, rows as integers, a split sum of integers and a whole one: bit for bit the eager results, with eager work between."""
    import torch
    gen = torch.Generator(device="cuda:0").manual_seed(2)
    new = lambda *s: torch.randn(s, generator=gen, device="cuda:0").half()
    empty = lambda *s, t=torch.float16: torch.empty(s, dtype=t, device="cuda:0")
    P, C = 40000, 64
    w8, w_scale = hb.hb_quantize_rows(new(48, 64 * 64), empty(48, 64 * 64, t=torch.int8), empty(48, t=torch.float32))
    ws = [torch.empty(max(1, n), dtype=torch.uint8, device="cuda:0") for n in (hb.hb_group_norm_workspace_size(1, P, C, 8), hb.hb_linear_i8_workspace_size(20, 48, 64 * 64))]
    assert ws[0].numel() > 1 and ws[1].numel() > 1
    normed, small, q, scale, out = empty(1, P, C), empty(20, 64, 64), empty(20, 64 * 64, t=torch.int8), empty(20, t=torch.float32), empty(20, 48)

    def step(x):
        hb.hb_group_norm(x, normed, 8, act="silu", workspace=ws[0])
        hb.hb_group_norm(normed[0, :20 * 64].view(20, 64, 64), small, 8, act="none", workspace=None)
        hb.hb_quantize_rows(small.view(20, 64 * 64), q, scale)
        hb.hb_linear_i8(q, w8, scale, w_scale, out, ws[1], None, None, "gelu")

    inputs, want = [new(1, P, C) for _ in range(2)], []
    for x in inputs:
        step(x)
        want.append((normed.clone(), q.clone(), scale.clone(), out.clone()))
    static = inputs[0].clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(static)
    for rep in range(5):
        static.copy_(inputs[rep & 1])
        for t in (normed, out, scale):
            t.fill_(-1.0)
        q.fill_(5)
        for w in ws:
            w.fill_(0xff)                                             # nothing is kept there between calls
        torch.mm(new(512, 512), new(512, 512))
        torch.cuda.synchronize()
        print("replay", rep, flush=True)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((normed, q, scale, out), want[rep & 1]))


def test_calls_on_two_streams_at_once():
    import torch
    gen = torch.Generator(device="cuda:0").manual_seed(4)
    x = [torch.randn((1, 60000, 64), generator=gen, device="cuda:0").half() for _ in range(2)]
    size = hb.hb_group_norm_workspace_size(1, 60000, 64, 32)
    ws = [torch.empty(size, dtype=torch.uint8, device="cuda:0") for _ in range(2)]
    alone = [hb.hb_group_norm(t, torch.empty_like(t), 32, act="gelu", workspace=ws[0]).clone() for t in x]
    outs, streams = [torch.empty_like(t) for t in x], [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                hb.hb_group_norm(x[i], outs[i], 32, act="gelu", workspace=ws[i])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(alone, outs))


def usual(torch):
    """Entry point -> (arguments of a usual call, which of them are its outputs)."""
    gen = torch.Generator(device="cuda:0").manual_seed(1)
    f16 = lambda *s: torch.randn(s, generator=gen, device="cuda:0").half()
    i8 = lambda *s: torch.randint(-127, 128, s, generator=gen, dtype=torch.int8, device="cuda:0")
    f32 = lambda *s: torch.rand(s, generator=gen, device="cuda:0")
    ws = lambda n: torch.empty(max(1, n), dtype=torch.uint8, device="cuda:0")
    zeros = lambda *s, t=torch.float16: torch.zeros(s, dtype=t, device="cuda:0")
    return {
        "group_norm": ([f16(2, 20, 30, 64), zeros(2, 20, 30, 64), 8, f16(64), f16(64), 1e-5, "silu", ws(hb.hb_group_norm_workspace_size(2, 600, 64, 8))], [1]),
        "quantize_rows": ([f16(40, 300), zeros(40, 300, t=torch.int8), zeros(40, t=torch.float32)], [1, 2]),
        "linear_i8": ([i8(40, 4096), i8(72, 4096), f32(40), f32(72), zeros(40, 72), ws(hb.hb_linear_i8_workspace_size(40, 72, 4096)), f16(72), f16(40, 72), "gelu"], [4]),
    }


@pytest.mark.parametrize("name", ["group_norm", "quantize_rows", "linear_i8"])
def test_taken_calls_equal_ctypes(name, monkeypatch):
    import torch
    hb.load()
    args, outs = usual(torch)[name]
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
    got = [args[o].clone() for o in outs]
    assert all(g.any() for g in got)
    for o in outs:
        args[o].zero_()
    with monkeypatch.context() as m:
        m.setattr(hb, "_calls", None)
        entry(*args)
    assert all(torch.equal(g, args[o]) for g, o in zip(got, outs))

    class Sub(torch.Tensor):
        pass
    for o in outs:
        args[o].zero_()
    for i in (0, *outs):
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
    for i, v in {"group_norm": {2: 8.0, 5: 1, 6: "swish"}, "quantize_rows": {2: None}, "linear_i8": {8: "swish", 2: None}}[name].items():
        other = list(args)
        other[i] = v
        assert call(*other) is False
    torch.cuda.synchronize()
    assert not any(args[o].any() for o in outs), "a call that was not taken wrote"


def test_maps_by_either_marshalling(monkeypatch):
    """Three and four dimensions, one row or column of pixels, images of one pixel, nothing optional."""
    import torch
    f16 = lambda *s: torch.randn(s, device="cuda:0").half()
    wide = f16(2, 9, 8, 64)
    for x in (f16(3, 50, 32), f16(2, 5, 10, 32), wide[:, :, 3:4], wide[:, 2:3], wide[:, 2:3, 1:5], f16(5, 1, 32), f16(1, 1, 1, 32), f16(4, 6, 32).transpose(0, 1)):
        outs = []
        for native in (True, False):
            out = torch.empty(x.shape, dtype=torch.float32, device="cuda:0")
            with monkeypatch.context() as m:
                if native:
                    assert hb._calls.group_norm(x, out, 4, None, None, 1e-5, "none", None) is True
                else:
                    m.setattr(hb, "_calls", None)
                    hb.hb_group_norm(x, out, 4)
            outs.append(out)
        assert torch.equal(*outs)
        want = oracle.group_norm(x.double().cpu().numpy().reshape(x.shape[0], -1, x.shape[-1]), 4)
        assert np.abs(outs[0].double().cpu().numpy().reshape(want.shape) - want).max() <= 1e-4
    x = wide[:, :, 1:5]                                   # pixels at two distances
    assert hb._calls.group_norm(x, torch.empty(x.shape, dtype=torch.float16, device="cuda:0"), 4, None, None, 1e-5, "none", None) is False
    for native in (True, False):                          # the library's own errors, by either way
        with monkeypatch.context() as m:
            if not native:
                m.setattr(hb, "_calls", None)
            with pytest.raises(hb.HbError) as e:
                hb.hb_group_norm(f16(2, 3, 32), f16(2, 3, 32), 5)
            assert e.value.code == hb.HB_ERR_INVALID_ARG and str(e.value).startswith("hb_group_norm failed: ")
