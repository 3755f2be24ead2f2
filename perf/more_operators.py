"""The operators around a feature map's blocks whose speed is tracked: hb_group_norm, hb_quantize_rows and hb_linear_i8.

``own`` chooses between the plain forms (elementary torch operations in fp32, rounded once at the end) and the library's entry
points.  ``listed()`` holds calls from one token to whole feature maps, ``draw()`` gives more of the same ranges, and ``exact()``
evaluates the definitions in fp64.  Activations are normal, with a mean and a deviation of each channel before a norm; 8-bit operands are
rows of normal values divided by their largest.
"""
from __future__ import annotations

import math

import torch

own = False

_ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]


def listed():
    return [
        # the coarsest feature map of one image, 8 x 8 pixels: latency counts
        {"name": "norm_1x64x512_g32_silu", "op": "norm", "N": 1, "P": 64, "C": 512, "groups": 32, "act": "silu", "affine": True, "f32_in": False, "f32_out": False, "pad": 0},
        # the tokens of eight 64 x 64 feature maps, before a projection
        {"name": "norm_8x4096x1024_g32", "op": "norm", "N": 8, "P": 4096, "C": 1024, "groups": 32, "act": "none", "affine": True, "f32_in": False, "f32_out": False, "pad": 0},
        # the convolution layer's 1024 x 1024 feature map of 64 channels, before the next layer: memory, no group fits a compute unit
        {"name": "norm_1x1048576x64_g32_silu", "op": "norm", "N": 1, "P": 1 << 20, "C": 64, "groups": 32, "act": "silu", "affine": True, "f32_in": False, "f32_out": False, "pad": 0},
        # an fp32 residual stream of odd sizes, a window of wider rows
        {"name": "norm_3x1079x180_g12_f32", "op": "norm", "N": 3, "P": 1079, "C": 180, "groups": 12, "act": "gelu", "affine": True, "f32_in": True, "f32_out": False, "pad": 24},
        # one token's activations, before a projection: latency counts
        {"name": "quantize_1x4096", "op": "quantize", "M": 1, "K": 4096, "pad": 0},
        # the tokens of eight 64 x 64 feature maps
        {"name": "quantize_32768x1024", "op": "quantize", "M": 32768, "K": 1024, "pad": 0},
        # odd sides, a window of wider rows
        {"name": "quantize_1917x1079_pad", "op": "quantize", "M": 1917, "K": 1079, "pad": 24},
        # one token through the first matrix of an MLP: the weights are read once, latency counts
        {"name": "linear_1x4096x1024_gelu", "op": "linear", "M": 1, "N": 4096, "K": 1024, "act": "gelu", "bias": True, "residual": False, "f32": False, "pad": 0},
        # keys and values of eight captions of 77 states
        {"name": "linear_616x2048x1024", "op": "linear", "M": 616, "N": 2048, "K": 1024, "act": "none", "bias": True, "residual": False, "f32": False, "pad": 0},
        # the first matrix of an MLP over the tokens of two 64 x 64 feature maps
        {"name": "linear_8192x8192x2048_gelu", "op": "linear", "M": 8192, "N": 8192, "K": 2048, "act": "gelu_tanh", "bias": True, "residual": False, "f32": False, "pad": 0},
        # the tokens of eight 64 x 64 feature maps through a projection, with the skip connection
        {"name": "linear_32768x1024x1024", "op": "linear", "M": 32768, "N": 1024, "K": 1024, "act": "none", "bias": True, "residual": True, "f32": False, "pad": 0},
        # odd sides (rows at any address), added to an fp32 residual stream
        {"name": "linear_1917x1079x1023_f32", "op": "linear", "M": 1917, "N": 1079, "K": 1023, "act": "silu", "bias": True, "residual": True, "f32": True, "pad": 0},
    ]


def _log_int(rng, lo, hi):
    """An integer from lo to hi, spread over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _size(rng, lo, hi):
    """As _log_int; half of them multiples of 16."""
    n = _log_int(rng, lo, hi)
    return n if n < 16 or rng.random() < 0.5 else n // 16 * 16


def draw(rng):
    op = rng.choice(["norm", "norm", "quantize", "linear", "linear"])
    if op == "norm":
        groups = rng.choice([1, 2, 4, 8, 16, 32, 32, 32, 3, 6, 12, 24])
        C = groups * _log_int(rng, 1, 64)
        P = _size(rng, 1, 1 << 20)
        P = max(1, min(P, (1 << 26) // C))
        N = max(1, min(_log_int(rng, 1, 64), (1 << 26) // (P * C)))
        return {"op": op, "N": N, "P": P, "C": C, "groups": groups, "act": rng.choice(_ACTS), "affine": rng.random() < 0.8,
                "f32_in": rng.random() < 0.25, "f32_out": rng.random() < 0.2, "pad": rng.choice([0, 0, 0, 24])}        # pad: x is a window of wider pixels
    if op == "quantize":
        M, K = _size(rng, 1, 1 << 17), _size(rng, 16, 16384)
        return {"op": op, "M": max(1, min(M, (1 << 25) // K)), "K": K, "pad": rng.choice([0, 0, 0, 24])}
    if rng.random() < 0.25:                                    # the pixels of a feature map
        M, N, K = _size(rng, 4096, 1 << 20), _size(rng, 16, 256), _size(rng, 16, 256)
        M = min(M, (1 << 25) // max(N, K))
    else:
        M, N, K = _size(rng, 1, 16384), _size(rng, 16, 8192), _size(rng, 16, 8192)
        M = max(1, min(M, (8192 * 8192 * 2048) // (N * K), (1 << 25) // max(N, K)))
    return {"op": op, "M": M, "N": N, "K": K, "act": rng.choice(_ACTS), "bias": rng.random() < 0.7, "residual": rng.random() < 0.5,
            "f32": rng.random() < 0.3, "pad": rng.choice([0, 0, 0, 16])}               # pad: x is a window of wider rows


# ---- what a program holds before the call ---------------------------------------------------------------

def _bytes_and_scales(x):
    """Rows of 8-bit integers and what each stands for, of rows of values."""
    top = x.abs().amax(dim=1)
    return torch.round(x * (127.0 / top)[:, None]).to(torch.int8), top / 127.0


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, std=1.0):
        return torch.randn(shape, generator=gen, device="cuda").mul_(std)

    s = {"op": case["op"]}
    if case["op"] == "norm":
        N, P, C = case["N"], case["P"], case["C"]
        wide = C + case["pad"]
        x = normal(N, P, wide).mul_(torch.rand(wide, generator=gen, device="cuda") + 0.5).add_(normal(wide))
        s.update(x=(x if case["f32_in"] else x.half())[:, :, :C], groups=case["groups"], act=case["act"], eps=1e-5,
                 weight=normal(C, std=0.2).add_(1.0).half() if case["affine"] else None, bias=normal(C, std=0.2).half() if case["affine"] else None,
                 out=torch.empty((N, P, C), dtype=torch.float32 if case["f32_out"] else torch.float16, device="cuda"))
    elif case["op"] == "quantize":
        M, K = case["M"], case["K"]
        s.update(x=normal(M, K + case["pad"]).half()[:, :K], q=torch.empty((M, K), dtype=torch.int8, device="cuda"),
                 scale=torch.empty(M, dtype=torch.float32, device="cuda"))
    else:
        M, N, K = case["M"], case["N"], case["K"]
        kind = torch.float32 if case["f32"] else torch.float16
        x, x_scale = _bytes_and_scales(normal(M, K + case["pad"]))
        w, w_scale = _bytes_and_scales(normal(N, K, std=K ** -0.5))
        s.update(x=x[:, :K], x_scale=x_scale, w=w, w_scale=w_scale, act=case["act"], bias=normal(N, std=0.5).half() if case["bias"] else None,
                 residual=normal(M, N).to(kind) if case["residual"] else None, out=torch.empty((M, N), dtype=kind, device="cuda"))
    return s


# ---- the plain forms ------------------------------------------------------------------------------------

def _act(v, act):
    if act == "relu":
        return torch.clamp(v, min=0.0)
    if act == "gelu":
        return 0.5 * v * (1.0 + torch.erf(v * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * v * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (v + 0.044715 * v * v * v)))
    if act == "silu":
        return v / (1.0 + torch.exp(-v))
    return v


def _plain_norm(s):
    N, P, C = s["x"].shape
    x = s["x"].float().reshape(N, P, s["groups"], C // s["groups"])
    d = x - x.mean(dim=(1, 3), keepdim=True)
    y = (d / torch.sqrt((d * d).mean(dim=(1, 3), keepdim=True) + s["eps"])).reshape(N, P, C)
    if s["weight"] is not None:
        y = y * s["weight"].float() + s["bias"].float()
    return _act(y, s["act"]).to(s["out"].dtype)


def _plain_quantize(s):
    x = s["x"].float()
    top = x.abs().amax(dim=1, keepdim=True)
    q = torch.where(top > 0.0, torch.round(x * 127.0 / top), torch.zeros_like(x))
    return {"q": q.to(torch.int8), "scale": (top / 127.0)[:, 0]}


def _plain_linear(s):
    v = (s["x"].float() @ s["w"].float().T) * s["x_scale"][:, None] * s["w_scale"]
    if s["bias"] is not None:
        v = v + s["bias"].float()
    v = _act(v, s["act"])
    if s["residual"] is not None:
        v = v + s["residual"].float()
    return v.to(s["out"].dtype)


# ---- one pass -------------------------------------------------------------------------------------------

def _workspace(s, size):
    """The scratch memory that a program keeps beside its weights: allocated at the first pass."""
    s["workspace"] = torch.empty(size, dtype=torch.uint8, device="cuda") if size else None


def _own_norm(s):
    from paper_2512_02371_amd import hb
    if "workspace" not in s:
        _workspace(s, hb.hb_group_norm_workspace_size(*s["x"].shape, s["groups"]))
    return hb.hb_group_norm(s["x"], s["out"], s["groups"], s["weight"], s["bias"], s["eps"], s["act"], s["workspace"])


def _own_quantize(s):
    from paper_2512_02371_amd import hb
    hb.hb_quantize_rows(s["x"], s["q"], s["scale"])
    return {"q": s["q"], "scale": s["scale"]}


def _own_linear(s):
    from paper_2512_02371_amd import hb
    if "workspace" not in s:
        _workspace(s, hb.hb_linear_i8_workspace_size(s["x"].shape[0], s["w"].shape[0], s["w"].shape[1]))
    return hb.hb_linear_i8(s["x"], s["w"], s["x_scale"], s["w_scale"], s["out"], s["workspace"], s["bias"], s["residual"], s["act"])


def run(state):
    if own:
        return {"norm": _own_norm, "quantize": _own_quantize, "linear": _own_linear}[state["op"]](state)
    return {"norm": _plain_norm, "quantize": _plain_quantize, "linear": _plain_linear}[state["op"]](state)


# ---- the definitions in fp64 ----------------------------------------------------------------------------

def _exact_act(y, act):
    if act == "relu":
        return torch.maximum(y, torch.zeros_like(y))
    if act == "gelu":
        return y * torch.erfc(-y / math.sqrt(2.0)) / 2.0
    if act == "gelu_tanh":                                     # (1 + tanh z) / 2 is the sigmoid of 2 z
        return y * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (y + 0.044715 * y ** 3))
    if act == "silu":
        return y * torch.sigmoid(y)
    return y


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        N, P, C = s["x"].shape
        out, size = torch.empty((N, P, C), dtype=torch.float64, device="cuda"), C // case["groups"]
        for n in range(N):
            for g in range(case["groups"]):
                these = slice(g * size, (g + 1) * size)
                x = s["x"][n, :, these].double()
                var, mean = torch.var_mean(x, correction=0)
                y = (x - mean) * torch.rsqrt(var + s["eps"])
                if s["weight"] is not None:
                    y = torch.addcmul(s["bias"][these].double(), y, s["weight"][these].double())
                out[n, :, these] = _exact_act(y, case["act"])
        return out
    if case["op"] == "quantize":
        q, scale = torch.empty((case["M"], case["K"]), dtype=torch.int8, device="cuda"), torch.empty(case["M"], dtype=torch.float64, device="cuda")
        for m in range(0, case["M"], 4096):
            x = s["x"][m:m + 4096].double()
            scale[m:m + 4096] = torch.linalg.vector_norm(x, ord=math.inf, dim=1)
            q[m:m + 4096] = torch.round(127.0 * x / torch.clamp(scale[m:m + 4096, None], min=2.0 ** -60)).to(torch.int8)
        return {"q": q, "scale": scale / 127.0}
    w, out = s["w"].double().t().contiguous(), torch.empty((case["M"], case["N"]), dtype=torch.float64, device="cuda")
    for m in range(0, case["M"], 65536):
        y = torch.mm(s["x"][m:m + 65536].double(), w) * torch.outer(s["x_scale"][m:m + 65536].double(), s["w_scale"].double())
        if s["bias"] is not None:
            y += s["bias"].double()
        y = _exact_act(y, case["act"])
        if s["residual"] is not None:
            y += s["residual"][m:m + 65536].double()
        out[m:m + 65536] = y
    return out


# ---- what a pass cannot do without ----------------------------------------------------------------------

def work(case):
    """Input bytes once, output bytes once; the multiply-adds of each definition, two operations each."""
    if case["op"] == "norm":
        n, C = case["N"] * case["P"] * case["C"], case["C"]
        return {"bytes": n * ((4 if case["f32_in"] else 2) + (4 if case["f32_out"] else 2)) + (4 * C if case["affine"] else 0), "flops": 7 * n}
    if case["op"] == "quantize":
        return {"bytes": case["M"] * (3 * case["K"] + 4), "flops": 3 * case["M"] * case["K"]}
    M, N, K, size = case["M"], case["N"], case["K"], 4 if case["f32"] else 2
    return {"bytes": M * K + N * K + 4 * (M + N) + (2 * N if case["bias"] else 0) + size * M * N * (2 if case["residual"] else 1), "flops": 2 * M * N * K}
