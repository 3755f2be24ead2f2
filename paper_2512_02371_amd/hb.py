"""ctypes binding of the C-ABI library declared in ``include/hb.h``.

Argument marshalling only: every function takes torch CUDA tensors (used purely
as device memory), pulls out pointers, shapes and pitches, and calls the entry
point of the same name on torch's current stream.  There is no fallback: if the
library is missing, ``load()`` raises.  The usual calls are marshalled by the
extension module ``_calls``, all others here.
"""
from __future__ import annotations

import ctypes
import logging
import os

import numpy as np
# torch before the library: it ships its own copy of the HIP runtime, and libhb.so must bind to that copy (the
# one that owns torch's streams and allocations), not load a second runtime from the system path
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libhb.so")

HB_OK = 0
HB_ERR_INVALID_ARG = 1
HB_ERR_UNSUPPORTED = 2
HB_ERR_WORKSPACE = 3
HB_ERR_HIP = 4
HB_MAX_TAPS = 64            # per axis, hb_sepblur
HB_MAX_TAPS_FIR1D = 256     # hb_fir1d
HB_MAX_TAPS_CONV2D = 32     # per axis, hb_conv2d
HB_LINEAR_MAX_PITCH = 1 << 21
HB_ATTENTION_MAX_D = 128
HB_ROPE_MAX_AXES = 4
HB_ACTS = {"none": 0, "relu": 1, "gelu": 2, "gelu_tanh": 3, "silu": 4}      # hb_linear

# every symbol include/hb.h declares
SYMBOLS = [
    "hb_status_string",
    "hb_fir1d", "hb_fir1d_valu",
    "hb_conv2d", "hb_conv2d_valu",
    "hb_down2", "hb_down2_valu", "hb_up2", "hb_up2_valu",
    "hb_resize_workspace_size", "hb_resize", "hb_resize_valu", "hb_lanczos3_band", "hb_lanczos3_matrix",
    "hb_iir2_workspace_size", "hb_iir2_abs_gain", "hb_iir2", "hb_iir2_valu",
    "hb_dct_denoise_workspace_size", "hb_dct_denoise", "hb_dct_denoise_valu",
    "hb_sepblur", "hb_sepblur_valu",
    "hb_sat2d_workspace_size", "hb_sat2d", "hb_sat2d_valu", "hb_sat2d_noalloc", "hb_sat2d_set_wait_limit",
    "hb_conv3x3", "hb_conv3x3_valu",
    "hb_pyr_level", "hb_pyr_level_valu",
    "hb_linear_workspace_size", "hb_linear", "hb_linear_valu",
    "hb_rope_axes",
    "hb_attention_workspace_size", "hb_attention", "hb_attention_valu",
    "hb_copy_f16_f32", "hb_mfma_probe",
]

_lib = None
_calls = None               # the native marshalling of the usual calls (csrc/calls.cpp), once the library is loaded


class HbError(RuntimeError):
    def __init__(self, fn: str, code: int):
        self.code = code
        super().__init__(f"{fn} failed: {status_string(code)} ({code})")


def load() -> ctypes.CDLL:
    """Load libhb.so (built by ``__graft_entry__.build()``); raise if it is absent."""
    global _lib, _calls
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(
            f"{LIB_PATH} is missing: build it with `python -c 'import __graft_entry__ as g; g.build()'`. "
            "There is no CPU fallback.")
    L = ctypes.CDLL(LIB_PATH)
    vp, I, I64 = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64
    L.hb_status_string.argtypes = [I]
    L.hb_status_string.restype = ctypes.c_char_p
    fir = [vp, vp, I, I, I64, I64, vp, I, I, vp]
    sep = [vp, vp, I, I, I64, I64, vp, I, I, vp, I, I, vp]
    c2d = [vp, vp, I, I, I64, I64, vp, I, I, I, I, vp]
    sat = [vp, vp, I, I, I64, I64, vp, ctypes.c_size_t, vp]
    conv = [vp, vp, vp, I, I, I, I, I, vp]
    pyr = [vp, vp, vp, I, I, I64, I64, I64, vp]
    for name, sig in (("hb_fir1d", fir), ("hb_fir1d_valu", fir), ("hb_conv2d", c2d), ("hb_conv2d_valu", c2d),
                      ("hb_down2", c2d), ("hb_down2_valu", c2d), ("hb_up2", c2d), ("hb_up2_valu", c2d), ("hb_sepblur", sep), ("hb_sepblur_valu", sep),
                      ("hb_sat2d", sat), ("hb_sat2d_valu", sat), ("hb_conv3x3", conv), ("hb_conv3x3_valu", conv),
                      ("hb_pyr_level", pyr), ("hb_pyr_level_valu", pyr),
                      ("hb_copy_f16_f32", [vp, vp, I64, vp]), ("hb_mfma_probe", [I, vp, vp, vp, vp])):
        f = getattr(L, name)
        f.argtypes = sig
        f.restype = I
    rsz = [vp, vp, vp, ctypes.c_size_t, I, I, I, I, I, I64, I64, I64, I64, vp, vp, I, vp, vp, I, vp]
    for name in ("hb_resize", "hb_resize_valu"):
        getattr(L, name).argtypes = rsz
        getattr(L, name).restype = I
    L.hb_resize_workspace_size.argtypes = [I, I, I]
    L.hb_resize_workspace_size.restype = ctypes.c_size_t
    L.hb_lanczos3_band.argtypes = [I, I]
    L.hb_lanczos3_band.restype = I
    L.hb_lanczos3_matrix.argtypes = [I, I, vp, vp]
    L.hb_lanczos3_matrix.restype = I
    iir = [vp, vp, I, I64, I64, I64, ctypes.c_float, ctypes.c_float, vp, ctypes.c_size_t, vp]
    for name in ("hb_iir2", "hb_iir2_valu"):
        getattr(L, name).argtypes = iir
        getattr(L, name).restype = I
    L.hb_iir2_workspace_size.argtypes = [I, I64]
    L.hb_iir2_workspace_size.restype = ctypes.c_size_t
    L.hb_iir2_abs_gain.argtypes = [ctypes.c_float, ctypes.c_float, I64]
    L.hb_iir2_abs_gain.restype = ctypes.c_double
    dct = [vp, vp, I, I, I, I64, I64, I64, I64, ctypes.c_float, vp, ctypes.c_size_t, vp]
    for name in ("hb_dct_denoise", "hb_dct_denoise_valu"):
        getattr(L, name).argtypes = dct
        getattr(L, name).restype = I
    L.hb_dct_denoise_workspace_size.argtypes = [I, I, I]
    L.hb_dct_denoise_workspace_size.restype = ctypes.c_size_t
    L.hb_sat2d_noalloc.argtypes = [vp, vp, I, I, I64, I64, vp]
    L.hb_sat2d_noalloc.restype = I
    L.hb_sat2d_set_wait_limit.argtypes = [I]
    L.hb_sat2d_set_wait_limit.restype = I
    L.hb_sat2d_workspace_size.argtypes = [I, I]
    L.hb_sat2d_workspace_size.restype = ctypes.c_size_t
    lin = [vp, vp, vp, vp, vp, I, I, I, I, I, I64, I64, I64, I64, vp, ctypes.c_size_t, vp]
    att = [vp, vp, vp, vp, I, I, I, I, I, I] + [I64] * 12 + [ctypes.c_float, vp, vp, I64, vp, ctypes.c_size_t, vp]
    for name, sig in (("hb_linear", lin), ("hb_linear_valu", lin), ("hb_attention", att), ("hb_attention_valu", att),
                      ("hb_rope_axes", [vp, vp, vp, vp, I, I, I, I] + [I64] * 8 + [vp, I, I, vp])):
        f = getattr(L, name)
        f.argtypes = sig
        f.restype = I
    for name, n in (("hb_linear_workspace_size", 3), ("hb_attention_workspace_size", 6)):
        f = getattr(L, name)
        f.argtypes = [I] * n
        f.restype = ctypes.c_size_t
    _lib = L
    # built against one torch: with another, or not built at all, it does not load, and ctypes makes every call
    try:
        from . import _calls as native
        native.bind({name: ctypes.cast(getattr(L, name), vp).value for name in SYMBOLS[1:]}, HbError)
        _calls = native
    except ImportError as e:
        logging.getLogger(__name__).warning("short calls take 1 to 2 us more, the native marshalling did not load: %s", e)
    return L


def status_string(code: int) -> str:
    return load().hb_status_string(int(code)).decode()


hb_status_string = status_string          # the entry point's own name


def _check(fn: str, code: int) -> None:
    if code != HB_OK:
        raise HbError(fn, code)


# Pointers and the stream handle are passed as plain integers, which ctypes converts to the declared argument
# types: with torch.cuda.current_stream() and a pointer object per argument the host took 10.5 us for a call of
# hb_fir1d, 6.5 without.  The two functions behind torch.cuda.current_stream() are private: without them it does.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream() -> int:
    """Handle of torch's current stream on the current device."""
    if _raw_stream is None or _device is None:
        return torch.cuda.current_stream().cuda_stream
    if not torch.cuda.is_initialized():
        torch.cuda.init()
    return _raw_stream(_device())


# On the host a call costs its launch (3.4 us) and what is done here or in _calls; with two array conversions and an address object
# per tap array, and a question to the tensor per stride and dimension, that was 3.6 of 7.0 us.
_U16, _F16 = np.dtype(np.uint16), np.dtype(np.float16)


def _taps(t):
    """Host fp16 bit patterns -> (row-major bytes, which ctypes passes by address and the library copies; count)."""
    if type(t) is not np.ndarray or (t.dtype is not _U16 and t.dtype is not _F16):
        t = np.asarray(t)
        if t.dtype != np.float16:
            t = np.asarray(t, dtype=np.uint16)
    return t.tobytes(), t.size


def _img2d(t, dtype):
    s = t.stride()
    assert t.is_cuda and len(s) == 2 and t.dtype == dtype and s[1] == 1, "row-major 2-D CUDA tensor expected"
    H, W = t.shape
    return t.data_ptr(), H, W, s[0]


def _planes(t, dtype):
    """A 3-D tensor of row-major planes -> (address, planes, height, width, row pitch, plane stride)."""
    s = t.stride()
    assert t.is_cuda and len(s) == 3 and t.dtype == dtype and s[2] == 1
    C, H, W = t.shape
    return t.data_ptr(), C, H, W, s[1], s[0]


def _fir(name, inp, out, taps, anchor):
    pi, H, W, ip = _img2d(inp, torch.float16)
    po, Ho, Wo, op = _img2d(out, torch.float32)
    assert (H, W) == (Ho, Wo)
    bits, n = _taps(taps)
    _check(name, getattr(_lib or load(), name)(pi, po, H, W, ip, op, bits, n, int(anchor), _stream()))
    return out


def hb_fir1d(inp, out, taps, anchor):
    if _calls is not None and _calls.fir1d(inp, out, taps, anchor):
        return out
    return _fir("hb_fir1d", inp, out, taps, anchor)


def hb_fir1d_valu(inp, out, taps, anchor):
    return _fir("hb_fir1d_valu", inp, out, taps, anchor)


def _conv2d(name, inp, out, taps2d, anchor_y, anchor_x, shape=lambda H, W: (H, W)):
    pi, H, W, ip = _img2d(inp, torch.float16)
    po, Ho, Wo, op = _img2d(out, torch.float32)
    assert shape(H, W) == (Ho, Wo), "output shape"
    k = np.asarray(taps2d)
    assert k.ndim == 2, "kh x kw tap array expected"
    bits, n = _taps(k)
    _check(name, getattr(_lib or load(), name)(pi, po, H, W, ip, op, bits, k.shape[0], k.shape[1],
                                               int(anchor_y), int(anchor_x), _stream()))
    return out


def hb_conv2d(inp, out, taps2d, anchor_y, anchor_x):
    if _calls is not None and _calls.conv2d(inp, out, taps2d, anchor_y, anchor_x):
        return out
    return _conv2d("hb_conv2d", inp, out, taps2d, anchor_y, anchor_x)


def hb_conv2d_valu(inp, out, taps2d, anchor_y, anchor_x):
    return _conv2d("hb_conv2d_valu", inp, out, taps2d, anchor_y, anchor_x)


def _half_shape(H, W):
    return (H + 1) // 2, (W + 1) // 2


def _double_shape(H, W):
    return 2 * H, 2 * W


def hb_down2(inp, out, taps2d, anchor_y, anchor_x):
    if _calls is not None and _calls.down2(inp, out, taps2d, anchor_y, anchor_x):
        return out
    return _conv2d("hb_down2", inp, out, taps2d, anchor_y, anchor_x, _half_shape)


def hb_down2_valu(inp, out, taps2d, anchor_y, anchor_x):
    return _conv2d("hb_down2_valu", inp, out, taps2d, anchor_y, anchor_x, _half_shape)


def hb_up2(inp, out, taps2d, anchor_y, anchor_x):
    if _calls is not None and _calls.up2(inp, out, taps2d, anchor_y, anchor_x):
        return out
    return _conv2d("hb_up2", inp, out, taps2d, anchor_y, anchor_x, _double_shape)


def hb_up2_valu(inp, out, taps2d, anchor_y, anchor_x):
    return _conv2d("hb_up2_valu", inp, out, taps2d, anchor_y, anchor_x, _double_shape)


def hb_dct_denoise_workspace_size(C, H, W):
    return int(load().hb_dct_denoise_workspace_size(int(C), int(H), int(W)))


def _dct(name, inp, out, threshold, workspace):
    pi, C, H, W, ip, il = _planes(inp, torch.float16)
    po, Co, Ho, Wo, op, ol = _planes(out, torch.float32)
    assert (C, H, W) == (Co, Ho, Wo)
    assert workspace.is_cuda and workspace.dtype == torch.uint8 and workspace.is_contiguous()
    _check(name, getattr(_lib or load(), name)(pi, po, C, H, W, ip, il, op, ol, float(threshold),
                                               workspace.data_ptr(), workspace.numel(), _stream()))
    return out


def hb_dct_denoise(inp, out, threshold, workspace):
    if _calls is not None and _calls.dct_denoise(inp, out, threshold, workspace):
        return out
    return _dct("hb_dct_denoise", inp, out, threshold, workspace)


def hb_dct_denoise_valu(inp, out, threshold, workspace):
    return _dct("hb_dct_denoise_valu", inp, out, threshold, workspace)


def hb_iir2_workspace_size(C, T):
    return int(load().hb_iir2_workspace_size(int(C), int(T)))


def hb_iir2_abs_gain(alpha, beta, T):
    return float(load().hb_iir2_abs_gain(float(alpha), float(beta), int(T)))


def _iir2(name, inp, out, alpha, beta, workspace):
    pi, C, T, ip = _img2d(inp, torch.float16)
    po, Co, To, op = _img2d(out, torch.float32)
    assert (C, T) == (Co, To)
    assert workspace.is_cuda and workspace.dtype == torch.uint8 and workspace.is_contiguous()
    _check(name, getattr(_lib or load(), name)(pi, po, C, T, ip, op, float(alpha), float(beta),
                                               workspace.data_ptr(), workspace.numel(), _stream()))
    return out


def hb_iir2(inp, out, alpha, beta, workspace):
    if _calls is not None and _calls.iir2(inp, out, alpha, beta, workspace):
        return out
    return _iir2("hb_iir2", inp, out, alpha, beta, workspace)


def hb_iir2_valu(inp, out, alpha, beta, workspace):
    return _iir2("hb_iir2_valu", inp, out, alpha, beta, workspace)


def hb_resize_workspace_size(C, H, Wo):
    return int(load().hb_resize_workspace_size(int(C), int(H), int(Wo)))


def hb_lanczos3_band(n_in, n_out):
    return int(load().hb_lanczos3_band(int(n_in), int(n_out)))


def hb_lanczos3_matrix(n_in, n_out):
    """Host arrays (start int32 [n_out], coef fp16 bit patterns [n_out, band]) built by the library."""
    band = hb_lanczos3_band(n_in, n_out)
    if band <= 0:
        raise HbError("hb_lanczos3_band", HB_ERR_INVALID_ARG)
    start = np.empty(n_out, dtype=np.int32)
    coef = np.empty((n_out, band), dtype=np.uint16)
    _check("hb_lanczos3_matrix", load().hb_lanczos3_matrix(int(n_in), int(n_out), start.ctypes.data_as(ctypes.c_void_p),
                                                          coef.ctypes.data_as(ctypes.c_void_p)))
    return start, coef


def _matrix(start, coef, n):
    """A banded matrix of n rows -> (address of its starts, of its coefficients, band)."""
    assert start.is_cuda and start.dtype == torch.int32 and start.is_contiguous() and start.shape == (n,)
    shape = coef.shape
    assert coef.is_cuda and coef.dtype == torch.float16 and coef.is_contiguous() and len(shape) == 2 and shape[0] == n
    return start.data_ptr(), coef.data_ptr(), shape[1]


def _resize(name, inp, out, workspace, start_y, coef_y, start_x, coef_x):
    pi, C, H, W, ip, il = _planes(inp, torch.float16)
    po, Co, Ho, Wo, op, ol = _planes(out, torch.float32)
    assert C == Co
    py, ky, by = _matrix(start_y, coef_y, Ho)
    px, kx, bx = _matrix(start_x, coef_x, Wo)
    assert workspace.is_cuda and workspace.dtype == torch.uint8 and workspace.is_contiguous()
    _check(name, getattr(_lib or load(), name)(pi, po, workspace.data_ptr(), workspace.numel(), C, H, W, Ho, Wo,
                                               ip, il, op, ol, py, ky, by, px, kx, bx, _stream()))
    return out


def hb_resize(inp, out, workspace, start_y, coef_y, start_x, coef_x):
    if _calls is not None and _calls.resize(inp, out, workspace, start_y, coef_y, start_x, coef_x):
        return out
    return _resize("hb_resize", inp, out, workspace, start_y, coef_y, start_x, coef_x)


def hb_resize_valu(inp, out, workspace, start_y, coef_y, start_x, coef_x):
    return _resize("hb_resize_valu", inp, out, workspace, start_y, coef_y, start_x, coef_x)


def _sep(name, inp, out, tx, ax, ty, ay):
    pi, H, W, ip = _img2d(inp, torch.float16)
    po, Ho, Wo, op = _img2d(out, torch.float32)
    assert (H, W) == (Ho, Wo)
    bx, nx = _taps(tx)
    by, ny = _taps(ty)
    _check(name, getattr(_lib or load(), name)(pi, po, H, W, ip, op, bx, nx, int(ax), by, ny, int(ay), _stream()))
    return out


def hb_sepblur(inp, out, taps_x, anchor_x, taps_y, anchor_y):
    if _calls is not None and _calls.sepblur(inp, out, taps_x, anchor_x, taps_y, anchor_y):
        return out
    return _sep("hb_sepblur", inp, out, taps_x, anchor_x, taps_y, anchor_y)


def hb_sepblur_valu(inp, out, taps_x, anchor_x, taps_y, anchor_y):
    return _sep("hb_sepblur_valu", inp, out, taps_x, anchor_x, taps_y, anchor_y)


def hb_sat2d_workspace_size(H, W) -> int:
    return int(load().hb_sat2d_workspace_size(int(H), int(W)))


def _sat(name, inp, out, workspace):
    pi, H, W, ip = _img2d(inp, torch.float16)
    po, Ho, Wo, op = _img2d(out, torch.float32)
    assert (H, W) == (Ho, Wo)
    assert workspace.is_cuda and workspace.is_contiguous()
    nbytes = workspace.numel() * workspace.element_size()
    _check(name, getattr(_lib or load(), name)(pi, po, H, W, ip, op, workspace.data_ptr(), nbytes, _stream()))
    return out


def hb_sat2d(inp, out, workspace):
    if _calls is not None and _calls.sat2d(inp, out, workspace):
        return out
    return _sat("hb_sat2d", inp, out, workspace)


def hb_sat2d_valu(inp, out, workspace):
    return _sat("hb_sat2d_valu", inp, out, workspace)


HB_SAT2D_NOALLOC_SCRATCH_BYTES = 5 << 20


def hb_sat2d_set_wait_limit(polls: int) -> int:
    return int(load().hb_sat2d_set_wait_limit(int(polls)))


def hb_sat2d_noalloc(inp, out):
    pi, H, W, ip = _img2d(inp, torch.float16)
    po, Ho, Wo, op = _img2d(out, torch.float32)
    assert (H, W) == (Ho, Wo)
    _check("hb_sat2d_noalloc", load().hb_sat2d_noalloc(pi, po, H, W, ip, op, _stream()))
    return out


def _conv(name, x, w, out):
    assert x.is_cuda and x.dtype == torch.float16 and x.is_contiguous() and x.dim() == 4
    assert w.is_cuda and w.dtype == torch.float16 and w.is_contiguous() and w.dim() == 4
    assert out.is_cuda and out.dtype == torch.float16 and out.is_contiguous() and out.dim() == 4
    N, H, W, Ci = x.shape
    Co = w.shape[3]
    assert tuple(w.shape) == (3, 3, Ci, Co) and tuple(out.shape) == (N, H, W, Co)
    _check(name, getattr(_lib or load(), name)(x.data_ptr(), w.data_ptr(), out.data_ptr(), N, H, W, Ci, Co, _stream()))
    return out


def hb_conv3x3(x_nhwc, w_hwio, out_nhwc):
    if _calls is not None and _calls.conv3x3(x_nhwc, w_hwio, out_nhwc):
        return out_nhwc
    return _conv("hb_conv3x3", x_nhwc, w_hwio, out_nhwc)


def hb_conv3x3_valu(x_nhwc, w_hwio, out_nhwc):
    return _conv("hb_conv3x3_valu", x_nhwc, w_hwio, out_nhwc)


def _pyr(name, inp, res, down):
    pi, H, W, ip = _img2d(inp, torch.float16)
    pr, Hr, Wr, rp = _img2d(res, torch.float32)
    assert (H, W) == (Hr, Wr)
    if down is not None:
        pd, Hd, Wd, dp = _img2d(down, torch.float16)
        assert (Hd, Wd) == (H // 2, W // 2)
    else:
        pd, dp = None, 0
    _check(name, getattr(_lib or load(), name)(pi, pr, pd, H, W, ip, rp, dp, _stream()))
    return res


def hb_pyr_level(inp, residual, down=None):
    if _calls is not None and _calls.pyr_level(inp, residual, down):
        return residual
    return _pyr("hb_pyr_level", inp, residual, down)


def hb_pyr_level_valu(inp, residual, down=None):
    return _pyr("hb_pyr_level_valu", inp, residual, down)


def _ints(*sizes):
    """Sizes as the library takes them: ctypes would pass the low 32 bits of larger ones."""
    n = [int(s) for s in sizes]
    assert max(n) <= 0x7fffffff, "sizes below 2^31 expected"
    return n


def hb_linear_workspace_size(M, N, K):
    return int(load().hb_linear_workspace_size(*_ints(M, N, K)))


def _scratch(t):
    """Address and size of a workspace; None is none."""
    if t is None:
        return None, 0
    assert t.is_cuda and t.dtype == torch.uint8 and t.is_contiguous(), "contiguous uint8 CUDA tensor expected"
    return t.data_ptr(), t.numel()


def _rows(t, dtype):
    """As _img2d; the stride from column to column of a single one has no meaning."""
    if t.dim() == 2 and t.shape[1] == 1:
        t = t.as_strided(t.shape, (t.stride(0), 1))
    return _img2d(t, dtype)


def _linear(name, x, w, out, workspace, bias, residual, act):
    px, M, K, xp = _rows(x, torch.float16)
    pw, N, Kw, wp = _rows(w, torch.float16)
    assert out.dtype in (torch.float16, torch.float32), "fp16 or fp32 output expected"
    po, Mo, No, op = _rows(out, out.dtype)
    assert K == Kw and (Mo, No) == (M, N), "x: M x K, w: N x K, out: M x N"
    _ints(M, N, K)
    pb = pr = None
    rp = N
    if bias is not None:
        assert bias.is_cuda and bias.dtype == torch.float16 and bias.shape == (N,) and bias.is_contiguous(), "bias: N"
        pb = bias.data_ptr()
    if residual is not None:
        pr, Mr, Nr, rp = _rows(residual, out.dtype)
        assert (Mr, Nr) == (M, N), "residual: M x N"
    pws, nws = _scratch(workspace)
    if M == 1:                                    # the pitch of a single row has no meaning, and torch gives any
        xp, op, rp = K, N, N
    if N == 1:
        wp = K
    _check(name, getattr(_lib or load(), name)(px, pw, pb, pr, po, 1 if out.dtype == torch.float32 else 0, HB_ACTS[act], M, N, K, xp, wp, rp, op,
                                               pws, nws, _stream()))
    return out


def hb_linear(x, w, out, workspace=None, bias=None, residual=None, act="none"):
    """out = act(x w^T + bias) + residual; x: M x K, w: N x K, out and residual: M x N, fp16 or fp32."""
    if _calls is not None and _calls.linear(x, w, out, workspace, bias, residual, act):
        return out
    return _linear("hb_linear", x, w, out, workspace, bias, residual, act)


def hb_linear_valu(x, w, out, workspace=None, bias=None, residual=None, act="none"):
    return _linear("hb_linear_valu", x, w, out, workspace, bias, residual, act)


def _heads(t):
    """B x L x H x D, the last axis dense -> (address, (B, L, H, D), strides of the first three)."""
    s = t.stride()
    assert t.is_cuda and t.dtype == torch.float16 and len(s) == 4 and (s[3] == 1 or t.shape[3] == 1), "B x L x H x D fp16 CUDA tensor expected"
    _ints(*t.shape)
    return t.data_ptr(), t.shape, s[:3]


def hb_rope_axes(x, out, positions, freq, sections, interleaved=False):
    """Turns channel pairs of x (B x L x H x D) by positions (B x L x axes) times freq; out may be x."""
    if _calls is not None and _calls.rope_axes(x, out, positions, freq, sections, interleaved):
        return out
    px, (B, L, H, D), xs = _heads(x)
    po, shape, os_ = _heads(out)
    assert shape == x.shape, "output shape"
    n = len(sections)
    ps = positions.stride()
    assert positions.is_cuda and positions.dtype == torch.int32 and tuple(positions.shape) == (B, L, n) and (ps[2] == 1 or n == 1), "positions: B x L x axes, int32"
    assert freq.is_cuda and freq.dtype == torch.float32 and freq.is_contiguous() and freq.shape == (sum(sections),), "freq: a value per pair, fp32"
    _check("hb_rope_axes", (_lib or load()).hb_rope_axes(px, po, positions.data_ptr(), freq.data_ptr(), B, L, H, D, *xs, *os_, ps[0], ps[1],
                                                         (ctypes.c_int32 * n)(*sections), n, int(bool(interleaved)), _stream()))
    return out


def hb_attention_workspace_size(B, Lq, Lk, Hq, Hkv, D):
    return int(load().hb_attention_workspace_size(*_ints(B, Lq, Lk, Hq, Hkv, D)))


def _attention(name, q, k, v, out, scale, workspace, key_len, key_mask):
    pq, (B, Lq, Hq, D), qs = _heads(q)
    pk, (Bk, Lk, Hkv, Dk), ks = _heads(k)
    pv, shape, vs = _heads(v)
    po, oshape, os_ = _heads(out)
    assert (Bk, Dk) == (B, D) and shape == k.shape and oshape == q.shape, "q, out: B x Lq x Hq x D, k, v: B x Lk x Hkv x D"
    pl = pm = None
    mp = 0
    if key_len is not None:
        assert key_len.is_cuda and key_len.dtype == torch.int32 and key_len.shape == (B,) and key_len.is_contiguous(), "key_len: B, int32"
        pl = key_len.data_ptr()
    if key_mask is not None:
        assert key_mask.is_cuda and key_mask.dtype in (torch.uint8, torch.bool) and key_mask.shape == (B, Lk), "key_mask: B x Lk, uint8 or bool"
        assert key_mask.stride(1) == 1 or Lk <= 1, "key_mask: dense rows"
        pm, mp = key_mask.data_ptr(), key_mask.stride(0)
    pws, nws = _scratch(workspace)
    _check(name, getattr(_lib or load(), name)(pq, pk, pv, po, B, Lq, Lk, Hq, Hkv, D, *qs, *ks, *vs, *os_, float(scale), pl, pm, mp,
                                               pws, nws, _stream()))
    return out


def hb_attention(q, k, v, out, scale, workspace=None, key_len=None, key_mask=None):
    """out = softmax(scale q k^T) v over the visible keys; q, out: B x Lq x Hq x D, k, v: B x Lk x Hkv x D."""
    if _calls is not None and _calls.attention(q, k, v, out, scale, workspace, key_len, key_mask):
        return out
    return _attention("hb_attention", q, k, v, out, scale, workspace, key_len, key_mask)


def hb_attention_valu(q, k, v, out, scale, workspace=None, key_len=None, key_mask=None):
    return _attention("hb_attention_valu", q, k, v, out, scale, workspace, key_len, key_mask)


def hb_copy_f16_f32(inp, out):
    n = inp.numel()
    assert out.numel() == n
    _check("hb_copy_f16_f32", load().hb_copy_f16_f32(inp.data_ptr(),
                                                     out.data_ptr(), n, _stream()))
    return out


def hb_mfma_probe(which, A, B, D):
    _check("hb_mfma_probe", load().hb_mfma_probe(int(which), A.data_ptr(),
                                                 B.data_ptr(),
                                                 D.data_ptr(), _stream()))
    return D
