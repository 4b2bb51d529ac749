"""Thin binding of the gated feed-forward block: argument marshalling only.

Tensors are [rows, channels] (or NDHWC: every leading dimension counts as rows), bf16 or fp32, dense, on the current device; w1
holds the gate's F rows and then the F rows that it multiplies.
"""
import ctypes

import torch

from ._lib import FfnDesc, check, lib
from .conv3d import _DT, PASS_DGRAD, PASS_FWD, PASS_WGRAD, _tdtype
from .glue import _current, _ptr

ACT = {"silu": 0, "gelu": 1}


def make_desc(rows, Cin, F, Cout, act, dtype):
    """act: "silu" or "gelu"."""
    return FfnDesc(rows, Cin, F, Cout, ACT[act], _DT[dtype])


def workspace_bytes(desc, pass_):
    return int(lib().mi3d_ffn_workspace_bytes(ctypes.byref(desc), pass_))


def workspace(desc, pass_):
    return torch.empty(max(workspace_bytes(desc, pass_), 16), dtype=torch.uint8, device="cuda")


def kernel_detail(desc, pass_):
    """The kernels that a call runs."""
    buf = ctypes.create_string_buffer(128)
    check(lib().mi3d_ffn_kernel_detail(ctypes.byref(desc), pass_, buf, 128), "ffn_kernel_detail")
    return buf.value.decode()


def _chk(dev, rows, C, dtype, **tensors):
    """Refuses what is not a dense tensor of rows x C values of this type on this device (None: left out)."""
    for name, t in tensors.items():
        if t is not None and (t.get_device() != dev or t.dtype is not dtype or t.shape[-1] != C or t.numel() != rows * C or not t.is_contiguous()):
            raise ValueError(f"{name}: need contiguous {dtype} tensor of {rows} x {C} on the current device, got {t.dtype} {tuple(t.shape)} on {t.device}")


def _new(like, C, rows):
    return torch.empty(tuple(like.shape[:-1]) + (C,) if like.numel() // max(like.shape[-1], 1) == rows else (rows, C), dtype=like.dtype, device=like.device)


def _ws(dev, desc, pass_, ws):
    if ws is None:
        return workspace(desc, pass_)
    _chk(dev, 1, ws.shape[-1], torch.uint8, ws=ws)
    return ws


def ffn_gate(desc, x, w1, h=None, gu=None):
    """h = act(g) * u with [g | u] = x w1^T, which gu (optional) receives."""
    if h is None:
        h = _new(x, desc.F, desc.rows)
    dt, (dev, stream) = _tdtype(desc), _current(x, "x")
    _chk(dev, desc.rows, desc.Cin, dt, x=x)
    _chk(dev, 2 * desc.F, desc.Cin, dt, w1=w1)
    _chk(dev, desc.rows, desc.F, dt, h=h)
    _chk(dev, desc.rows, 2 * desc.F, dt, gu=gu)
    check(lib().mi3d_ffn_gate(ctypes.byref(desc), x.data_ptr(), w1.data_ptr(), h.data_ptr(), _ptr(gu), stream), "ffn_gate")
    return h


def ffn_fwd(desc, x, w1, w2, y=None, gu=None, ws=None):
    """y = (act(g) * u) w2^T; gu (optional) receives [g | u] for the backward pass."""
    if y is None:
        y = _new(x, desc.Cout, desc.rows)
    dt, (dev, stream) = _tdtype(desc), _current(x, "x")
    _chk(dev, desc.rows, desc.Cin, dt, x=x)
    _chk(dev, 2 * desc.F, desc.Cin, dt, w1=w1)
    _chk(dev, desc.Cout, desc.F, dt, w2=w2)
    _chk(dev, desc.rows, desc.Cout, dt, y=y)
    _chk(dev, desc.rows, 2 * desc.F, dt, gu=gu)
    ws = _ws(dev, desc, PASS_FWD, ws)
    check(lib().mi3d_ffn_fwd(ctypes.byref(desc), x.data_ptr(), w1.data_ptr(), w2.data_ptr(), y.data_ptr(), _ptr(gu), ws.data_ptr(), ws.numel(), stream), "ffn_fwd")
    return y


def ffn_dgrad(desc, dy, w1, w2, gu, dx=None, dgu=None, h=None, ws=None):
    """(dx, dgu, h): the gradients of x and of [g | u], and act(g) * u again; ffn_wgrad reads the last two."""
    if dx is None:
        dx = _new(dy, desc.Cin, desc.rows)
    if dgu is None:
        dgu = _new(dy, 2 * desc.F, desc.rows)
    if h is None:
        h = _new(dy, desc.F, desc.rows)
    dt, (dev, stream) = _tdtype(desc), _current(dy, "dy")
    _chk(dev, desc.rows, desc.Cout, dt, dy=dy)
    _chk(dev, 2 * desc.F, desc.Cin, dt, w1=w1)
    _chk(dev, desc.Cout, desc.F, dt, w2=w2)
    _chk(dev, desc.rows, 2 * desc.F, dt, gu=gu, dgu=dgu)
    _chk(dev, desc.rows, desc.F, dt, h=h)
    _chk(dev, desc.rows, desc.Cin, dt, dx=dx)
    ws = _ws(dev, desc, PASS_DGRAD, ws)
    check(lib().mi3d_ffn_dgrad(ctypes.byref(desc), dy.data_ptr(), w1.data_ptr(), w2.data_ptr(), gu.data_ptr(), dgu.data_ptr(), h.data_ptr(), dx.data_ptr(),
                               ws.data_ptr(), ws.numel(), stream), "ffn_dgrad")
    return dx, dgu, h


def ffn_wgrad(desc, x, dgu, h, dy, dw1=None, dw2=None, ws=None):
    """(dw1, dw2), fp32."""
    if dw1 is None:
        dw1 = torch.empty((2 * desc.F, desc.Cin), dtype=torch.float32, device=x.device)
    if dw2 is None:
        dw2 = torch.empty((desc.Cout, desc.F), dtype=torch.float32, device=x.device)
    dt, (dev, stream) = _tdtype(desc), _current(x, "x")
    _chk(dev, desc.rows, desc.Cin, dt, x=x)
    _chk(dev, desc.rows, 2 * desc.F, dt, dgu=dgu)
    _chk(dev, desc.rows, desc.F, dt, h=h)
    _chk(dev, desc.rows, desc.Cout, dt, dy=dy)
    _chk(dev, 2 * desc.F, desc.Cin, torch.float32, dw1=dw1)
    _chk(dev, desc.Cout, desc.F, torch.float32, dw2=dw2)
    ws = _ws(dev, desc, PASS_WGRAD, ws)
    check(lib().mi3d_ffn_wgrad(ctypes.byref(desc), x.data_ptr(), dgu.data_ptr(), h.data_ptr(), dy.data_ptr(), dw1.data_ptr(), dw2.data_ptr(),
                               ws.data_ptr(), ws.numel(), stream), "ffn_wgrad")
    return dw1, dw2
