"""Thin binding of the elementwise / loss / optimiser entry points (marshalling only)."""
import ctypes

import torch

from ._lib import check, lib
from .swap import _stream


def _p(t):
    return ctypes.c_void_p(t.data_ptr())


def leaky_relu_fwd(a, slope=0.01):
    check(lib().mi3d_leaky_relu_fwd(_p(a), a.numel(), slope, _stream()), "leaky_relu_fwd")


def leaky_relu_bwd(da, a, slope=0.01):
    assert da.numel() == a.numel() and da.dtype == a.dtype
    if da.dtype == torch.float32:
        check(lib().mi3d_leaky_relu_bwd_f32(_p(da), _p(a), a.numel(), slope, _stream()), "leaky_relu_bwd_f32")
    else:
        check(lib().mi3d_leaky_relu_bwd(_p(da), _p(a), a.numel(), slope, _stream()), "leaky_relu_bwd")


def concat_channels(a, b, out):
    Ca, Cb = a.shape[-1], b.shape[-1]
    vox = a.numel() // Ca
    assert b.numel() // Cb == vox and out.numel() == vox * (Ca + Cb)
    check(lib().mi3d_concat_channels(_p(a), Ca, _p(b), Cb, _p(out), vox, _stream()), "concat_channels")


def split_channels(x, a, b):
    Ca, Cb = a.shape[-1], b.shape[-1]
    vox = a.numel() // Ca
    assert b.numel() // Cb == vox and x.numel() == vox * (Ca + Cb)
    check(lib().mi3d_split_channels(_p(x), Ca, Cb, _p(a), _p(b), vox, _stream()), "split_channels")


def slice_channels(x, c_off, out):
    Ct, C = x.shape[-1], out.shape[-1]
    vox = out.numel() // C
    assert x.numel() == vox * Ct
    check(lib().mi3d_slice_channels(_p(x), Ct, c_off, C, _p(out), vox, _stream()), "slice_channels")


def place_channels(x, out, c_off):
    """out[..., c_off : c_off + C] = x; the other channels of out stay as they are."""
    C, Ct = x.shape[-1], out.shape[-1]
    vox = x.numel() // C
    assert out.numel() == vox * Ct
    check(lib().mi3d_place_channels(_p(x), C, _p(out), Ct, c_off, vox, _stream()), "place_channels")


def skip_grad(da, dcat, c_off, a, slope=0.01):
    """da <- (da + dcat[..., c_off : c_off + C]) * (a > 0 ? 1 : slope), in place on da."""
    Ct, C = dcat.shape[-1], da.shape[-1]
    vox = da.numel() // C
    assert dcat.numel() == vox * Ct and a.numel() == da.numel()
    check(lib().mi3d_skip_grad(_p(da), _p(dcat), Ct, c_off, _p(a), C, vox, slope, _stream()), "skip_grad")


def add_inplace(a, b):
    assert a.numel() == b.numel()
    check(lib().mi3d_add_inplace(_p(a), _p(b), a.numel(), _stream()), "add_inplace")


def dice_workspace(classes=3):
    return torch.empty(lib().mi3d_dice_workspace_bytes(classes), dtype=torch.uint8, device="cuda")


def dice_loss(logits, labels, ws, sums, loss, eps=1e-5):
    C = logits.shape[-1]
    vox = logits.numel() // C
    fn = lib().mi3d_dice_loss_f32 if logits.dtype == torch.float32 else lib().mi3d_dice_loss
    check(fn(_p(logits), _p(labels), vox, C, eps, _p(ws), ws.numel(), _p(sums), _p(loss), _stream()), "dice_loss")


def dice_grad(logits, labels, sums, dlogits, eps=1e-5):
    C = logits.shape[-1]
    vox = logits.numel() // C
    assert logits.dtype == dlogits.dtype
    fn = lib().mi3d_dice_grad_f32 if logits.dtype == torch.float32 else lib().mi3d_dice_grad
    check(fn(_p(logits), _p(labels), vox, C, eps, _p(sums), _p(dlogits), _stream()), "dice_grad")


def sgd_update(w32, dw32, w16, lr):
    """w16 None: no bf16 working copy (the fp32 step)."""
    assert w32.numel() == dw32.numel() and (w16 is None or w16.numel() == w32.numel())
    check(lib().mi3d_sgd_update(_p(w32), _p(dw32), None if w16 is None else _p(w16), w32.numel(), lr, _stream()), "sgd_update")


def adam_update(w32, dw32, m32, v32, w16, lr, step, beta1=0.9, beta2=0.999, eps=1e-8):
    assert w32.numel() == dw32.numel() == m32.numel() == v32.numel() and (w16 is None or w16.numel() == w32.numel())
    check(lib().mi3d_adam_update(_p(w32), _p(dw32), _p(m32), _p(v32), None if w16 is None else _p(w16), w32.numel(), lr, beta1, beta2, eps, int(step), _stream()), "adam_update")


IN_EPS = 1e-5


def instnorm_workspace(N, C):
    return torch.empty(lib().mi3d_instnorm_workspace_bytes(N, C), dtype=torch.uint8, device="cuda")


def instnorm_stats(z, stats, ws, eps=IN_EPS):
    """stats[n, c] = (mean, 1 / sqrt(var + eps)) of z[n, ..., c]."""
    N, C = z.shape[0], z.shape[-1]
    vox = z.numel() // (N * C)
    assert tuple(stats.shape) == (N, C, 2) and stats.dtype == torch.float32
    fn = lib().mi3d_instnorm_stats_f32 if z.dtype == torch.float32 else lib().mi3d_instnorm_stats
    check(fn(_p(z), N, vox, C, eps, _p(stats), _p(ws), ws.numel(), _stream()), "instnorm_stats")


def instnorm_lrelu_fwd(z, stats, slope=0.01):
    N, C = z.shape[0], z.shape[-1]
    fn = lib().mi3d_instnorm_lrelu_fwd_f32 if z.dtype == torch.float32 else lib().mi3d_instnorm_lrelu_fwd
    check(fn(_p(z), _p(stats), N, z.numel() // (N * C), C, slope, _stream()), "instnorm_lrelu_fwd")


def instnorm_lrelu_bwd_sums(da, a, stats, sums, slope=0.01):
    """da <- dz given the two means (mean g, mean g * xhat) per (sample, channel)."""
    N, C = a.shape[0], a.shape[-1]
    assert da.numel() == a.numel() and tuple(sums.shape) == (N, C, 2) and sums.dtype == torch.float32
    assert a.dtype == torch.bfloat16 and da.dtype == torch.bfloat16      # (bf16 only: the kernels that deliver the sums are)
    check(lib().mi3d_instnorm_lrelu_bwd_sums(_p(da), _p(a), _p(stats), _p(sums), N, a.numel() // (N * C), C, slope, _stream()), "instnorm_lrelu_bwd_sums")


def instnorm_lrelu_bwd(da, a, stats, ws, slope=0.01):
    N, C = a.shape[0], a.shape[-1]
    assert da.numel() == a.numel() and da.dtype == a.dtype
    fn = lib().mi3d_instnorm_lrelu_bwd_f32 if a.dtype == torch.float32 else lib().mi3d_instnorm_lrelu_bwd
    check(fn(_p(da), _p(a), _p(stats), N, a.numel() // (N * C), C, slope, _p(ws), ws.numel(), _stream()), "instnorm_lrelu_bwd")


def _current(t, name):
    """The current stream of the current device, where t has to be (half a microsecond; a torch stream object takes three)."""
    dev = t.get_device()
    if dev < 0 or dev != torch.cuda.current_device():
        raise ValueError(f"{name}: need a tensor on the current device, got one on {t.device}")
    return dev, torch._C._cuda_getCurrentRawStream(dev)


def _operands(dev, dtype, shape, **tensors):
    """Refuses what is not a dense tensor of this type and shape on this device (None: left out)."""
    for name, t in tensors.items():
        if t is not None and (t.get_device() != dev or t.dtype is not dtype or t.shape != shape or not t.is_contiguous()):
            raise ValueError(f"{name}: need contiguous {dtype} tensor of shape {tuple(shape)} on the current device, got {t.dtype} {tuple(t.shape)} on {t.device}")


def _typed(name, dtype):
    if dtype is torch.bfloat16:
        return getattr(lib(), name)
    if dtype is torch.float32:
        return getattr(lib(), name + "_f32")
    raise ValueError(f"{name[5:]}: bf16 and fp32 tensors, got {dtype}")


def _ptr(t):
    return None if t is None else t.data_ptr()


def layernorm_workspace(rows, C):
    return torch.empty(lib().mi3d_layernorm_workspace_bytes(rows, C), dtype=torch.uint8, device="cuda")


def layernorm_fwd(x, gamma, beta, y=None, stats=None, eps=IN_EPS):
    """y = gamma * (x - mean) * rstd + beta over the last dimension of x, stats[row] = (mean, rstd); gamma, beta and stats fp32.
    y may be x."""
    fn, shape, C, dt = _typed("mi3d_layernorm_fwd", x.dtype), x.shape, x.shape[-1], torch.float32
    dev, stream = _current(x, "x")
    rows = x.numel() // max(C, 1)
    if y is None:
        y = torch.empty_like(x, memory_format=torch.contiguous_format)
    if stats is None:
        stats = torch.empty((rows, 2), dtype=torch.float32, device=x.device)
    _operands(dev, x.dtype, shape, x=x, y=y)
    _operands(dev, dt, (C,), gamma=gamma, beta=beta)
    _operands(dev, dt, (rows, 2), stats=stats)
    check(fn(x.data_ptr(), gamma.data_ptr(), beta.data_ptr(), rows, C, eps, y.data_ptr(), stats.data_ptr(), stream), "layernorm_fwd")
    return y, stats


def layernorm_bwd(dy, x, stats, gamma, dx=None, dgamma=None, dbeta=None, ws=None, add=None):
    """dx (+ add, the gradient of a connection past the block), dgamma, dbeta.  dx may be dy, x or add."""
    fn, shape, C, dt = _typed("mi3d_layernorm_bwd", x.dtype), x.shape, x.shape[-1], torch.float32
    dev, stream = _current(x, "x")
    rows = x.numel() // max(C, 1)
    if dx is None:
        dx = torch.empty_like(x, memory_format=torch.contiguous_format)
    if dgamma is None:
        dgamma = torch.empty(C, dtype=torch.float32, device=x.device)
    if dbeta is None:
        dbeta = torch.empty(C, dtype=torch.float32, device=x.device)
    _operands(dev, x.dtype, shape, dy=dy, x=x, dx=dx, add=add)
    _operands(dev, dt, (C,), gamma=gamma, dgamma=dgamma, dbeta=dbeta)
    _operands(dev, dt, (rows, 2), stats=stats)
    if ws is None:
        ws = layernorm_workspace(rows, C)
    _operands(dev, torch.uint8, ws.shape, ws=ws)
    check(fn(dy.data_ptr(), x.data_ptr(), stats.data_ptr(), gamma.data_ptr(), _ptr(add), rows, C, dx.data_ptr(), dgamma.data_ptr(), dbeta.data_ptr(),
             ws.data_ptr(), ws.numel(), stream), "layernorm_bwd")
    return dx, dgamma, dbeta


def dropout_fwd(a, p, seed, offset=0, residual=None, out=None, dev_offset=None):
    """out = residual + dropout(a) with the numbers of stream (seed, offset); dev_offset: an int64 of one value on the device that is
    added to offset when the kernel runs: calls that share it need offsets further apart than it ever grows (layer << 40, say), or
    one layer draws in this step what another one drew in an earlier step.  out may be a or residual."""
    fn, (dev, stream) = _typed("mi3d_dropout_fwd", a.dtype), _current(a, "a")
    if out is None:
        out = torch.empty_like(a, memory_format=torch.contiguous_format)
    _operands(dev, a.dtype, a.shape, a=a, residual=residual, out=out)
    _operands(dev, torch.int64, (1,), dev_offset=dev_offset)
    check(fn(a.data_ptr(), _ptr(residual), out.data_ptr(), a.numel(), p, seed, offset, _ptr(dev_offset), stream), "dropout_fwd")
    return out


def dropout_bwd(dout, p, seed, offset=0, da=None, dev_offset=None):
    """da = the gradient of dropout_fwd's a: the same values are dropped (seed, offset and dev_offset as in the forward pass).  da may be
    dout."""
    fn, (dev, stream) = _typed("mi3d_dropout_bwd", dout.dtype), _current(dout, "dout")
    if da is None:
        da = torch.empty_like(dout, memory_format=torch.contiguous_format)
    _operands(dev, dout.dtype, dout.shape, dout=dout, da=da)
    _operands(dev, torch.int64, (1,), dev_offset=dev_offset)
    check(fn(dout.data_ptr(), da.data_ptr(), dout.numel(), p, seed, offset, _ptr(dev_offset), stream), "dropout_bwd")
    return da


def dropout_channels(a, p, seed, offset=0, out=None, dev_offset=None):
    """Drops whole channels of the samples of a [N, ..., C]; forward and backward pass alike.  dev_offset: as in dropout_fwd.  out may
    be a."""
    if a.dim() < 2:
        raise ValueError(f"a: need [N, ..., C], got {tuple(a.shape)}")
    fn, (dev, stream) = _typed("mi3d_dropout_channels", a.dtype), _current(a, "a")
    if out is None:
        out = torch.empty_like(a, memory_format=torch.contiguous_format)
    _operands(dev, a.dtype, a.shape, a=a, out=out)
    _operands(dev, torch.int64, (1,), dev_offset=dev_offset)
    N, C = a.shape[0], a.shape[-1]
    check(fn(a.data_ptr(), out.data_ptr(), N, a.numel() // max(N * C, 1), C, p, seed, offset, _ptr(dev_offset), stream), "dropout_channels")
    return out
