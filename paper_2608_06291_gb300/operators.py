"""The operators that run and score a quantised model, same names as the C ABI:
the product with a quantised weight, the root-mean-square norm, the log
probabilities of given tokens, and the gradients of the last two.

Tensors may have any number of leading dimensions where their rows are evenly
spaced (or else are copied); the last dimension is contiguous.  Work is enqueued on
``stream`` (default: the current one).
"""
from __future__ import annotations

import functools

import torch

from .bakron import BF16, E4M3, F32, OK, BakronError, lib

_DTYPES = {torch.float32: F32, torch.bfloat16: BF16, torch.float8_e4m3fn: E4M3}
_ACTIVATIONS = {None: 0, "none": 0, "relu": 1, "silu": 2, "gelu": 3}


def _check(rc, what):
    if rc != OK:
        raise BakronError(rc, what)


def _rows(t, name, dtypes, device=None):
    """t as rows x d: (tensor, number of rows, row stride in elements)."""
    if t.dtype not in dtypes:
        raise ValueError(f"{name} must be {' or '.join(str(d)[6:] for d in dtypes)}")
    if not t.is_cuda or t.dim() < 1 or (device is not None and t.device != device):
        raise ValueError(f"{name} must be a CUDA tensor" + ("" if device is None else f" on {device}"))
    d = t.shape[-1]
    if t.dim() != 2:
        t = t.reshape(-1, d) if d else t.reshape(0, 0)
    if t.stride(1) != 1 and d > 1 or t.shape[0] > 1 and t.stride(0) < d:
        t = t.contiguous()
    return t, t.shape[0], max(t.stride(0), d)


def _vector(t, n, name, dtypes, device):
    if t is None:
        return None
    if t.device != device or t.dtype not in dtypes or t.numel() != n:
        raise ValueError(f"{name} must be {n} values of {' or '.join(str(d)[6:] for d in dtypes)} on {device}")
    return t.contiguous()


def _like(t, shape, name, dtype, device):
    """A tensor of the shape and type asked for, as rows."""
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}")
    return _rows(t, name, (dtype,), device)


def _p(t):
    return None if t is None else t.data_ptr()


def _placed(fn):
    """Runs fn on the device of its first argument and on ``stream``: also what fn copies
    and allocates belongs to that stream."""
    @functools.wraps(fn)
    def call(t, *args, stream=None, **kwargs):
        if stream is not None:
            with torch.cuda.stream(stream):
                return call(t, *args, **kwargs)
        if t.is_cuda and t.device.index != torch.cuda.current_device():
            with torch.cuda.device(t.device):
                return fn(t, *args, **kwargs)
        return fn(t, *args, **kwargs)
    return call


def _stream(device):
    return torch.cuda.current_stream(device).cuda_stream


class PackedWeight:
    """A quantised m x n weight laid out for ``bakron_linear``."""

    def __init__(self, m, n, qmax, group_size, buf):
        self.m, self.n, self.qmax, self.group_size, self.buf = m, n, qmax, group_size, buf

    @property
    def device(self):
        return self.buf.device


@_placed
def bakron_pack_weight(codes, scales, zeros, qmax: int, group_size: int = 0) -> PackedWeight:
    """Lay out codes (m x n uint8, 0..qmax), scales and zeros (m x G fp32) as the solve
    leaves them: code c of row i, group g stands for s[i, g] (c - z[i, g]).  group_size 0
    or a multiple of 32.  4 bits a code up to qmax 15, else 8.  Synchronous."""
    if codes.dim() != 2:
        raise ValueError("codes must be m x n")
    codes, m, ldc = _rows(codes, "codes", (torch.uint8,))
    n, group_size = codes.shape[1], int(group_size)
    G = 1 if group_size <= 0 else n // group_size
    dev = codes.device
    scales = _like(scales, (m, G), "scales", torch.float32, dev)[0].contiguous()
    zeros = _like(zeros, (m, G), "zeros", torch.float32, dev)[0].contiguous()
    L = lib()
    size = L.bakron_packed_bytes(m, n, int(qmax), group_size)
    buf = torch.empty(size, dtype=torch.uint8, device=dev)
    _check(L.bakron_pack_weight(codes.data_ptr(), ldc, scales.data_ptr(), zeros.data_ptr(), m, n, int(qmax),
                                group_size, buf.data_ptr(), size, _stream(dev)), "bakron_pack_weight")
    return PackedWeight(m, n, int(qmax), group_size, buf)


@_placed
def bakron_linear(x, weight: PackedWeight, x_scales=None, bias=None, activation=None, residual=None,
                  out_dtype=torch.bfloat16, out=None, workspace=None, sync: bool = False):
    """act(x What^T + bias) + residual for the tokens x (... x n, bfloat16 or
    float8_e4m3fn with ``x_scales``, one fp32 a token).  ``activation``: None, "relu",
    "silu" or "gelu".  ``bias``: m fp32; ``residual`` and the result (... x m): ``out_dtype``,
    bfloat16 or float32.  ``out`` may be ``residual``.  ``sync``: wait, and raise what the
    device reports (``bakron_read_status(workspace)`` tells it later)."""
    shape, dev = x.shape, weight.buf.device
    x, rows, ldx = _rows(x, "x", (torch.bfloat16, torch.float8_e4m3fn), dev)
    m, n = weight.m, weight.n
    if x.shape[1] != n:
        raise ValueError(f"x must have {n} columns")
    if activation not in _ACTIVATIONS:
        raise ValueError(f"activation must be one of {[a for a in _ACTIVATIONS if a]} or None")
    if out is not None:
        out_dtype = out.dtype
    if out_dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("the result must be bfloat16 or float32")
    yshape = (*shape[:-1], m)
    x_scales = _vector(x_scales, rows, "x_scales", (torch.float32,), dev)
    bias = _vector(bias, m, "bias", (torch.float32,), dev)
    ldr = 0
    if residual is not None:
        residual, _, ldr = _like(residual, yshape, "residual", out_dtype, dev)
    L = lib()
    if out is None:
        out = torch.empty(yshape, dtype=out_dtype, device=dev)
    y, _, ldy = _like(out, yshape, "out", out_dtype, dev)
    if y.data_ptr() != out.data_ptr():
        raise ValueError("out must have evenly spaced rows and a contiguous last dimension")
    dt = _DTYPES[x.dtype]
    need = L.bakron_linear_workspace_bytes(x.data_ptr(), dt, rows, ldx, n, weight.qmax, weight.group_size)
    if need and workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=dev)
    rc = L.bakron_linear(x.data_ptr(), dt, rows, ldx, _p(x_scales), weight.buf.data_ptr(), m, n, weight.qmax,
                         weight.group_size, _p(bias), _ACTIVATIONS[activation], _p(residual), ldr,
                         y.data_ptr(), _DTYPES[out_dtype], ldy, _p(workspace),
                         0 if workspace is None else workspace.numel(), 1 if sync else 0, _stream(dev))
    if rc != OK:
        raise BakronError(rc, "bakron_linear")
    return out


@_placed
def bakron_rmsnorm(x, weight, eps: float = 1e-6, residual=None, out_dtype=None):
    """h = x + residual, y = weight h / sqrt(mean(h^2) + eps) over the last dimension.
    Returns (y, scales, h): y of ``out_dtype`` (default x's; or float8_e4m3fn with
    ``scales``, one fp32 a row, else None), h of x's type (None without a residual)."""
    shape, dev, dtype = x.shape, x.device, x.dtype
    x, rows, ldx = _rows(x, "x", (torch.float32, torch.bfloat16))
    d = x.shape[1]
    weight = _vector(weight, d, "weight", (torch.float32, torch.bfloat16), dev)
    out_dtype = out_dtype or dtype
    if out_dtype not in (dtype, torch.float8_e4m3fn):
        raise ValueError("out_dtype must be x's or float8_e4m3fn")
    ldr = 0
    if residual is not None:
        residual, _, ldr = _like(residual, shape, "residual", dtype, dev)
    L = lib()
    y = torch.empty(shape, dtype=out_dtype, device=dev)
    h = torch.empty(shape, dtype=dtype, device=dev) if residual is not None else None
    scales = torch.empty(shape[:-1], dtype=torch.float32, device=dev) if out_dtype != dtype else None
    rc = L.bakron_rmsnorm(x.data_ptr(), _DTYPES[dtype], rows, d, ldx, _p(residual), ldr, weight.data_ptr(),
                          _DTYPES[weight.dtype], float(eps), _p(h), d, y.data_ptr(), _DTYPES[out_dtype], d,
                          _p(scales), _stream(dev))
    if rc != OK:
        raise BakronError(rc, "bakron_rmsnorm")
    return y, scales, h


@_placed
def bakron_rmsnorm_backward(dy, h, weight, eps: float = 1e-6, dsum=None):
    """Gradients of y = weight h / sqrt(mean(h^2) + eps), given dy and the gradient ``dsum``
    that reaches h past the norm.  Returns (dx of h's type, dweight fp32)."""
    shape, dev, dtype = h.shape, h.device, h.dtype
    h, rows, ldh = _rows(h, "h", (torch.float32, torch.bfloat16))
    d = h.shape[1]
    dy, _, lddy = _like(dy, shape, "dy", dtype, dev)
    weight = _vector(weight, d, "weight", (torch.float32, torch.bfloat16), dev)
    ldds = 0
    if dsum is not None:
        dsum, _, ldds = _like(dsum, shape, "dsum", dtype, dev)
    L = lib()
    dx = torch.empty(shape, dtype=dtype, device=dev)
    dw = torch.empty(d, dtype=torch.float32, device=dev)
    size = L.bakron_rmsnorm_backward_workspace_bytes(rows, d)
    ws = torch.empty(size, dtype=torch.uint8, device=dev)
    rc = L.bakron_rmsnorm_backward(dy.data_ptr(), lddy, h.data_ptr(), ldh, _DTYPES[dtype], rows, d,
                                   weight.data_ptr(), _DTYPES[weight.dtype], float(eps), _p(dsum), ldds,
                                   dx.data_ptr(), d, dw.data_ptr(), ws.data_ptr(), size, _stream(dev))
    if rc != OK:
        raise BakronError(rc, "bakron_rmsnorm_backward")
    return dx, dw


@_placed
def bakron_token_logprobs(logits, targets=None, top: int = 0):
    """Log probabilities of the tokens ``targets`` (int64; outside 0..v-1: not scored, 0)
    under logits (... x v, float32 or bfloat16).  Returns (logp, entropy, lse, top_logp,
    top_ids): logp None without targets, the last two (... x top; fp32 and int32; the
    larger first, then the lower index) None without ``top``."""
    shape, dev = logits.shape, logits.device
    logits, rows, ldl = _rows(logits, "logits", (torch.float32, torch.bfloat16))
    v, top = logits.shape[1], int(top)
    targets = _vector(targets, rows, "targets", (torch.int64,), dev)
    L = lib()
    scalars = torch.empty((3, *shape[:-1]), dtype=torch.float32, device=dev)
    logp, entropy, lse = scalars
    top_logp = torch.empty((*shape[:-1], top), dtype=torch.float32, device=dev) if top > 0 else None
    top_ids = torch.empty((*shape[:-1], top), dtype=torch.int32, device=dev) if top > 0 else None
    if targets is None:
        logp = None
    rc = L.bakron_token_logprobs(logits.data_ptr(), _DTYPES[logits.dtype], rows, v, ldl, _p(targets), top,
                                 _p(logp), entropy.data_ptr(), lse.data_ptr(), _p(top_logp), _p(top_ids),
                                 _stream(dev))
    if rc != OK:
        raise BakronError(rc, "bakron_token_logprobs")
    return logp, entropy, lse, top_logp, top_ids


@_placed
def bakron_token_logprobs_backward(logits, targets, lse, dlogp, entropy=None, dentropy=None, out=None):
    """The gradient at the logits of sum(dlogp logp + dentropy entropy), in their type;
    ``lse`` and ``entropy`` from ``bakron_token_logprobs``.  Either gradient may be None;
    ``out`` may be ``logits``."""
    shape, dev, dtype = logits.shape, logits.device, logits.dtype
    logits, rows, ldl = _rows(logits, "logits", (torch.float32, torch.bfloat16))
    v = logits.shape[1]
    f32 = (torch.float32,)
    targets = _vector(targets, rows, "targets", (torch.int64,), dev)
    lse, dlogp = _vector(lse, rows, "lse", f32, dev), _vector(dlogp, rows, "dlogp", f32, dev)
    entropy, dentropy = _vector(entropy, rows, "entropy", f32, dev), _vector(dentropy, rows, "dentropy", f32, dev)
    L = lib()
    if out is None:
        out = torch.empty(shape, dtype=dtype, device=dev)
    d, _, ldd = _like(out, shape, "out", dtype, dev)
    if d.data_ptr() != out.data_ptr():
        raise ValueError("out must have evenly spaced rows and a contiguous last dimension")
    rc = L.bakron_token_logprobs_backward(logits.data_ptr(), _DTYPES[dtype], rows, v, ldl, _p(targets),
                                          _p(lse), _p(dlogp), _p(entropy), _p(dentropy), d.data_ptr(), ldd,
                                          _stream(dev))
    if rc != OK:
        raise BakronError(rc, "bakron_token_logprobs_backward")
    return out
