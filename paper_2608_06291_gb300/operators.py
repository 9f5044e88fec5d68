"""The operators that run and score a quantised model, same names as the C ABI:
the product with a quantised weight, the root-mean-square norm and the layer norm, the log
probabilities of given tokens from logits or straight from the hidden states, and the
gradients of each (the product's at its tokens).

Results carry no autograd graph, whatever their inputs ask for: a training step calls the
``*_backward`` operators itself.

Tensors may have any number of leading dimensions where their rows are evenly
spaced (or else are copied); the last dimension is contiguous.  Work is enqueued on
``stream`` (default: the current one), and what a call allocates or copies belongs to it.
A decoding step's kernels take a few microseconds, less than a careless binding, so the
usual case (contiguous tensors, one GPU) goes through few Python operations.
"""
from __future__ import annotations

import torch

from .bakron import BF16, E4M3, F32, OK, BakronError, lib

_F32, _BF16, _E4M3 = torch.float32, torch.bfloat16, torch.float8_e4m3fn
_DTYPES = {_F32: F32, _BF16: BF16, _E4M3: E4M3}
_ACTIVATIONS = {None: 0, "none": 0, "relu": 1, "silu": 2, "gelu": 3}
_empty = torch.empty
_MOST = 2 ** 31 - 1

try:     # the stream's handle without a Stream object around it
    from torch._C import _cuda_getCurrentRawStream as _raw_stream
except ImportError:
    def _raw_stream(index):
        return torch.cuda.current_stream(index).cuda_stream


def _names(dtypes):
    return " or ".join(str(d)[6:] for d in dtypes)


def _rows(t, name, dtypes, device):
    """t as rows x d: (tensor, number of rows, row stride in elements).  device: an index."""
    if t.dtype not in dtypes:
        raise ValueError(f"{name} must be {_names(dtypes)}")
    if t.get_device() != device or device < 0:
        raise ValueError(f"{name} must be a CUDA tensor" + (f" on cuda:{device}" if device >= 0 else ""))
    d, count = t.shape[-1], t.numel()
    if count > _MOST and max(d, count // d) > _MOST:     # counts are 32-bit integers below
        raise ValueError(f"{name} must have at most 2^31 - 1 rows and columns")
    if t.is_contiguous():
        return t, count // d if d else 0, d
    t = t.reshape(-1, d)
    if t.stride(1) != 1 and d > 1 or t.shape[0] > 1 and t.stride(0) < d:
        t = t.contiguous()
    return t, t.shape[0], max(t.stride(0), d)


def _like(t, shape, name, dtype, device):
    """A tensor of the shape and type asked for, as rows."""
    if t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}")
    return _rows(t, name, (dtype,), device)


def _result(t, shape, name, dtype, device):
    r, _, ld = _like(t, shape, name, dtype, device)
    if r.data_ptr() != t.data_ptr():
        raise ValueError(f"{name} must have evenly spaced rows and a contiguous last dimension")
    return ld


def _vector(t, n, name, dtypes, device):
    if t.dtype not in dtypes or t.numel() != n or t.get_device() != device:
        raise ValueError(f"{name} must be {n} values of {_names(dtypes)} on cuda:{device}")
    return t if t.is_contiguous() else t.contiguous()


def _workspace(given, size, dev):
    """The caller's workspace, or one of `size` bytes: (tensor, bytes)."""
    if given is None:
        return _empty(size, dtype=torch.uint8, device=dev), size
    if given.get_device() != dev or not given.is_contiguous():
        raise ValueError(f"workspace must be a contiguous tensor on cuda:{dev}")
    return given, given.nbytes


_gpus = 0


def _elsewhere(t, stream):
    """Whether a call has to be made again on another stream or device: the context."""
    global _gpus
    if stream is not None:
        return torch.cuda.stream(stream)
    if not _gpus:
        _gpus = torch.cuda.device_count()
    if _gpus > 1 and t.is_cuda and t.get_device() != torch.cuda.current_device():
        return torch.cuda.device(t.get_device())
    return None


class PackedWeight:
    """A quantised m x n weight laid out for ``bakron_linear``."""

    def __init__(self, m, n, qmax, group_size, buf):
        self.m, self.n, self.qmax, self.group_size, self.buf = m, n, qmax, group_size, buf

    @property
    def device(self):
        return self.buf.device


def bakron_pack_weight(codes, scales, zeros, qmax: int, group_size: int = 0, stream=None) -> PackedWeight:
    """Lay out codes (m x n uint8, 0..qmax), scales and zeros (m x G fp32) as the solve
    leaves them: code c of row i, group g stands for s[i, g] (c - z[i, g]).  group_size 0
    or a multiple of 32.  4 bits a code up to qmax 15, else 8.  Synchronous."""
    if stream is not None or _gpus != 1:
        there = _elsewhere(codes, stream)
        if there is not None:
            with there:
                return bakron_pack_weight(codes, scales, zeros, qmax, group_size)
    if codes.dim() != 2:
        raise ValueError("codes must be m x n")
    dev = codes.get_device()
    codes, m, ldc = _rows(codes, "codes", (torch.uint8,), dev)
    n, group_size, qmax = codes.shape[1], int(group_size), int(qmax)
    G = 1 if group_size <= 0 else n // group_size
    scales = _like(scales, (m, G), "scales", _F32, dev)[0].contiguous()
    zeros = _like(zeros, (m, G), "zeros", _F32, dev)[0].contiguous()
    L = lib()
    size = L.bakron_packed_bytes(m, n, qmax, group_size)
    buf = _empty(size, dtype=torch.uint8, device=dev)
    rc = L.bakron_pack_weight(codes.data_ptr(), ldc, scales.data_ptr(), zeros.data_ptr(), m, n, qmax, group_size,
                              buf.data_ptr(), size, _raw_stream(dev))
    if rc != OK:
        raise BakronError(rc, "bakron_pack_weight")
    return PackedWeight(m, n, qmax, group_size, buf)


def bakron_linear(x, weight: PackedWeight, x_scales=None, bias=None, activation=None, residual=None,
                  out_dtype=_BF16, out=None, workspace=None, sync: bool = False, stream=None):
    """act(x What^T + bias) + residual for the tokens x (... x n, bfloat16 or
    float8_e4m3fn with ``x_scales``, one fp32 a token).  ``activation``: None, "relu",
    "silu" or "gelu".  ``bias``: m fp32; ``residual`` and the result (... x m): ``out_dtype``,
    bfloat16 or float32.  ``out`` may be ``residual``.  ``sync``: wait, and raise what the
    device reports (``bakron_read_status(workspace)`` tells it later)."""
    if stream is not None or _gpus != 1:
        there = _elsewhere(x, stream)
        if there is not None:
            with there:
                return bakron_linear(x, weight, x_scales, bias, activation, residual, out_dtype, out, workspace, sync)
    m, n, dev = weight.m, weight.n, weight.buf.get_device()
    shape = x.shape
    x, rows, ldx = _rows(x, "x", (_BF16, _E4M3), dev)
    if shape[-1] != n:
        raise ValueError(f"x must have {n} columns")
    act = _ACTIVATIONS.get(activation)
    if act is None:
        raise ValueError(f"activation must be one of {[a for a in _ACTIVATIONS if a]} or None")
    if out is not None:
        out_dtype = out.dtype
    if out_dtype is not _BF16 and out_dtype is not _F32:
        raise ValueError("the result must be bfloat16 or float32")
    yshape = shape[:-1] + (m,)
    xs = b = r = ws = None
    ldr = size = 0
    if x_scales is not None:
        x_scales = _vector(x_scales, rows, "x_scales", (_F32,), dev)
        xs = x_scales.data_ptr()
    if bias is not None:
        bias = _vector(bias, m, "bias", (_F32,), dev)
        b = bias.data_ptr()
    if residual is not None:
        residual, _, ldr = _like(residual, yshape, "residual", out_dtype, dev)
        r = residual.data_ptr()
    if out is None:
        out, ldy = _empty(yshape, dtype=out_dtype, device=dev), m
    else:
        ldy = _result(out, yshape, "out", out_dtype, dev)
    L = lib()
    px, dt = x.data_ptr(), _DTYPES[x.dtype]
    if workspace is not None:
        if workspace.get_device() != dev or not workspace.is_contiguous():
            raise ValueError(f"workspace must be a contiguous tensor on cuda:{dev}")
    else:
        size = L.bakron_linear_workspace_bytes(px, dt, rows, ldx, n, weight.qmax, weight.group_size)
        if size:
            workspace = _empty(size, dtype=torch.uint8, device=dev)
    if workspace is not None:
        ws, size = workspace.data_ptr(), workspace.nbytes
    rc = L.bakron_linear(px, dt, rows, ldx, xs, weight.buf.data_ptr(), m, n, weight.qmax, weight.group_size, b, act, r,
                         ldr, out.data_ptr(), _DTYPES[out_dtype], ldy, ws, size, 1 if sync else 0,
                         _raw_stream(dev))
    if rc != OK:
        raise BakronError(rc, "bakron_linear")
    return out


def bakron_linear_backward(dy, weight: PackedWeight, out=None, workspace=None, sync: bool = False, stream=None):
    """dx = dy What, the gradient of ``bakron_linear``'s product at its tokens: dy (... x m,
    bfloat16) is the gradient at x What^T, before bias, activation and residual.  Returns
    dx (... x n, bfloat16).  ``sync``: wait, and raise what the device reports
    (``bakron_read_status(workspace)`` tells it later)."""
    if stream is not None or _gpus != 1:
        there = _elsewhere(dy, stream)
        if there is not None:
            with there:
                return bakron_linear_backward(dy, weight, out, workspace, sync)
    m, n, dev = weight.m, weight.n, weight.buf.get_device()
    shape = dy.shape
    dy, rows, lddy = _rows(dy, "dy", (_BF16,), dev)
    if shape[-1] != m:
        raise ValueError(f"dy must have {m} columns")
    xshape = shape[:-1] + (n,)
    if out is None:
        out, ldx = _empty(xshape, dtype=_BF16, device=dev), n
    else:
        ldx = _result(out, xshape, "out", _BF16, dev)
    L = lib()
    py = dy.data_ptr()
    size = L.bakron_linear_backward_workspace_bytes(py, rows, lddy, m, n, weight.qmax, weight.group_size)
    ws, size = _workspace(workspace, size, dev)
    rc = L.bakron_linear_backward(py, rows, lddy, weight.buf.data_ptr(), m, n, weight.qmax, weight.group_size,
                                  out.data_ptr(), ldx, ws.data_ptr(), size, 1 if sync else 0, _raw_stream(dev))
    if rc != OK:
        raise BakronError(rc, "bakron_linear_backward")
    return out


def bakron_rmsnorm(x, weight, eps: float = 1e-6, residual=None, out_dtype=None, stream=None):
    """h = x + residual, y = weight h / sqrt(mean(h^2) + eps) over the last dimension.
    Returns (y, scales, h): y of ``out_dtype`` (default x's; or float8_e4m3fn with
    ``scales``, one fp32 a row, else None), h of x's type (None without a residual)."""
    if stream is not None or _gpus != 1:
        there = _elsewhere(x, stream)
        if there is not None:
            with there:
                return bakron_rmsnorm(x, weight, eps, residual, out_dtype)
    shape, dev, dtype = x.shape, x.get_device(), x.dtype
    x, rows, ldx = _rows(x, "x", (_F32, _BF16), dev)
    d = shape[-1]
    weight = _vector(weight, d, "weight", (_F32, _BF16), dev)
    if out_dtype is None:
        out_dtype = dtype
    elif out_dtype is not dtype and out_dtype is not _E4M3:
        raise ValueError("out_dtype must be x's or float8_e4m3fn")
    y = _empty(shape, dtype=out_dtype, device=dev)
    scales = h = s = ph = r = None
    ldr = 0
    if residual is not None:
        residual, _, ldr = _like(residual, shape, "residual", dtype, dev)
        h = _empty(shape, dtype=dtype, device=dev)
        ph, r = h.data_ptr(), residual.data_ptr()
    if out_dtype is _E4M3:
        scales = _empty(shape[:-1], dtype=_F32, device=dev)
        s = scales.data_ptr()
    rc = lib().bakron_rmsnorm(x.data_ptr(), _DTYPES[dtype], rows, d, ldx, r, ldr, weight.data_ptr(),
                              _DTYPES[weight.dtype], eps, ph, d, y.data_ptr(), _DTYPES[out_dtype], d, s,
                              _raw_stream(dev))
    if rc != OK:
        raise BakronError(rc, "bakron_rmsnorm")
    return y, scales, h


def bakron_rmsnorm_backward(dy, h, weight, eps: float = 1e-6, dsum=None, stream=None):
    """Gradients of y = weight h / sqrt(mean(h^2) + eps), given dy and the gradient ``dsum``
    that reaches h past the norm.  Returns (dx of h's type, dweight fp32)."""
    if stream is not None or _gpus != 1:
        there = _elsewhere(dy, stream)
        if there is not None:
            with there:
                return bakron_rmsnorm_backward(dy, h, weight, eps, dsum)
    shape, dev, dtype = h.shape, h.get_device(), h.dtype
    h, rows, ldh = _rows(h, "h", (_F32, _BF16), dev)
    d = shape[-1]
    dy, _, lddy = _like(dy, shape, "dy", dtype, dev)
    weight = _vector(weight, d, "weight", (_F32, _BF16), dev)
    ps, ldds = None, 0
    if dsum is not None:
        dsum, _, ldds = _like(dsum, shape, "dsum", dtype, dev)
        ps = dsum.data_ptr()
    L = lib()
    dx = _empty(shape, dtype=dtype, device=dev)
    dw = _empty(d, dtype=_F32, device=dev)
    size = L.bakron_rmsnorm_backward_workspace_bytes(rows, d)
    ws = _empty(size, dtype=torch.uint8, device=dev)
    rc = L.bakron_rmsnorm_backward(dy.data_ptr(), lddy, h.data_ptr(), ldh, _DTYPES[dtype], rows, d,
                                   weight.data_ptr(), _DTYPES[weight.dtype], eps, ps, ldds, dx.data_ptr(), d,
                                   dw.data_ptr(), ws.data_ptr(), size, _raw_stream(dev))
    if rc != OK:
        raise BakronError(rc, "bakron_rmsnorm_backward")
    return dx, dw


def bakron_layernorm(x, weight, bias=None, eps: float = 1e-5, residual=None, out_dtype=None, stream=None):
    """h = x + residual, y = weight (h - mean(h)) / sqrt(var(h) + eps) + bias over the last
    dimension.  Returns (y, scales, h) as ``bakron_rmsnorm`` does."""
    if stream is not None or _gpus != 1:
        there = _elsewhere(x, stream)
        if there is not None:
            with there:
                return bakron_layernorm(x, weight, bias, eps, residual, out_dtype)
    shape, dev, dtype = x.shape, x.get_device(), x.dtype
    x, rows, ldx = _rows(x, "x", (_F32, _BF16), dev)
    d = shape[-1]
    weight = _vector(weight, d, "weight", (_F32, _BF16), dev)
    if out_dtype is None:
        out_dtype = dtype
    elif out_dtype is not dtype and out_dtype is not _E4M3:
        raise ValueError("out_dtype must be x's or float8_e4m3fn")
    y = _empty(shape, dtype=out_dtype, device=dev)
    scales = h = s = ph = r = b = None
    ldr = bt = 0
    if bias is not None:
        bias = _vector(bias, d, "bias", (_F32, _BF16), dev)
        b, bt = bias.data_ptr(), _DTYPES[bias.dtype]
    if residual is not None:
        residual, _, ldr = _like(residual, shape, "residual", dtype, dev)
        h = _empty(shape, dtype=dtype, device=dev)
        ph, r = h.data_ptr(), residual.data_ptr()
    if out_dtype is _E4M3:
        scales = _empty(shape[:-1], dtype=_F32, device=dev)
        s = scales.data_ptr()
    rc = lib().bakron_layernorm(x.data_ptr(), _DTYPES[dtype], rows, d, ldx, r, ldr, weight.data_ptr(),
                                _DTYPES[weight.dtype], b, bt, eps, ph, d, y.data_ptr(), _DTYPES[out_dtype], d, s,
                                _raw_stream(dev))
    if rc != OK:
        raise BakronError(rc, "bakron_layernorm")
    return y, scales, h


def bakron_layernorm_backward(dy, h, weight, eps: float = 1e-5, dsum=None, stream=None):
    """Gradients of y = weight (h - mean(h)) / sqrt(var(h) + eps) + bias, given dy and the
    gradient ``dsum`` that reaches h past the norm.  Returns (dx of h's type, dweight fp32,
    dbias fp32)."""
    if stream is not None or _gpus != 1:
        there = _elsewhere(dy, stream)
        if there is not None:
            with there:
                return bakron_layernorm_backward(dy, h, weight, eps, dsum)
    shape, dev, dtype = h.shape, h.get_device(), h.dtype
    h, rows, ldh = _rows(h, "h", (_F32, _BF16), dev)
    d = shape[-1]
    dy, _, lddy = _like(dy, shape, "dy", dtype, dev)
    weight = _vector(weight, d, "weight", (_F32, _BF16), dev)
    ps, ldds = None, 0
    if dsum is not None:
        dsum, _, ldds = _like(dsum, shape, "dsum", dtype, dev)
        ps = dsum.data_ptr()
    L = lib()
    dx = _empty(shape, dtype=dtype, device=dev)
    dw, db = _empty(d, dtype=_F32, device=dev), _empty(d, dtype=_F32, device=dev)
    size = L.bakron_layernorm_backward_workspace_bytes(rows, d)
    ws = _empty(size, dtype=torch.uint8, device=dev)
    rc = L.bakron_layernorm_backward(dy.data_ptr(), lddy, h.data_ptr(), ldh, _DTYPES[dtype], rows, d,
                                     weight.data_ptr(), _DTYPES[weight.dtype], eps, ps, ldds, dx.data_ptr(), d,
                                     dw.data_ptr(), db.data_ptr(), ws.data_ptr(), size, _raw_stream(dev))
    if rc != OK:
        raise BakronError(rc, "bakron_layernorm_backward")
    return dx, dw, db


def bakron_token_logprobs(logits, targets=None, top: int = 0, stream=None):
    """Log probabilities of the tokens ``targets`` (int64; outside 0..v-1: not scored, 0)
    under logits (... x v, float32 or bfloat16).  Returns (logp, entropy, lse, top_logp,
    top_ids): logp None without targets, the last two (... x top; fp32 and int32; the
    larger first, then the lower index) None without ``top``."""
    if stream is not None or _gpus != 1:
        there = _elsewhere(logits, stream)
        if there is not None:
            with there:
                return bakron_token_logprobs(logits, targets, top)
    shape, dev = logits.shape, logits.get_device()
    logits, rows, ldl = _rows(logits, "logits", (_F32, _BF16), dev)
    lead = shape[:-1]
    t = pl = logp = top_logp = top_ids = pv = pi = None
    if targets is not None:
        targets = _vector(targets, rows, "targets", (torch.int64,), dev)
        logp = _empty(lead, dtype=_F32, device=dev)
        t, pl = targets.data_ptr(), logp.data_ptr()
    entropy, lse = _empty(lead, dtype=_F32, device=dev), _empty(lead, dtype=_F32, device=dev)
    if top > 0:
        top_logp = _empty(lead + (top,), dtype=_F32, device=dev)
        top_ids = _empty(lead + (top,), dtype=torch.int32, device=dev)
        pv, pi = top_logp.data_ptr(), top_ids.data_ptr()
    rc = lib().bakron_token_logprobs(logits.data_ptr(), _DTYPES[logits.dtype], rows, shape[-1], ldl, t, top, pl,
                                     entropy.data_ptr(), lse.data_ptr(), pv, pi, _raw_stream(dev))
    if rc != OK:
        raise BakronError(rc, "bakron_token_logprobs")
    return logp, entropy, lse, top_logp, top_ids


def bakron_token_logprobs_backward(logits, targets, lse, dlogp, entropy=None, dentropy=None, out=None, stream=None):
    """The gradient at the logits of sum(dlogp logp + dentropy entropy), in their type;
    ``lse`` and ``entropy`` from ``bakron_token_logprobs``.  Either gradient may be None;
    ``out`` may be ``logits``."""
    if stream is not None or _gpus != 1:
        there = _elsewhere(logits, stream)
        if there is not None:
            with there:
                return bakron_token_logprobs_backward(logits, targets, lse, dlogp, entropy, dentropy, out)
    shape, dev, dtype = logits.shape, logits.get_device(), logits.dtype
    logits, rows, ldl = _rows(logits, "logits", (_F32, _BF16), dev)
    v, f32 = shape[-1], (_F32,)
    t = g = e = u = None
    if targets is not None:
        targets = _vector(targets, rows, "targets", (torch.int64,), dev)
        t = targets.data_ptr()
    lse = _vector(lse, rows, "lse", f32, dev)
    if dlogp is not None:
        dlogp = _vector(dlogp, rows, "dlogp", f32, dev)
        g = dlogp.data_ptr()
    if entropy is not None:
        entropy = _vector(entropy, rows, "entropy", f32, dev)
        e = entropy.data_ptr()
    if dentropy is not None:
        dentropy = _vector(dentropy, rows, "dentropy", f32, dev)
        u = dentropy.data_ptr()
    if out is None:
        out, ldd = _empty(shape, dtype=dtype, device=dev), v
    else:
        ldd = _result(out, shape, "out", dtype, dev)
    rc = lib().bakron_token_logprobs_backward(logits.data_ptr(), _DTYPES[dtype], rows, v, ldl, t, lse.data_ptr(), g,
                                              e, u, out.data_ptr(), ldd, _raw_stream(dev))
    if rc != OK:
        raise BakronError(rc, "bakron_token_logprobs_backward")
    return out


def _matrix(t, n, name, dev):
    """A bf16 matrix of n columns: (tensor, rows, row stride)."""
    if t.dim() != 2 or t.shape[1] != n:
        raise ValueError(f"{name} must be a matrix of {n} columns")
    return _rows(t, name, (_BF16,), dev)


def bakron_head_logprobs(h, weight, targets=None, sync: bool = False, workspace=None, stream=None):
    """``bakron_token_logprobs`` of the logits h weight^T, which are not kept: h (... x d) and
    weight (v x d) bfloat16, ``targets`` int64 (outside 0..v-1: not scored, 0).  Returns
    (logp, entropy, lse), fp32; logp None without targets.  ``sync``: wait, and raise what
    the device reports (``bakron_read_status(workspace)`` tells it later)."""
    if stream is not None or _gpus != 1:
        there = _elsewhere(h, stream)
        if there is not None:
            with there:
                return bakron_head_logprobs(h, weight, targets, sync, workspace)
    shape, dev = h.shape, h.get_device()
    h, rows, ldh = _rows(h, "h", (_BF16,), dev)
    lead, d = shape[:-1], shape[-1]
    weight, v, ldw = _matrix(weight, d, "weight", dev)
    t = pl = logp = None
    if targets is not None:
        targets = _vector(targets, rows, "targets", (torch.int64,), dev)
        logp = _empty(lead, dtype=_F32, device=dev)
        t, pl = targets.data_ptr(), logp.data_ptr()
    entropy, lse = _empty(lead, dtype=_F32, device=dev), _empty(lead, dtype=_F32, device=dev)
    L = lib()
    ph, pw = h.data_ptr(), weight.data_ptr()
    size = L.bakron_head_logprobs_workspace_bytes(ph, ldh, pw, ldw, rows, v, d)
    ws, size = _workspace(workspace, size, dev)
    rc = L.bakron_head_logprobs(ph, ldh, pw, ldw, rows, v, d, t, pl, entropy.data_ptr(), lse.data_ptr(),
                                ws.data_ptr(), size, 1 if sync else 0, _raw_stream(dev))
    if rc != OK:
        raise BakronError(rc, "bakron_head_logprobs")
    return logp, entropy, lse


def bakron_head_logprobs_backward(h, weight, targets, lse, dlogp, entropy=None, dentropy=None,
                                  weight_grad: bool = True, sync: bool = False, workspace=None, stream=None):
    """The gradients of sum(dlogp logp + dentropy entropy) at h and at the weight, bfloat16;
    ``lse`` and ``entropy`` from ``bakron_head_logprobs``.  Either gradient may be None.
    Returns (dh, dweight), dweight None without ``weight_grad``."""
    if stream is not None or _gpus != 1:
        there = _elsewhere(h, stream)
        if there is not None:
            with there:
                return bakron_head_logprobs_backward(h, weight, targets, lse, dlogp, entropy, dentropy, weight_grad,
                                                     sync, workspace)
    shape, dev, f32 = h.shape, h.get_device(), (_F32,)
    h, rows, ldh = _rows(h, "h", (_BF16,), dev)
    d = shape[-1]
    weight, v, ldw = _matrix(weight, d, "weight", dev)
    t = g = e = u = pdw = None
    if targets is not None:
        targets = _vector(targets, rows, "targets", (torch.int64,), dev)
        t = targets.data_ptr()
    lse = _vector(lse, rows, "lse", f32, dev)
    if dlogp is not None:
        dlogp = _vector(dlogp, rows, "dlogp", f32, dev)
        g = dlogp.data_ptr()
    if entropy is not None:
        entropy = _vector(entropy, rows, "entropy", f32, dev)
        e = entropy.data_ptr()
    if dentropy is not None:
        dentropy = _vector(dentropy, rows, "dentropy", f32, dev)
        u = dentropy.data_ptr()
    dh, dweight = _empty(shape, dtype=_BF16, device=dev), None
    if weight_grad:
        dweight = _empty((v, d), dtype=_BF16, device=dev)
        pdw = dweight.data_ptr()
    L = lib()
    ph, pw = h.data_ptr(), weight.data_ptr()
    size = L.bakron_head_logprobs_backward_workspace_bytes(ph, ldh, pw, ldw, rows, v, d, 1 if weight_grad else 0)
    ws, size = _workspace(workspace, size, dev)
    rc = L.bakron_head_logprobs_backward(ph, ldh, pw, ldw, rows, v, d, t, lse.data_ptr(), g, e, u, dh.data_ptr(), d,
                                         pdw, d, ws.data_ptr(), size, 1 if sync else 0, _raw_stream(dev))
    if rc != OK:
        raise BakronError(rc, "bakron_head_logprobs_backward")
    return dh, dweight
