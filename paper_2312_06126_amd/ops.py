"""The operators of a recurrent residual block on torch tensors (spz_scan_* .. spz_quant_* of
include/spz.h): argument checks, outputs and workspaces; every step runs in the HIP library.

Tensors are on one GPU; float32 or bfloat16 as the header says, states, scales and parameter vectors
float32. The last dimension is contiguous, the others have any strides. `stream`: a
torch.cuda.Stream or a hipStream_t address (default: the device's current stream); the call is
enqueued on it, and where `stream` is given tensors that belong to another one are kept alive until it has run; what
was enqueued elsewhere is the caller's to order. Nothing waits for the GPU, so calls may be
captured into a HIP graph. Errors: SpzError.

torch's autograd does not record the calls: gradients come from scan_backward, block_norm_backward and, for dropout,
the same call on the gradient (quant_linear has none). Tensors that require a gradient are refused, so that none is
lost; within torch.no_grad() they are taken. The calls work on data pointers: they are not for tracing or vmap.
"""
from __future__ import annotations

import ctypes
import functools
import struct
from typing import NamedTuple, Optional

import torch

from .spz import GATES, NORMS, SPZ_EINVAL, SPZ_OK, SpzError, load, pack_block_norm, pack_scan

_PREC = {torch.float32: 0, torch.bfloat16: 1}
_F32 = torch.float32
_NULL = 0


def _refuse(msg: str):
    raise SpzError(SPZ_EINVAL, msg)


def _done(rc: int):
    if rc != SPZ_OK:
        raise SpzError(rc, load().spz_last_error(None).decode())


def _size(n: int) -> int:
    if n < 0:
        raise SpzError(n, load().spz_last_error(None).decode())
    return n


def _ptr(t: Optional[torch.Tensor]) -> int:
    return _NULL if t is None else t.data_ptr()


_grad_on = torch.is_grad_enabled


def _refuse_grad(name: str):
    _refuse("%s requires a gradient, which autograd would not record here: call within torch.no_grad() or detach it" % name)


def _like(t, name: str, gpu: int, shape, dtype, contiguous: bool = False):
    """Checks an argument's device, shape, type and layout (None passes)."""
    if t is None:
        return
    if not isinstance(t, torch.Tensor):
        _refuse("%s is no tensor" % name)
    if t.get_device() != gpu:
        _refuse("%s is on %s, not on cuda:%d" % (name, t.device, gpu))
    if t.shape != shape:
        _refuse("%s has shape %s, not %s" % (name, tuple(t.shape), tuple(shape)))
    if t.dtype is not dtype:
        _refuse("%s has type %s, not %s" % (name, t.dtype, dtype))
    if t.requires_grad and _grad_on():
        _refuse_grad(name)
    if t.is_contiguous():
        return
    if contiguous:
        _refuse("%s is not contiguous" % name)
    if shape[-1] > 1 and t.stride(-1) != 1:
        _refuse("%s is not contiguous in its last dimension" % name)


def _flags_2d(t, name: str, gpu: int, shape):
    """A uint8 or bool argument with any strides (torch keeps either as bytes)."""
    if not isinstance(t, torch.Tensor) or t.get_device() != gpu or t.shape != shape or t.dtype not in (torch.uint8, torch.bool):
        _refuse("%s is no uint8 or bool tensor %s on cuda:%d" % (name, tuple(shape), gpu))


def _operand(t, name: str, dims: int) -> int:
    """The leading operand, a GPU tensor in one of the two precisions; returns its device's ordinal."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        _refuse("%s is no GPU tensor" % name)
    if t.dtype not in _PREC:
        _refuse("%s has type %s" % (name, t.dtype))
    if t.dim() != dims:
        _refuse("%s has %d dimensions, not %d" % (name, t.dim(), dims))
    if t.requires_grad and _grad_on():
        _refuse_grad(name)
    if not t.is_contiguous() and t.shape[-1] > 1 and t.stride(-1) != 1:
        _refuse("%s is not contiguous in its last dimension" % name)
    return t.get_device()


_device = torch._C._cuda_getDevice
_stream = torch._C._cuda_getCurrentRawStream


def _elsewhere(stream, gpu: int, tensors, call):
    """call() with the tensors' device and the given stream current, so that what it allocates belongs to
    that stream; the tensors stay alive until the stream has run."""
    if stream is None:
        with torch.cuda.device(gpu):
            return call()
    if isinstance(stream, int):
        stream = torch.cuda.ExternalStream(stream, device=gpu) if stream else torch.cuda.default_stream(gpu)
    elif stream.device.index != gpu:
        _refuse("the stream is on %s, the tensors are on cuda:%d" % (stream.device, gpu))
    with torch.cuda.stream(stream):
        out = call()
    for t in tensors:
        if t is not None:
            t.record_stream(stream)
    return out


def _empty(x: torch.Tensor) -> torch.Tensor:
    return torch.empty_like(x) if x.is_contiguous() else x.new_empty(x.shape)


def _workspace(n: int, ref: torch.Tensor) -> Optional[torch.Tensor]:
    return ref.new_empty((n,), dtype=torch.uint8) if n else None


# ----------------------------------------------------------------------------- scan

@functools.lru_cache(maxsize=4096)
def _scan_sizes(B: int, T: int, D: int, prec: int):
    """Floats of `saved` and bytes of the workspaces, forward and backward: functions of the sizes alone."""
    lib = load()
    a = pack_scan(B, T, D, *([0] * 27), prec)
    return _size(lib.spz_scan_saved(a)), _size(lib.spz_scan_workspace(a, 0)), _size(lib.spz_scan_workspace(a, 1))


def _scan_check(f, v, h0, reset, lengths) -> int:
    gpu = _operand(f, "f", 3)
    B, T, D = shape = f.shape
    _like(v, "v", gpu, shape, f.dtype)
    if v is None:
        _refuse("v is missing")
    _like(h0, "h0", gpu, (B, D), _F32, contiguous=True)
    _like(lengths, "lengths", gpu, (B,), torch.int32, contiguous=True)
    if reset is not None:
        _flags_2d(reset, "reset", gpu, (B, T))
    return gpu


def _outer(t):
    """Strides of the batch and time dimensions (no tensor: 0)."""
    return (0, 0) if t is None else t.stride()[:2]


def _sequences(f: torch.Tensor) -> torch.Tensor:
    """An empty [batch, steps, width] tensor with the outer dimensions in the order of f's."""
    B, T, D = f.shape
    s = f.stride()
    if s[0] < s[1] and B > 1:
        return f.new_empty((T, B, D)).transpose(0, 1)
    return f.new_empty((B, T, D))


def scan(f, v, h0=None, *, reset=None, lengths=None, save: bool = False, out=None, hT=None, stream=None):
    """Gated linear recurrence: a = sigmoid(f), h_t = a_t h_{t-1} + (1 - a_t) v_t over [batch, steps,
    width] -> (y, hT), or (y, hT, saved) with save=True, for scan_backward.

    h0, hT: float32 [batch, width], the state in front (default zeros) and behind; pass hT=h0 to update
    a state in place. reset [batch, steps] (uint8 or bool): steps that start an episode, cut off from
    the state before. lengths [batch] (int32): steps of each sequence; y is 0 behind it. `out`: y."""
    lib = load()
    gpu = _scan_check(f, v, h0, reset, lengths)
    B, T, D = f.shape
    prec = _PREC[f.dtype]
    _like(out, "out", gpu, f.shape, f.dtype)
    _like(hT, "hT", gpu, (B, D), _F32, contiguous=True)
    n_saved, n, _ = _scan_sizes(B, T, D, prec)

    if stream is not None or gpu != _device():
        return _elsewhere(stream, gpu, (f, v, h0, reset, lengths, out, hT),
                          lambda: scan(f, v, h0, reset=reset, lengths=lengths, save=save, out=out, hT=hT))
    s = _stream(gpu)
    y = out if out is not None else _sequences(f)
    last = hT if hT is not None else torch.empty_like(h0) if h0 is not None else f.new_empty((B, D), dtype=_F32)
    saved = f.new_empty((n_saved,), dtype=_F32) if save else None
    ws = _workspace(n, f)
    a = pack_scan(B, T, D, f.data_ptr(), v.data_ptr(), *_outer(f), *_outer(v), _ptr(reset), *_outer(reset), _ptr(lengths),
                  _ptr(h0), y.data_ptr(), *_outer(y), last.data_ptr(), _ptr(saved), 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, prec)
    rc = lib.spz_scan_forward(a, _ptr(ws), n, s)
    if rc:
        _done(rc)
    return (y, last, saved) if save else (y, last)


def scan_backward(f, v, dy, saved, *, dhT=None, reset=None, lengths=None, out=None, stream=None):
    """Gradients (df, dv, dh0) of scan's (y, hT) from dy (None: zeros) and dhT (None: zeros), with the
    `saved` of the forward call. `out`: the tensors (df, dv) to write, e.g. two parts of one."""
    lib = load()
    gpu = _scan_check(f, v, None, reset, lengths)
    B, T, D = f.shape
    prec = _PREC[f.dtype]
    n_saved, _, n = _scan_sizes(B, T, D, prec)
    _like(dy, "dy", gpu, f.shape, f.dtype)
    _like(dhT, "dhT", gpu, (B, D), _F32, contiguous=True)
    if saved is None:
        _refuse("saved is missing: scan(..., save=True) makes it")
    _like(saved, "saved", gpu, (n_saved,), _F32, contiguous=True)
    if out is not None:
        if len(out) != 2 or out[0] is None or out[1] is None:
            _refuse("out holds df and dv")
        for name, t in zip(("df", "dv"), out):
            _like(t, name, gpu, f.shape, f.dtype)

    if stream is not None or gpu != _device():
        return _elsewhere(stream, gpu, (f, v, dy, saved, dhT, reset, lengths) + tuple(out or ()),
                          lambda: scan_backward(f, v, dy, saved, dhT=dhT, reset=reset, lengths=lengths, out=out))
    s = _stream(gpu)
    df, dv = out if out is not None else (_sequences(f), _sequences(f))
    dh0 = f.new_empty((B, D), dtype=_F32)
    ws = _workspace(n, f)
    a = pack_scan(B, T, D, f.data_ptr(), v.data_ptr(), *_outer(f), *_outer(v), _ptr(reset), *_outer(reset), _ptr(lengths),
                  0, 0, 0, 0, 0, saved.data_ptr(), _ptr(dy), *_outer(dy), _ptr(dhT), df.data_ptr(), dv.data_ptr(),
                  *_outer(df), *_outer(dv), dh0.data_ptr(), prec)
    _done(lib.spz_scan_backward(a, _ptr(ws), n, s))
    return df, dv, dh0


# ----------------------------------------------------------------------------- block norm

def _block_check(x, h, z, vectors, post, pre, gate, valid) -> int:
    gpu = _operand(x, "x", 2)
    R, D = shape = x.shape
    if post not in NORMS or pre not in NORMS:
        _refuse("norms are %s" % ", ".join(NORMS))
    if gate not in GATES:
        _refuse("gates are %s" % ", ".join(GATES))
    _like(h, "h", gpu, shape, x.dtype)
    if gate != "none" and h is not None and z is None:
        _refuse("the gate needs z")
    _like(z, "z", gpu, shape, x.dtype)
    for i, t in enumerate(vectors):
        if t is not None and not (isinstance(t, torch.Tensor) and t.dtype is _F32 and t.dim() == 1 and t.numel() == D
                                  and t.get_device() == gpu and t.is_contiguous() and not t.requires_grad):
            _like(t, ("w_post", "b_post", "scale", "w_pre", "b_pre")[i], gpu, (D,), _F32)
    if valid is not None:
        _like(valid, "valid", gpu, (R,), torch.bool if getattr(valid, "dtype", None) is torch.bool else torch.uint8, contiguous=True)
    return gpu


def _row(t) -> int:
    return 0 if t is None else t.stride(0)


_NOT_NUMBERS = (struct.error, ctypes.ArgumentError, TypeError, ValueError, OverflowError)


def _block_pack(x, h, z, vectors, valid, outs, backs, drop, eps, post, pre, gate) -> bytes:
    """The argument block; outs: x_out, u, backs: dx_out, du, then the gradients."""
    x_out, u = outs
    dx_out, du, dx, dh, dz, dw_post, db_post, dscale, dw_pre, db_pre = backs
    try:
        p, seed, step, tensor = drop if drop is not None else (0.0, 0, 0, 0)
        return pack_block_norm(
            x.shape[0], x.shape[1], x.data_ptr(), _ptr(h), _ptr(z), x.stride(0), _row(h), _row(z), *map(_ptr, vectors), _ptr(valid),
            _ptr(x_out), _ptr(u), _row(x_out), _row(u), _ptr(dx_out), _ptr(du), _row(dx_out), _row(du), _ptr(dx), _ptr(dh),
            _ptr(dz), _row(dx), _row(dh), _row(dz), _ptr(dw_post), _ptr(db_post), _ptr(dscale), _ptr(dw_pre), _ptr(db_pre),
            int(seed) & 0xFFFFFFFFFFFFFFFF, int(step) & 0xFFFFFFFF, int(tensor) & 0xFFFFFFFF, p, eps, NORMS[post], NORMS[pre],
            GATES[gate], _PREC[x.dtype])
    except _NOT_NUMBERS as e:
        _refuse("drop is not (p, seed, step, tensor) or eps no number: %s" % e)


def block_norm(x, h=None, z=None, w_post=None, b_post=None, scale=None, w_pre=None, b_pre=None, *, post="rms", pre="rms",
               gate="none", eps=1e-6, drop=None, valid=None, stream=None):
    """x' = x + scale * dropout(gate(z) * (post(h) * w_post + b_post)), u = pre(x') * w_pre + b_pre, over
    rows [rows, width] -> (x', u); u is None with pre="none". Without h: x' is x (the first block's
    norm). Norms "none", "rms", "layer"; gates "none", "sigmoid", "silu". drop: (p, seed, step, tensor) as
    dropout takes them. Rows with valid == 0 (uint8 or bool) are not read, their outputs are zero."""
    lib = load()
    vectors = (w_post, b_post, scale, w_pre, b_pre)
    gpu = _block_check(x, h, z, vectors, post, pre, gate, valid)

    if stream is not None or gpu != _device():
        return _elsewhere(stream, gpu, (x, h, z, *vectors, valid),
                          lambda: block_norm(x, h, z,
                              w_post, b_post, scale, w_pre, b_pre, post=post, pre=pre, gate=gate, eps=eps,
                              drop=drop, valid=valid))
    s = _stream(gpu)
    x_out = _empty(x) if h is not None else None
    u = _empty(x) if pre != "none" else None
    a = _block_pack(x, h, z, vectors, valid, (x_out, u), (None,) * 10, drop, eps, post, pre, gate)
    rc = lib.spz_block_norm_forward(a, s)
    if rc:
        _done(rc)
    return (x if h is None else x_out), u


def block_norm_backward(dx_out, du, x, h=None, z=None, w_post=None, b_post=None, scale=None, w_pre=None, b_pre=None, *,
                        post="rms", pre="rms", gate="none", eps=1e-6, drop=None, valid=None, stream=None):
    """Gradients of block_norm from those of x' and u (None: zeros): a dict of dx, dh, dz and, for the
    vectors that were given, dw_post, dscale, dw_pre, db_post, db_pre (float32, summed over rows)."""
    lib = load()
    vectors = (w_post, b_post, scale, w_pre, b_pre)
    gpu = _block_check(x, h, z, vectors, post, pre, gate, valid)
    _like(dx_out, "dx_out", gpu, x.shape, x.dtype)
    _like(du, "du", gpu, x.shape, x.dtype)

    if stream is not None or gpu != _device():
        return _elsewhere(stream, gpu, (x, dx_out, du, h, z, *vectors, valid),
                          lambda: block_norm_backward(dx_out, du, x, h, z,
                              w_post, b_post, scale, w_pre, b_pre, post=post, pre=pre, gate=gate, eps=eps,
                              drop=drop, valid=valid))
    s = _stream(gpu)
    g = {"dx": _empty(x), "dh": None if h is None else _empty(x),
         "dz": _empty(x) if h is not None and gate != "none" else None}
    wanted = (("dw_post", w_post), ("dscale", scale), ("dw_pre", w_pre), ("db_post", b_post), ("db_pre", b_pre))
    sums = iter(x.new_empty((sum(t is not None for _, t in wanted), x.shape[1]), dtype=_F32).unbind(0))
    for k, t in wanted:
        g[k] = None if t is None else next(sums)
    a = _block_pack(x, h, z, vectors, valid, (None, None),
                    (dx_out, du, g["dx"], g["dh"], g["dz"], g["dw_post"], g["db_post"], g["dscale"], g["dw_pre"], g["db_pre"]),
                    drop, eps, post, pre, gate)
    n = _size(lib.spz_block_norm_workspace(a))
    ws = _workspace(n, x)
    _done(lib.spz_block_norm_backward(a, _ptr(ws), n, s))
    return g


def dropout(x, p: float, seed: int, step: int, tensor: int = 0, *, out=None, stream=None):
    """x [rows, width] with elements dropped with probability p, the others scaled up. The mask is a
    function of (seed, step, tensor) and the element's index, so the same call on the gradient is
    the backward pass. `out` may be x."""
    lib = load()
    gpu = _operand(x, "x", 2)
    _like(out, "out", gpu, x.shape, x.dtype)

    if stream is not None or gpu != _device():
        return _elsewhere(stream, gpu, (x, out), lambda: dropout(x, p, seed, step, tensor, out=out))
    s = _stream(gpu)
    rows, width = x.shape
    y = out if out is not None else _empty(x)
    try:
        rc = lib.spz_dropout(_PREC[x.dtype], rows, width, x.data_ptr(), x.stride(0), y.data_ptr(), y.stride(0), p,
                             int(seed) & 0xFFFFFFFFFFFFFFFF, int(step) & 0xFFFFFFFF, int(tensor) & 0xFFFFFFFF, s)
    except _NOT_NUMBERS as e:
        _refuse("p, seed, step or tensor is no number: %s" % e)
    if rc:
        _done(rc)
    return y


# ----------------------------------------------------------------------------- 8-bit product

class QuantWeights(NamedTuple):
    """Weights of quant_linear: the integers in the product's order and a scale for each channel."""
    image: torch.Tensor
    scale: torch.Tensor
    outer: int
    inner: int


@functools.lru_cache(maxsize=4096)
def _quant_sizes(prec: int, rows: int, outer: int, inner: int):
    """Bytes of the weights' image and of the workspace."""
    lib = load()
    return _size(lib.spz_quant_image_bytes(outer, inner)), _size(lib.spz_quant_linear_workspace(prec, rows, outer, inner))


def quant_rows(x, *, stream=None):
    """x [rows, width] -> (q, scale): int8 q = x / scale rounded, scale = max |x| * float32(1 / 127) a row."""
    lib = load()
    gpu = _operand(x, "x", 2)

    if stream is not None or gpu != _device():
        return _elsewhere(stream, gpu, (x,), lambda: quant_rows(x))
    s = _stream(gpu)
    rows, width = x.shape
    q = x.new_empty((rows, width), dtype=torch.int8)
    scale = x.new_empty((rows,), dtype=_F32)
    _done(lib.spz_quant_rows(_PREC[x.dtype], rows, width, x.data_ptr(), x.stride(0), q.data_ptr(), q.stride(0),
                             scale.data_ptr(), s))
    return q, scale


def quant_pack(q, scale, *, stream=None) -> QuantWeights:
    """Weights q (int8 [outer, inner], e.g. of quant_rows) with a scale for each channel, laid out for
    quant_linear: once per set of weights."""
    lib = load()
    if not isinstance(q, torch.Tensor) or not q.is_cuda or q.dim() != 2:
        _refuse("q is no GPU tensor [outer, inner]")
    gpu = q.get_device()
    outer, inner = q.shape
    _like(q, "q", gpu, q.shape, torch.int8)
    if scale is None:
        _refuse("scale is missing")
    _like(scale, "scale", gpu, (outer,), _F32, contiguous=True)
    n = _size(lib.spz_quant_image_bytes(outer, inner))

    if stream is not None or gpu != _device():
        return _elsewhere(stream, gpu, (q, scale), lambda: quant_pack(q, scale))
    s = _stream(gpu)
    image = q.new_empty((n,))
    _done(lib.spz_quant_pack(outer, inner, q.data_ptr(), q.stride(0), image.data_ptr(), s))
    return QuantWeights(image, scale, outer, inner)


def quant_linear(x, weights: QuantWeights, *, bias=None, out=None, stream=None):
    """y [rows, outer] = x [rows, inner] times the packed weights, + bias (float32 [outer]): x is quantised a row
    at a time within the call, products and sums are exact integers, y has x's type."""
    lib = load()
    gpu = _operand(x, "x", 2)
    if not isinstance(weights, tuple) or len(weights) != 4:
        _refuse("weights are not those of quant_pack")
    image, scale, N, K = weights
    M = x.shape[0]
    if x.shape[1] != K:
        _refuse("x has %d columns, the weights have %d" % (x.shape[1], K))
    prec = _PREC[x.dtype]
    n_image, n = _quant_sizes(prec, M, N, K)
    _like(image, "weights.image", gpu, (n_image,), torch.int8, contiguous=True)
    _like(scale, "weights.scale", gpu, (N,), _F32, contiguous=True)
    _like(bias, "bias", gpu, (N,), _F32)
    _like(out, "out", gpu, (M, N), x.dtype)

    if stream is not None or gpu != _device():
        return _elsewhere(stream, gpu, (x, image, scale, bias, out), lambda: quant_linear(x, weights, bias=bias, out=out))
    s = _stream(gpu)
    y = out if out is not None else x.new_empty((M, N))
    ws = _workspace(n, x)
    rc = lib.spz_quant_linear(prec, M, N, K, x.data_ptr(), x.stride(0), image.data_ptr(), scale.data_ptr(), _ptr(bias),
                              y.data_ptr(), y.stride(0), _ptr(ws), n, s)
    if rc:
        _done(rc)
    return y
