"""The operators of recurrent and linear-attention blocks and their optimizer on torch tensors (spz_scan_* .. spz_adamw
of include/spz.h): argument checks, outputs and workspaces; every step runs in the HIP library.

Tensors are on one GPU; float32 or bfloat16 as the header says, states, scales and parameter vectors
float32. The last dimension is contiguous, the others have any strides. `stream`: a
torch.cuda.Stream or a hipStream_t address (default: the device's current stream); the call is
enqueued on it, and where `stream` is given tensors that belong to another one are kept alive until it has run; what
was enqueued elsewhere is the caller's to order. Nothing waits for the GPU, so calls may be
captured into a HIP graph. Errors: SpzError.

torch's autograd does not record the calls: gradients come from scan_backward, block_norm_backward, head_norm_backward,
linear_attention_backward and, for dropout, the same call on the gradient (quant_linear has none). Tensors that require a gradient are refused, so that none is
lost; within torch.no_grad() they are taken. A tensor that a caller gives to be written counts as changed in place, so that autograd
refuses what it has saved of it. The calls work on data pointers: they are not for tracing or vmap.
"""
from __future__ import annotations

import ctypes
import functools
import math
import struct
from typing import NamedTuple, Optional, Sequence

import numpy as np
import torch

from .spz import (ADAMW_BLOCK, GATES, NORMS, PAIRS, SPZ_EINVAL, SPZ_OK, SpzError, load, pack_adamw, pack_adamw_tensor,
                  pack_block_norm, pack_head_norm, pack_linear_attention, pack_scan)

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


def _wrote(*given: Optional[torch.Tensor]):
    """Marks a caller's own tensors as written: what autograd has saved of one is not what it was."""
    given = [t for t in given if t is not None]
    if given:
        torch.autograd.graph.increment_version(given)


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
    _wrote(out, hT)
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
    _wrote(*out or ())
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
    _wrote(out)
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
    _wrote(out)
    return y


# ----------------------------------------------------------------------------- head norms

def rotation_freqs(dim: int, base: float = 10000.0, device="cuda") -> torch.Tensor:
    """Angles a position for head_norm: base^(-2 i / dim), i < dim / 2 (float64)."""
    return torch.tensor([base ** (-2.0 * i / dim) for i in range(dim // 2)], dtype=torch.float64, device=device)


def _head_check(q, k, vectors, norm, positions, freqs, pairs, valid) -> int:
    gpu = _operand(q, "q", 3)
    R, _, D = q.shape
    if norm not in NORMS:
        _refuse("norms are %s" % ", ".join(NORMS))
    if pairs not in PAIRS:
        _refuse("pairs are %s" % ", ".join(PAIRS))
    if k is not None:
        if not isinstance(k, torch.Tensor) or k.dim() != 3:
            _refuse("k is no tensor [rows, heads, dim]")
        _like(k, "k", gpu, (R, k.shape[1], D), q.dtype)
    for i, t in enumerate(vectors):
        if t is not None and not (isinstance(t, torch.Tensor) and t.dtype is _F32 and t.dim() == 1 and t.numel() == D
                                  and t.get_device() == gpu and t.is_contiguous() and not t.requires_grad):
            _like(t, ("w_q", "b_q", "w_k", "b_k")[i], gpu, (D,), _F32)
    if freqs is not None and positions is not None:
        if not (isinstance(positions, torch.Tensor) and positions.dtype is torch.int32 and positions.dim() == 1 and positions.numel() == R
                and positions.get_device() == gpu and positions.is_contiguous()):
            _like(positions, "positions", gpu, (R,), torch.int32, contiguous=True)
        if not isinstance(freqs, torch.Tensor) or freqs.dim() != 1 or 2 * freqs.numel() > D:
            _refuse("freqs is no tensor of at most dim / 2 angles")
        if freqs.dtype is not torch.float64 or freqs.get_device() != gpu or not freqs.is_contiguous() or freqs.requires_grad:
            _like(freqs, "freqs", gpu, freqs.shape, torch.float64, contiguous=True)
    elif positions is not freqs:
        _refuse("positions and freqs come together")
    if valid is not None:
        _like(valid, "valid", gpu, (R,), torch.bool if getattr(valid, "dtype", None) is torch.bool else torch.uint8, contiguous=True)
    return gpu


def _two(t):
    """Strides of the rows and heads (no tensor: 0)."""
    return (0, 0) if t is None else t.stride()[:2]


def _pair_out(out, q, k, gpu, names):
    """The two tensors of an `out` argument, checked."""
    if not isinstance(out, (tuple, list)) or len(out) != 2 or out[0] is None or (out[1] is None) != (k is None):
        _refuse("out holds %s and %s" % names)
    _like(out[0], names[0], gpu, q.shape, q.dtype)
    if k is not None:
        _like(out[1], names[1], gpu, k.shape, q.dtype)
    return out


def _head_pack(q, k, vectors, positions, freqs, valid, outs, back, grads, eps, norm, pairs) -> bytes:
    """The argument block; outs (forward): q_out, k_out; back (backward): dq_out, dk_out, dq, dk; grads: dw_q, db_q, dw_k, db_k."""
    R, H, D = q.shape
    rq, hq, _ = q.stride()
    if k is None:
        K = pk = rk = hk = 0
    else:
        K, pk, (rk, hk, _) = k.shape[1], k.data_ptr(), k.stride()
    wq, bq, wk, bk = vectors
    try:
        if outs is not None:
            a, b = outs
            rest = (a.data_ptr(), _ptr(b), *_two(a), *_two(b), 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0)
        else:
            rest = (0, 0, 0, 0, 0, 0, _ptr(back[0]), _ptr(back[1]), *_two(back[0]), *_two(back[1]), _ptr(back[2]), _ptr(back[3]), *_two(back[2]),
                    *_two(back[3]), *map(_ptr, grads))
        return pack_head_norm(R, H, K, D, 0 if freqs is None else freqs.numel(), q.data_ptr(), pk, rq, hq, rk, hk, _ptr(wq), _ptr(bq), _ptr(wk), _ptr(bk),
                              _ptr(positions), _ptr(freqs), _ptr(valid), *rest, eps, NORMS[norm], PAIRS[pairs], _PREC[q.dtype])
    except _NOT_NUMBERS as e:
        _refuse("eps is no number: %s" % e)


def head_norm(q, k=None, w_q=None, w_k=None, b_q=None, b_k=None, *, norm="rms", eps=1e-6, positions=None, freqs=None, pairs="halves",
              valid=None, out=None, stream=None):
    """norm(x) * w + b of each head of q [rows, heads, dim] and k [rows, other heads, dim] (None: no keys), with the
    first 2 len(freqs) columns turned in pairs by the angle positions[row] * freqs[i] -> (q', k').

    norm "none", "rms", "layer"; pairs "halves" (columns i and len(freqs) + i) or "neighbours" (2 i and 2 i + 1).
    positions int32 [rows] and freqs float64 (rotation_freqs makes some) come together. Rows with valid == 0 are
    not read, their outputs are zero. `out`: (q', k'); they may be q and k and otherwise share no elements with them or each other."""
    lib = load()
    vectors = (w_q, b_q, w_k, b_k)
    gpu = _head_check(q, k, vectors, norm, positions, freqs, pairs, valid)
    q_out, k_out = (None, None) if out is None else _pair_out(out, q, k, gpu, ("q'", "k'"))

    if stream is not None or gpu != _device():
        return _elsewhere(stream, gpu, (q, k, *vectors, positions, freqs, valid, q_out, k_out),
                          lambda: head_norm(q, k, w_q, w_k, b_q, b_k, norm=norm, eps=eps, positions=positions, freqs=freqs, pairs=pairs,
                                            valid=valid, out=out))
    s = _stream(gpu)
    if q_out is None:
        q_out, k_out = q.new_empty(q.shape), None if k is None else q.new_empty(k.shape)
    rc = lib.spz_head_norm_forward(_head_pack(q, k, vectors, positions, freqs, valid, (q_out, k_out), None, None, eps, norm, pairs), s)
    if rc:
        _done(rc)
    _wrote(*out or ())
    return q_out, k_out


def head_norm_backward(dq_out, dk_out, q, k=None, w_q=None, w_k=None, b_q=None, b_k=None, *, norm="rms", eps=1e-6, positions=None,
                       freqs=None, pairs="halves", valid=None, out=None, stream=None):
    """Gradients of head_norm from those of q' and k' (None: zeros): a dict of dq, dk and, for the vectors that were
    given, dw_q, db_q, dw_k, db_k (float32, summed over rows and heads). `out`: (dq, dk), e.g. two parts of one; dq may be dq_out or q and dk dk_out or k, and
    otherwise they share no elements with these or each other."""
    lib = load()
    vectors = (w_q, b_q, w_k, b_k)
    gpu = _head_check(q, k, vectors, norm, positions, freqs, pairs, valid)
    _like(dq_out, "dq_out", gpu, q.shape, q.dtype)
    if k is None and dk_out is not None:
        _refuse("dk_out without k")
    if k is not None:
        _like(dk_out, "dk_out", gpu, k.shape, q.dtype)
    dq, dk = (None, None) if out is None else _pair_out(out, q, k, gpu, ("dq", "dk"))

    if stream is not None or gpu != _device():
        return _elsewhere(stream, gpu, (dq_out, dk_out, q, k, *vectors, positions, freqs, valid, dq, dk),
                          lambda: head_norm_backward(dq_out, dk_out, q, k, w_q, w_k, b_q, b_k, norm=norm, eps=eps, positions=positions, freqs=freqs,
                                                     pairs=pairs, valid=valid, out=out))
    s = _stream(gpu)
    if dq is None:
        dq, dk = q.new_empty(q.shape), None if k is None else q.new_empty(k.shape)
    g = {"dq": dq, "dk": dk}
    sums = iter(q.new_empty((4, q.shape[2]), dtype=_F32).unbind(0))
    for name, t in zip(("dw_q", "db_q", "dw_k", "db_k"), vectors):
        g[name] = None if t is None else next(sums)
    a = _head_pack(q, k, vectors, positions, freqs, valid, None, (dq_out, dk_out, dq, dk),
                   (g["dw_q"], g["db_q"], g["dw_k"], g["db_k"]), eps, norm, pairs)
    n = _size(lib.spz_head_norm_workspace(a))
    ws = _workspace(n, q)
    _done(lib.spz_head_norm_backward(a, _ptr(ws), n, s))
    _wrote(*out or ())
    return g


# ----------------------------------------------------------------------------- linear attention

@functools.lru_cache(maxsize=4096)
def _attention_sizes(B: int, T: int, H: int, K: int, V: int, prec: int):
    """Bytes of the workspaces, forward and backward: functions of the sizes alone."""
    lib = load()
    a = pack_linear_attention(B, T, H, K, V, *([0] * 41), 0.0, prec)
    return _size(lib.spz_linear_attention_workspace(a, 0)), _size(lib.spz_linear_attention_workspace(a, 1))


def _attention_check(q, k, v, rate, state, reset, lengths) -> int:
    gpu = _operand(q, "q", 4)
    B, T, H, K = shape = q.shape
    if k is None or v is None:
        _refuse("k or v is missing")
    _like(k, "k", gpu, shape, q.dtype)
    if not isinstance(v, torch.Tensor) or v.dim() != 4:
        _refuse("v is no tensor [batch, steps, heads, width]")
    V = v.shape[3]
    _like(v, "v", gpu, (B, T, H, V), q.dtype)
    if rate is not None:
        _like(rate, "rate", gpu, (H,), _F32, contiguous=True)
    if state is not None:
        _like(state, "state", gpu, (B, H, K, V), _F32, contiguous=True)
    if lengths is not None:
        _like(lengths, "lengths", gpu, (B,), torch.int32, contiguous=True)
    if reset is not None:
        _flags_2d(reset, "reset", gpu, (B, T))
    return gpu


def _three(t):
    """Strides of the batch, time and head dimensions (no tensor: 0)."""
    return (0, 0, 0) if t is None else t.stride()[:3]


def _steps(like: torch.Tensor, width: int) -> torch.Tensor:
    """An empty [batch, steps, heads, width] tensor with the outer two dimensions in the order of like's."""
    B, T, H, _ = like.shape
    s = like.stride()
    if s[0] < s[1] and B > 1:
        return like.new_empty((T, B, H, width)).transpose(0, 1)
    return like.new_empty((B, T, H, width))


def linear_attention(q, k, v, rate=None, state=None, *, scale=None, reset=None, lengths=None, out=None, last=None, stream=None):
    """S_t = exp(-rate) S_{t-1} + k_t^T v_t, y_t = scale q_t S_t in each head of q, k [batch, steps, heads, width] and
    v [batch, steps, heads, other width] (at most 256 wide) -> (y, last).

    rate: float32 [heads] (default zeros). state, last: float32 [batch, heads, width, other width], S in front
    (default zeros) and behind; pass last=state to update a state in place. scale: default 1 / sqrt(width). reset
    [batch, steps] (uint8 or bool): steps that start an episode, cut off from the state before. lengths [batch]
    (int32): steps of each sequence; y is 0 behind it. Heads may share q, k or v (stride 0). `out`: y; it may be v and
    otherwise shares no elements with the operands. Products of queries with keys and states are taken in float32 before decays
    and values meet them: include/spz.h says which magnitudes that takes."""
    lib = load()
    gpu = _attention_check(q, k, v, rate, state, reset, lengths)
    B, T, H, K = q.shape
    V = v.shape[3]
    if out is not None:
        _like(out, "out", gpu, v.shape, q.dtype)
    if last is not None and last is not state:
        _like(last, "last", gpu, (B, H, K, V), _F32, contiguous=True)
    n = _attention_sizes(B, T, H, K, V, _PREC[q.dtype])[0]

    if stream is not None or gpu != _device():
        return _elsewhere(stream, gpu, (q, k, v, rate, state, reset, lengths, out, last),
                          lambda: linear_attention(q, k, v, rate, state, scale=scale, reset=reset, lengths=lengths, out=out, last=last))
    s = _stream(gpu)
    y = out if out is not None else _steps(q, V)
    end = last if last is not None else q.new_empty((B, H, K, V), dtype=_F32)
    ws = _workspace(n, q)
    try:
        a = pack_linear_attention(
            B, T, H, K, V, q.data_ptr(), k.data_ptr(), v.data_ptr(), *_three(q), *_three(k), *_three(v), _ptr(rate), _ptr(reset), *_outer(reset),
            _ptr(lengths), _ptr(state), y.data_ptr(), *_three(y), end.data_ptr(), *([0] * 18),
            1.0 / math.sqrt(max(K, 1)) if scale is None else scale, _PREC[q.dtype])
    except _NOT_NUMBERS as e:
        _refuse("scale is no number: %s" % e)
    rc = lib.spz_linear_attention_forward(a, _ptr(ws), n, s)
    if rc:
        _done(rc)
    _wrote(out, last)
    return y, end


def linear_attention_backward(q, k, v, dy, rate=None, state=None, *, scale=None, dlast=None, reset=None, lengths=None, out=None, stream=None):
    """Gradients (dq, dk, dv, dstate) of linear_attention's (y, last) from dy and dlast (None: zeros), with the forward
    call's other arguments (`state` as it was before the call). Those of shared heads are one for each
    head. `out`: the tensors (dq, dk, dv) to write, e.g. three parts of one; they share no elements with each other or the operands."""
    lib = load()
    gpu = _attention_check(q, k, v, rate, state, reset, lengths)
    B, T, H, K = q.shape
    V = v.shape[3]
    _like(dy, "dy", gpu, v.shape, q.dtype)
    _like(dlast, "dlast", gpu, (B, H, K, V), _F32, contiguous=True)
    if out is not None:
        if not isinstance(out, (tuple, list)) or len(out) != 3 or any(t is None for t in out):
            _refuse("out holds dq, dk and dv")
        for name, t, w in zip(("dq", "dk", "dv"), out, (q, k, v)):
            _like(t, name, gpu, w.shape, q.dtype)
    n = _attention_sizes(B, T, H, K, V, _PREC[q.dtype])[1]

    if stream is not None or gpu != _device():
        return _elsewhere(stream, gpu, (q, k, v, dy, rate, state, dlast, reset, lengths) + tuple(out or ()),
                          lambda: linear_attention_backward(q, k, v, dy, rate, state, scale=scale, dlast=dlast, reset=reset, lengths=lengths, out=out))
    s = _stream(gpu)
    dq, dk, dv = out if out is not None else (_steps(q, K), _steps(q, K), _steps(q, V))
    dstate = q.new_empty((B, H, K, V), dtype=_F32)
    ws = _workspace(n, q)
    try:
        a = pack_linear_attention(
            B, T, H, K, V, q.data_ptr(), k.data_ptr(), v.data_ptr(), *_three(q), *_three(k), *_three(v), _ptr(rate), _ptr(reset), *_outer(reset),
            _ptr(lengths), _ptr(state), 0, 0, 0, 0, 0, _ptr(dy), *_three(dy), _ptr(dlast), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(),
            *_three(dq), *_three(dk), *_three(dv), dstate.data_ptr(), 1.0 / math.sqrt(max(K, 1)) if scale is None else scale, _PREC[q.dtype])
    except _NOT_NUMBERS as e:
        _refuse("scale is no number: %s" % e)
    _done(lib.spz_linear_attention_backward(a, _ptr(ws), n, s))
    _wrote(*out or ())
    return dq, dk, dv, dstate


# ----------------------------------------------------------------------------- AdamW

class AdamW:
    """AdamW over a list of contiguous float32 or bfloat16 GPU tensors, which step() updates in place.

    bits=32: the moments are float32. bits=8: e4m3 codes (of the second moment's root, for v) with a scale for
    each 256 of them, rounded at random by `seed` and the step, so that small changes count on average. `m`, `v` and,
    for 8 bits, `m_scale`, `v_scale` hold the moments of all tensors one after the other, each from places[i] on, and are
    the state to save; they start as zeros and may be copied into. copies: bfloat16 tensors that get each new value as
    well (a list with None for none). weight_decay: a number, or one for each tensor. No two parameters or copies
    share elements, and no gradient shares any with another parameter or its copy."""

    def __init__(self, params: Sequence[torch.Tensor], *, bits: int = 32, copies=None, weight_decay=0.0, seed: int = 0):
        params = list(params)
        if not params:
            _refuse("no parameters")
        if bits not in (8, 32):
            _refuse("bits are 8 or 32")
        first = params[0]
        if not isinstance(first, torch.Tensor) or not first.is_cuda:
            _refuse("params[0] is no GPU tensor")
        self._gpu = gpu = first.get_device()
        copies = [None] * len(params) if copies is None else list(copies)
        try:
            decay = [float(d) for d in weight_decay] if hasattr(weight_decay, "__len__") else [float(weight_decay)] * len(params)
            self._seed = int(seed) & 0xFFFFFFFFFFFFFFFF
        except _NOT_NUMBERS as e:
            _refuse("weight_decay or seed is no number: %s" % e)
        if len(copies) != len(params) or len(decay) != len(params):
            _refuse("copies and weight_decay have one entry for each tensor")
        spans, at, self.places = [], 0, []
        for i, (p, c, d) in enumerate(zip(params, copies, decay)):
            self._tensor(p, "params[%d]" % i)
            if c is not None:
                if p.dtype is not _F32:
                    _refuse("copies[%d] of a tensor that is not float32" % i)
                if not isinstance(c, torch.Tensor) or c.requires_grad:
                    _refuse("copies[%d] is no tensor, or requires a gradient" % i)
                _like(c, "copies[%d]" % i, gpu, p.shape, torch.bfloat16, contiguous=True)
            if not math.isfinite(d):
                _refuse("weight_decay of params[%d] is not finite" % i)
            spans += [(t.data_ptr(), t.data_ptr() + t.numel() * t.element_size()) for t in (p, c) if t is not None and t.numel()]
            self.places.append(at)
            at += -(-p.numel() // ADAMW_BLOCK) * ADAMW_BLOCK
        spans.sort()
        if any(a[1] > b[0] for a, b in zip(spans, spans[1:])):
            _refuse("two of the tensors share elements")
        self.params, self.copies, self.bits, self.weight_decay = tuple(params), tuple(copies), bits, tuple(decay)
        kind = torch.float8_e4m3fn if bits == 8 else _F32
        dev = first.device
        self.m, self.v = (torch.zeros(at, dtype=kind, device=dev) for _ in range(2))
        self.m_scale, self.v_scale = (torch.zeros(at // ADAMW_BLOCK, device=dev) if bits == 8 else None for _ in range(2))
        self._moments = at
        self._written = (*params, *(c for c in copies if c is not None))
        self._layout = [(p, c, p.shape, p.numel(), p.data_ptr(), _ptr(c)) for p, c in zip(params, copies)]
        # One row of 64-bit words for each tensor, as the library reads them (spz_adamw_tensor).
        self._plan = np.frombuffer(b"".join(pack_adamw_tensor(p.data_ptr(), 0, _ptr(c), p.numel(), at, d)
                                            for p, c, at, d in zip(params, copies, self.places, decay)), np.uint64).reshape(len(params), 6)
        self._one_type = first.dtype if all(p.dtype is first.dtype for p in params) else None

    def _tensor(self, p, name):
        if not isinstance(p, torch.Tensor) or p.get_device() != self._gpu or p.dtype not in _PREC or not p.is_contiguous():
            _refuse("%s is no contiguous float32 or bfloat16 tensor on cuda:%d" % (name, self._gpu))
        if p.requires_grad and not p.is_leaf:
            _refuse("%s is not a leaf" % name)

    def _state(self):
        """The moments, which a user may have replaced by tensors of their own."""
        kind = torch.float8_e4m3fn if self.bits == 8 else _F32
        _like(self.m, "m", self._gpu, (self._moments,), kind, contiguous=True)
        _like(self.v, "v", self._gpu, (self._moments,), kind, contiguous=True)
        if self.bits == 8:
            _like(self.m_scale, "m_scale", self._gpu, (self._moments // ADAMW_BLOCK,), _F32, contiguous=True)
            _like(self.v_scale, "v_scale", self._gpu, (self._moments // ADAMW_BLOCK,), _F32, contiguous=True)

    def step(self, grads, *, step, lr, betas=(0.9, 0.999), eps: float = 1e-8, grad_scale=None, stream=None):
        """One update with the gradients (float32 or bfloat16, a list with None for tensors that stay as they are).

        step: the count of this update, from 1, or an int64 GPU tensor of one element; lr: a number, or a float32
        GPU tensor of one element. Tensors are read when the kernel runs, so that a captured graph follows them.
        grad_scale: a float32 GPU tensor of one element that multiplies the gradients (a clip, a loss scale)."""
        lib = load()
        gpu = self._gpu
        if not isinstance(grads, (tuple, list)) or len(grads) != len(self.params):
            _refuse("grads is no list of %d" % len(self.params))
        self._state()
        for name, t, kind in (("step", step, torch.int64), ("lr", lr, _F32), ("grad_scale", grad_scale, _F32)):
            if isinstance(t, torch.Tensor):
                if t.numel() != 1:
                    _refuse("%s has more than one element, or none" % name)
                _like(t, name, gpu, t.shape, kind, contiguous=True)
        if grad_scale is not None and not isinstance(grad_scale, torch.Tensor):
            _refuse("grad_scale is no tensor")
        grad_on, first = _grad_on(), None
        plain, addresses = True, []    # plain: all tensors have a gradient, of one type
        for i, (g, (p, c, shape, n, at, to)) in enumerate(zip(grads, self._layout)):
            if g is None:
                plain = False
                addresses.append(0)
                continue
            if not isinstance(g, torch.Tensor) or g.dtype not in _PREC or g.shape != shape or g.get_device() != gpu or not g.is_contiguous():
                _refuse("grads[%d] is no contiguous float32 or bfloat16 tensor %s on cuda:%d" % (i, tuple(shape), gpu))
            if grad_on and g.requires_grad:
                _refuse_grad("grads[%d]" % i)
            if p.data_ptr() != at or p.numel() != n or (c is not None and c.data_ptr() != to):
                _refuse("params[%d] or its copy is not where it was: make another AdamW of the new tensors" % i)
            addresses.append(g.data_ptr())
            kind = g.dtype
            if kind is not first:
                plain = plain and first is None
                first = kind

        if stream is not None or gpu != _device():
            tensors = [*self.params, *self.copies, *grads, self.m, self.v, self.m_scale, self.v_scale, grad_scale]
            tensors += [t for t in (step, lr) if isinstance(t, torch.Tensor)]
            return _elsewhere(stream, gpu, tensors, lambda: self.step(grads, step=step, lr=lr, betas=betas, eps=eps, grad_scale=grad_scale))
        s = _stream(gpu)
        on_step, on_lr = isinstance(step, torch.Tensor), isinstance(lr, torch.Tensor)
        # The entries of a call: a copy of the plan's with the gradients' addresses, one call for each pair of types.
        entries = self._plan.copy()
        entries[:, 1] = addresses
        if plain and self._one_type:
            calls = ((_PREC[self._one_type], _PREC[first], entries),)
        else:
            kinds = [None if g is None else (_PREC[p.dtype], _PREC[g.dtype]) for p, g in zip(self.params, grads)]
            calls = [(*k, entries[[i for i, x in enumerate(kinds) if x == k]]) for k in sorted(set(kinds) - {None})]
        for p_prec, g_prec, block in calls:
            try:
                b1, b2 = betas
                a = pack_adamw(len(block), self._moments, block.ctypes.data, self.m.data_ptr(), self.v.data_ptr(), _ptr(self.m_scale),
                               _ptr(self.v_scale), _ptr(grad_scale), step.data_ptr() if on_step else 0, lr.data_ptr() if on_lr else 0,
                               0 if on_step else step, 0.0 if on_lr else lr, b1, b2, eps, self._seed, self.bits, p_prec, g_prec, 0)
            except _NOT_NUMBERS as e:
                _refuse("step, lr, betas or eps is no number: %s" % e)
            rc = lib.spz_adamw(a, s)
            if rc:
                _done(rc)
        _wrote(*self._written if plain else (t for p, c, g in zip(self.params, self.copies, grads) if g is not None for t in (p, c)))
