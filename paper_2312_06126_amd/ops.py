"""The operators of a recurrent residual block on torch tensors (spz_scan_* .. spz_quant_* of
include/spz.h): argument checks, outputs and workspaces; every step runs in the HIP library.

Tensors are on one GPU; float32 or bfloat16 as the header says, states, scales and parameter vectors
float32. The last dimension is contiguous, the others have any strides. `stream`: a
torch.cuda.Stream or a hipStream_t address (default: the device's current stream); the call is
enqueued on it, and tensors that belong to another stream are kept alive until it has run; what
was enqueued elsewhere is the caller's to order. Nothing waits for the GPU, so calls may be
captured into a HIP graph. Errors: SpzError.
"""
from __future__ import annotations

import ctypes
from typing import NamedTuple, Optional

import torch

from .spz import GATES, NORMS, SPZ_EINVAL, SPZ_OK, BlockNormArgs, ScanArgs, SpzError, load

_PREC = {torch.float32: 0, torch.bfloat16: 1}
_byref = ctypes.byref


def _refuse(msg: str):
    raise SpzError(SPZ_EINVAL, msg)


def _done(lib, rc: int):
    if rc != SPZ_OK:
        raise SpzError(rc, lib.spz_last_error(None).decode())


def _size(lib, n: int) -> int:
    if n < 0:
        raise SpzError(n, lib.spz_last_error(None).decode())
    return n


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _like(t, name: str, ref: torch.Tensor, shape, dtype, contiguous: bool = False):
    """Checks one argument against the device of `ref`, a shape and a type (None stays None)."""
    if t is None:
        return
    if not isinstance(t, torch.Tensor):
        _refuse("%s is no tensor" % name)
    if t.device != ref.device:
        _refuse("%s is on %s, not on %s" % (name, t.device, ref.device))
    if t.shape != shape:
        _refuse("%s has shape %s, not %s" % (name, tuple(t.shape), tuple(shape)))
    if t.dtype not in (dtype if isinstance(dtype, tuple) else (dtype,)):
        _refuse("%s has type %s" % (name, t.dtype))
    if contiguous:
        if not t.is_contiguous():
            _refuse("%s is not contiguous" % name)
    elif t.shape[-1] > 1 and t.stride(-1) != 1:
        _refuse("%s is not contiguous in its last dimension" % name)


def _operand(t, name: str, dims: int):
    """The leading operand: a GPU tensor in one of the two precisions."""
    if not isinstance(t, torch.Tensor) or t.device.type != "cuda":
        _refuse("%s is no GPU tensor" % name)
    if t.dtype not in _PREC:
        _refuse("%s has type %s" % (name, t.dtype))
    if t.dim() != dims:
        _refuse("%s has %d dimensions, not %d" % (name, t.dim(), dims))
    _like(t, name, t, t.shape, t.dtype)


def _on_stream(stream, tensors, call):
    """call(stream address) on the device of the first tensor, with allocations on the stream."""
    device = tensors[0].device
    if stream is None:
        if device.index == torch.cuda.current_device():
            return call(torch.cuda.current_stream(device).cuda_stream)
        with torch.cuda.device(device):
            return call(torch.cuda.current_stream(device).cuda_stream)
    if isinstance(stream, int):
        stream = torch.cuda.ExternalStream(stream, device=device) if stream else torch.cuda.default_stream(device)
    elif stream.device != device:
        _refuse("the stream is on %s, the tensors are on %s" % (stream.device, device))
    with torch.cuda.stream(stream):
        out = call(stream.cuda_stream)
    for t in tensors:
        if t is not None:
            t.record_stream(stream)
    return out


def _workspace(n: int, ref: torch.Tensor) -> Optional[torch.Tensor]:
    return torch.empty(n, dtype=torch.uint8, device=ref.device) if n else None


# ----------------------------------------------------------------------------- scan

def _scan_args(f, v, h0, reset, lengths) -> ScanArgs:
    _operand(f, "f", 3)
    B, T, D = f.shape
    _like(v, "v", f, f.shape, f.dtype)
    _like(h0, "h0", f, (B, D), torch.float32, contiguous=True)
    _like(lengths, "lengths", f, (B,), torch.int32, contiguous=True)
    a = ScanArgs(B, T, D, f.data_ptr(), v.data_ptr(), f.stride(0), f.stride(1), v.stride(0), v.stride(1))
    if reset is not None:
        if not isinstance(reset, torch.Tensor) or reset.device != f.device or reset.shape != (B, T) or \
                reset.dtype not in (torch.uint8, torch.bool):
            _refuse("reset is no uint8 or bool tensor [batch, steps] on the device of f")
        a.reset, a.reset_batch, a.reset_step = reset.data_ptr(), reset.stride(0), reset.stride(1)
    a.lengths, a.h0, a.prec = _ptr(lengths), _ptr(h0), _PREC[f.dtype]
    return a


def _sequences(f: torch.Tensor) -> torch.Tensor:
    """An empty [batch, steps, width] tensor with the outer dimensions in the order of f's."""
    B, T, D = f.shape
    if f.stride(0) < f.stride(1) and B > 1:
        return torch.empty((T, B, D), dtype=f.dtype, device=f.device).transpose(0, 1)
    return torch.empty((B, T, D), dtype=f.dtype, device=f.device)


def scan(f, v, h0=None, *, reset=None, lengths=None, save: bool = False, out=None, hT=None, stream=None):
    """Gated linear recurrence: a = sigmoid(f), h_t = a_t h_{t-1} + (1 - a_t) v_t over [batch, steps,
    width] -> (y, hT), or (y, hT, saved) with save=True, for scan_backward.

    h0, hT: float32 [batch, width], the state in front (default zeros) and behind; pass hT=h0 to update
    a state in place. reset [batch, steps] (uint8 or bool): steps that start an episode, cut off from
    the state before. lengths [batch] (int32): steps of each sequence; y is 0 behind it. `out`: y."""
    lib = load()
    a = _scan_args(f, v, h0, reset, lengths)
    B, T, D = f.shape
    _like(out, "out", f, f.shape, f.dtype)
    _like(hT, "hT", f, (B, D), torch.float32, contiguous=True)

    def call(s):
        y = out if out is not None else _sequences(f)
        last = hT if hT is not None else torch.empty((B, D), dtype=torch.float32, device=f.device)
        saved = torch.empty(_size(lib, lib.spz_scan_saved(_byref(a))), dtype=torch.float32, device=f.device) if save else None
        a.y, a.y_batch, a.y_step, a.hT, a.saved = y.data_ptr(), y.stride(0), y.stride(1), last.data_ptr(), _ptr(saved)
        n = _size(lib, lib.spz_scan_workspace(_byref(a), 0))
        ws = _workspace(n, f)
        _done(lib, lib.spz_scan_forward(_byref(a), _ptr(ws), n, s))
        return (y, last, saved) if save else (y, last)

    return _on_stream(stream, (f, v, h0, reset, lengths, out, hT), call)


def scan_backward(f, v, dy, saved, *, dhT=None, reset=None, lengths=None, out=None, stream=None):
    """Gradients (df, dv, dh0) of scan's (y, hT) from dy (None: zeros) and dhT (None: zeros), with the
    `saved` of the forward call. `out`: the tensors (df, dv) to write, e.g. two parts of one."""
    lib = load()
    a = _scan_args(f, v, None, reset, lengths)
    B, T, D = f.shape
    _like(dy, "dy", f, f.shape, f.dtype)
    _like(dhT, "dhT", f, (B, D), torch.float32, contiguous=True)
    _like(saved, "saved", f, (_size(lib, lib.spz_scan_saved(_byref(a))),), torch.float32, contiguous=True)
    if saved is None:
        _refuse("saved is missing: scan(..., save=True) makes it")
    for name, t in zip(("df", "dv"), out or ()):
        _like(t, name, f, f.shape, f.dtype)
    if dy is not None:
        a.dy, a.dy_batch, a.dy_step = dy.data_ptr(), dy.stride(0), dy.stride(1)
    a.saved, a.dhT = saved.data_ptr(), _ptr(dhT)

    def call(s):
        df, dv = out if out is not None else (_sequences(f), _sequences(f))
        dh0 = torch.empty((B, D), dtype=torch.float32, device=f.device)
        a.df, a.df_batch, a.df_step = df.data_ptr(), df.stride(0), df.stride(1)
        a.dv, a.dv_batch, a.dv_step = dv.data_ptr(), dv.stride(0), dv.stride(1)
        a.dh0 = dh0.data_ptr()
        n = _size(lib, lib.spz_scan_workspace(_byref(a), 1))
        ws = _workspace(n, f)
        _done(lib, lib.spz_scan_backward(_byref(a), _ptr(ws), n, s))
        return df, dv, dh0

    return _on_stream(stream, (f, v, dy, saved, dhT, reset, lengths) + tuple(out or ()), call)


# ----------------------------------------------------------------------------- block norm

def _block_args(x, h, z, w_post, b_post, scale, w_pre, b_pre, post, pre, gate, eps, drop, valid) -> BlockNormArgs:
    _operand(x, "x", 2)
    R, D = x.shape
    if post not in NORMS or pre not in NORMS:
        _refuse("norms are %s" % ", ".join(NORMS))
    if gate not in GATES:
        _refuse("gates are %s" % ", ".join(GATES))
    _like(h, "h", x, x.shape, x.dtype)
    if gate != "none" and h is not None and z is None:
        _refuse("the gate needs z")
    _like(z, "z", x, x.shape, x.dtype)
    for name, t in (("w_post", w_post), ("b_post", b_post), ("scale", scale), ("w_pre", w_pre), ("b_pre", b_pre)):
        _like(t, name, x, (D,), torch.float32)
    _like(valid, "valid", x, (R,), (torch.uint8, torch.bool), contiguous=True)
    p, seed, step, tensor = drop if drop is not None else (0.0, 0, 0, 0)
    a = BlockNormArgs(R, D, x.data_ptr(), _ptr(h), _ptr(z), x.stride(0), 0 if h is None else h.stride(0),
                      0 if z is None else z.stride(0), _ptr(w_post), _ptr(b_post), _ptr(scale), _ptr(w_pre), _ptr(b_pre),
                      _ptr(valid))
    a.seed, a.step, a.tensor, a.drop_p, a.eps = int(seed), int(step) & 0xFFFFFFFF, int(tensor) & 0xFFFFFFFF, p, eps
    a.post, a.pre, a.gate, a.prec = NORMS[post], NORMS[pre], GATES[gate], _PREC[x.dtype]
    return a


def block_norm(x, h=None, z=None, w_post=None, b_post=None, scale=None, w_pre=None, b_pre=None, *, post="rms", pre="rms",
               gate="none", eps=1e-6, drop=None, valid=None, stream=None):
    """x' = x + scale * dropout(gate(z) * (post(h) * w_post + b_post)), u = pre(x') * w_pre + b_pre, over
    rows [rows, width] -> (x', u); u is None with pre="none". Without h: x' is x (the first block's
    norm). Norms "none", "rms", "layer"; gates "none", "sigmoid", "silu". drop: (p, seed, step, tensor) as
    dropout takes them. Rows with valid == 0 are neither read nor anything but zero."""
    lib = load()
    a = _block_args(x, h, z, w_post, b_post, scale, w_pre, b_pre, post, pre, gate, eps, drop, valid)

    def call(s):
        x_out = torch.empty(x.shape, dtype=x.dtype, device=x.device) if h is not None else x
        u = torch.empty(x.shape, dtype=x.dtype, device=x.device) if pre != "none" else None
        if h is not None:
            a.x_out, a.x_out_row = x_out.data_ptr(), x_out.stride(0)
        if u is not None:
            a.u, a.u_row = u.data_ptr(), u.stride(0)
        _done(lib, lib.spz_block_norm_forward(_byref(a), s))
        return x_out, u

    return _on_stream(stream, (x, h, z, w_post, b_post, scale, w_pre, b_pre, valid), call)


def block_norm_backward(dx_out, du, x, h=None, z=None, w_post=None, b_post=None, scale=None, w_pre=None, b_pre=None, *,
                        post="rms", pre="rms", gate="none", eps=1e-6, drop=None, valid=None, stream=None):
    """Gradients of block_norm from those of x' and u (None: zeros): a dict of dx, dh, dz and, for the
    vectors that were given, dw_post, dscale, dw_pre, db_post, db_pre (float32, summed over rows)."""
    lib = load()
    a = _block_args(x, h, z, w_post, b_post, scale, w_pre, b_pre, post, pre, gate, eps, drop, valid)
    _like(dx_out, "dx_out", x, x.shape, x.dtype)
    _like(du, "du", x, x.shape, x.dtype)
    a.dx_out, a.dx_out_row = _ptr(dx_out), 0 if dx_out is None else dx_out.stride(0)
    a.du, a.du_row = _ptr(du), 0 if du is None else du.stride(0)

    def call(s):
        rows = {"dx": x, "dh": h, "dz": z if h is not None and gate != "none" else None}
        grads = {k: None if t is None else torch.empty(x.shape, dtype=x.dtype, device=x.device) for k, t in rows.items()}
        for k, t in (("dw_post", w_post), ("dscale", scale), ("dw_pre", w_pre), ("db_post", b_post), ("db_pre", b_pre)):
            grads[k] = None if t is None else torch.empty(t.shape, dtype=torch.float32, device=x.device)
        for k, t in grads.items():
            if t is not None:
                setattr(a, k, t.data_ptr())
        a.dx_row = a.dh_row = a.dz_row = x.shape[1]
        n = _size(lib, lib.spz_block_norm_workspace(_byref(a)))
        ws = _workspace(n, x)
        _done(lib, lib.spz_block_norm_backward(_byref(a), _ptr(ws), n, s))
        return grads

    return _on_stream(stream, (x, dx_out, du, h, z, w_post, b_post, scale, w_pre, b_pre, valid), call)


def dropout(x, p: float, seed: int, step: int, tensor: int = 0, *, out=None, stream=None):
    """x [rows, width] with elements dropped with probability p, the others scaled up. The mask is a
    function of (seed, step, tensor) and the element's index, so the same call on the gradient is
    the backward pass. `out` may be x."""
    lib = load()
    _operand(x, "x", 2)
    _like(out, "out", x, x.shape, x.dtype)

    def call(s):
        y = out if out is not None else torch.empty(x.shape, dtype=x.dtype, device=x.device)
        _done(lib, lib.spz_dropout(_PREC[x.dtype], x.shape[0], x.shape[1], x.data_ptr(), x.stride(0), y.data_ptr(), y.stride(0),
                                   p, int(seed) & 0xFFFFFFFFFFFFFFFF, int(step) & 0xFFFFFFFF, int(tensor) & 0xFFFFFFFF, s))
        return y

    return _on_stream(stream, (x, out), call)


# ----------------------------------------------------------------------------- 8-bit product

class QuantWeights(NamedTuple):
    """Weights of quant_linear: the integers in the product's order and a scale for each channel."""
    image: torch.Tensor
    scale: torch.Tensor
    outer: int
    inner: int


def quant_rows(x, *, stream=None):
    """x [rows, width] -> (q, scale): int8 q = x / scale rounded, scale = max |x| / 127 a row."""
    lib = load()
    _operand(x, "x", 2)

    def call(s):
        q = torch.empty(x.shape, dtype=torch.int8, device=x.device)
        scale = torch.empty((x.shape[0],), dtype=torch.float32, device=x.device)
        _done(lib, lib.spz_quant_rows(_PREC[x.dtype], x.shape[0], x.shape[1], x.data_ptr(), x.stride(0), q.data_ptr(), q.stride(0),
                                      scale.data_ptr(), s))
        return q, scale

    return _on_stream(stream, (x,), call)


def quant_pack(q, scale, *, stream=None) -> QuantWeights:
    """Weights q (int8 [outer, inner], e.g. of quant_rows) with a scale for each channel, laid out for
    quant_linear: once per set of weights."""
    lib = load()
    if not isinstance(q, torch.Tensor) or q.device.type != "cuda" or q.dim() != 2:
        _refuse("q is no GPU tensor [outer, inner]")
    _like(q, "q", q, q.shape, torch.int8)
    _like(scale, "scale", q, (q.shape[0],), torch.float32, contiguous=True)
    if scale is None:
        _refuse("scale is missing")
    n = _size(lib, lib.spz_quant_image_bytes(q.shape[0], q.shape[1]))

    def call(s):
        image = torch.empty(n, dtype=torch.int8, device=q.device)
        _done(lib, lib.spz_quant_pack(q.shape[0], q.shape[1], q.data_ptr(), q.stride(0), image.data_ptr(), s))
        return QuantWeights(image, scale, q.shape[0], q.shape[1])

    return _on_stream(stream, (q, scale), call)


def quant_linear(x, weights: QuantWeights, *, bias=None, out=None, stream=None):
    """y [rows, outer] = x [rows, inner] times the packed weights, + bias (float32 [outer]): x is quantised a row
    at a time within the call, products and sums are exact integers, y has x's type."""
    lib = load()
    _operand(x, "x", 2)
    M, N, K = x.shape[0], weights.outer, weights.inner
    if x.shape[1] != K:
        _refuse("x has %d columns, the weights have %d" % (x.shape[1], K))
    _like(weights.image, "weights.image", x, (_size(lib, lib.spz_quant_image_bytes(N, K)),), torch.int8, contiguous=True)
    _like(weights.scale, "weights.scale", x, (N,), torch.float32, contiguous=True)
    _like(bias, "bias", x, (N,), torch.float32)
    _like(out, "out", x, (M, N), x.dtype)

    def call(s):
        y = out if out is not None else torch.empty((M, N), dtype=x.dtype, device=x.device)
        n = _size(lib, lib.spz_quant_linear_workspace(_PREC[x.dtype], M, N, K))
        ws = _workspace(n, x)
        _done(lib, lib.spz_quant_linear(_PREC[x.dtype], M, N, K, x.data_ptr(), x.stride(0), weights.image.data_ptr(),
                                        weights.scale.data_ptr(), _ptr(bias), y.data_ptr(), y.stride(0), _ptr(ws), n, s))
        return y

    return _on_stream(stream, (x, weights.image, weights.scale, bias, out), call)
