"""Head norms, linear attention and AdamW in float64 numpy, from their formulas, with error bounds.

As in ops_reference: each value comes with a bound on what float32 arithmetic may be off from it, U being
float32's unit roundoff; `ops_reference.rounded` adds the output type's own half ulp.
"""
import numpy as np

from .ops_reference import U

SPLIT = 2.0 ** -16   # bfloat16 calls: scores and states enter a product as two bfloat16 numbers each, which keep 2^-17 of each
BLOCK = 256


# ----------------------------------------------------------------------------- head norms

def turn(x, cos, sin, pairs):
    """x [rows, heads, dim] with its first 2 half columns turned by the angles of cos, sin [rows, half]."""
    half = cos.shape[1]
    y = x.copy()
    a, b = (slice(0, half), slice(half, 2 * half)) if pairs == "halves" else (slice(0, 2 * half, 2), slice(1, 2 * half, 2))
    c, s = cos[:, None], sin[:, None]
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
    return y


def turn_bound(size, far, half, pairs):
    """Error of a turned pair of these magnitudes: sine and cosine to 8 U (the part of a turn is rounded once, and the
    functions to 4 ulp) and the angle's own 2^-51, and two products and a sum."""
    e = np.zeros_like(size)
    if half:
        a, b = (slice(0, half), slice(half, 2 * half)) if pairs == "halves" else (slice(0, 2 * half, 2), slice(1, 2 * half, 2))
        both = size[..., a] + size[..., b]
        e[..., a] = e[..., b] = (12 * U + 2.0 ** -51 * far) * both
    return e


def head_norm(x, w=None, b=None, kind="rms", eps=1e-6, positions=None, freqs=None, pairs="halves", valid=None, dy=None):
    """One of queries and keys [rows, heads, dim] -> dict of y and, with dy, dx, dw, db: (value, bound)."""
    R, H, D = x.shape
    live = np.ones(R, bool) if valid is None else np.asarray(valid) != 0
    row = live[:, None, None]
    x = np.where(row, x, 0.0)
    K = 64 * U
    n, r = x, np.ones((R, H, 1))
    if kind != "none":
        n = x - x.mean(-1, keepdims=True) if kind == "layer" else x
        r = 1.0 / np.sqrt((n * n).mean(-1, keepdims=True) + eps)
        n = n * r
        en = K * (np.abs(n) + np.abs(x).max(-1, keepdims=True) * r)
    else:
        en = np.zeros_like(n)
    wv, bv = (np.ones(D) if w is None else w), (np.zeros(D) if b is None else b)
    t = n * wv + bv
    et = np.abs(wv) * en + 4 * U * (np.abs(n * wv) + np.abs(bv))
    half, cos, sin, far = 0, None, None, 0.0
    if freqs is not None:
        half = len(freqs)
        angle = np.where(live[:, None], positions[:, None].astype(float) * freqs, 0.0)
        cos, sin, far = np.cos(angle), np.sin(angle), np.abs(angle).max(initial=0.0)
    y = turn(t, cos, sin, pairs) if half else t
    ey = turn(et, np.abs(cos), -np.abs(sin), pairs) if half else et       # |a| |c| + |b| |s|
    ey = np.maximum(ey, turn(et, np.abs(cos), np.abs(sin), pairs)) if half else ey
    ey = ey + turn_bound(np.abs(t), far, half, pairs)
    out = {"y": (y * row, ey * row)}
    if dy is None:
        return out
    dy = np.where(row, dy, 0.0)
    d = turn(dy, cos, -sin, pairs) if half else dy
    ed = turn_bound(np.abs(dy), far, half, pairs)
    dn = d * wv
    edn = np.abs(wv) * ed + 2 * U * np.abs(dn)
    if kind != "none":
        g = dn - n * (dn * n).mean(-1, keepdims=True)
        dx = r * (g - dn.mean(-1, keepdims=True) if kind == "layer" else g)
        big = lambda q: r * (q + (1 + np.abs(n)) * (q * (1 + np.abs(n))).mean(-1, keepdims=True))   # noqa: E731
        rel = 256 * U + en.max(-1, keepdims=True) / (1e-30 + np.abs(n).max(-1, keepdims=True))
        edx = 4 * rel * big(np.abs(dn)) + big(edn)
    else:
        dx, edx = dn, edn
    out["dx"] = (dx * row, edx * row)
    for name, v, e in (("dw", d * n, np.abs(n) * ed + np.abs(d) * en + 2 * U * np.abs(d * n)), ("db", d, ed)):
        v, e = v * row, e * row
        out[name] = (v.sum((0, 1)), e.sum((0, 1)) + (R * H + 64) * U * np.abs(v).sum((0, 1)) + 1e-37)
    return out


# ----------------------------------------------------------------------------- linear attention

def attention(q, k, v, rate=None, state=None, scale=1.0, reset=None, lengths=None, dy=None, dlast=None, prec="fp32"):
    """Step by step -> dict name -> (value, bound) of y, last and, with dy or dlast, dq, dk, dv, dstate.

    The bounds: a result is a sum of products of three numbers and a weight, in whatever order; each of some
    additions, and the weights' exponentials, adds a U of the sum of the products' magnitudes."""
    B, T, H, K = q.shape
    V = v.shape[3]
    rate = np.zeros(H) if rate is None else rate
    d = np.exp(-rate)[None, :, None, None]
    keep = np.ones((B, T)) if reset is None else (np.asarray(reset) == 0).astype(float)
    n = np.full(B, T) if lengths is None else np.clip(lengths, 0, T)
    some = U * (2 * K + 2 * V + 192 + 8 * (T // 64))
    split = SPLIT if prec == "bf16" else 0.0
    zero = np.zeros((B, H, K, V))
    S = zero.copy() if state is None else state.copy()
    A = np.abs(S)
    states, sizes = np.zeros((T, B, H, K, V)), np.zeros((T, B, H, K, V))
    y, ey = np.zeros((B, T, H, V)), np.zeros((B, T, H, V))
    on = np.arange(T)[None] < n[:, None]
    q, k, v = (np.where(on[..., None, None], x, 0.0) for x in (q, k, v))
    for t in range(T):
        live = on[:, t, None, None, None]
        cut = keep[:, t, None, None, None] == 0
        S = np.where(live, np.where(cut, 0.0, d * S) + k[:, t, :, :, None] * v[:, t, :, None], S)
        A = np.where(live, np.where(cut, 0.0, d * A) + np.abs(k[:, t, :, :, None] * v[:, t, :, None]), A)
        states[t], sizes[t] = S, A
        y[:, t] = np.where(on[:, t, None, None], scale * (q[:, t, :, :, None] * S).sum(2), 0.0)
        ey[:, t] = np.where(on[:, t, None, None], (some + split) * abs(scale) * (np.abs(q[:, t, :, :, None]) * A).sum(2), 0.0)
    out = {"y": (y, ey), "last": (S, some * A)}
    if dy is None and dlast is None:
        return out
    dy = np.zeros((B, T, H, V)) if dy is None else np.where(on[..., None, None], dy, 0.0)
    C = zero.copy() if dlast is None else dlast.copy()
    D = np.abs(C)
    g = {m: np.zeros((B, T, H, w)) for m, w in (("dq", K), ("dk", K), ("dv", V), ("eq", K), ("ek", K), ("ev", V))}
    for t in range(T - 1, -1, -1):
        live = on[:, t, None, None, None]
        flat = on[:, t, None, None]
        G = C + scale * q[:, t, :, :, None] * dy[:, t, :, None]
        E = D + np.abs(scale * q[:, t, :, :, None] * dy[:, t, :, None])
        g["dq"][:, t] = np.where(flat, scale * (states[t] * dy[:, t, :, None]).sum(3), 0.0)
        g["eq"][:, t] = np.where(flat, abs(scale) * (sizes[t] * np.abs(dy[:, t, :, None])).sum(3), 0.0)
        g["dk"][:, t] = np.where(flat, (G * v[:, t, :, None]).sum(3), 0.0)
        g["ek"][:, t] = np.where(flat, (E * np.abs(v[:, t, :, None])).sum(3), 0.0)
        g["dv"][:, t] = np.where(flat, (G * k[:, t, :, :, None]).sum(2), 0.0)
        g["ev"][:, t] = np.where(flat, (E * np.abs(k[:, t, :, :, None])).sum(2), 0.0)
        cut = keep[:, t, None, None, None] == 0
        C = np.where(live, np.where(cut, 0.0, d * G), C)
        D = np.where(live, np.where(cut, 0.0, d * E), D)
    for m in "qkv":
        out["d" + m] = (g["d" + m], (some + split) * g["e" + m])
    out["dstate"] = (C, some * D)
    return out


# ----------------------------------------------------------------------------- AdamW

def moment_words(elements, seed, t):
    """The 16-bit words of m and of v for these places in the moments, by the published generator (SC'11)."""
    u = np.uint64
    low = u(0xFFFFFFFF)
    e = np.asarray(elements, np.uint64)
    i = e >> u(2)
    c = [i & low, np.full(len(e), t & 0xFFFFFFFF, np.uint64), u(6) + ((i >> u(32)) << u(8)), np.zeros(len(e), np.uint64)]
    k0, k1 = seed & 0xFFFFFFFF, seed >> 32
    for _ in range(10):
        p, q = c[0] * u(0xD2511F53), c[2] * u(0xCD9E8D57)
        c = [(q >> u(32)) ^ c[1] ^ u(k0), q & low, (p >> u(32)) ^ c[3] ^ u(k1), p & low]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    w = np.stack(c, 1)[np.arange(len(e)), (e & u(3)).astype(int)]
    return (w & u(0xFFFF)).astype(np.int64), (w >> u(16)).astype(np.int64)


def e4m3(codes):
    """The values of e4m3 codes (uint8)."""
    c = np.asarray(codes).astype(int)
    e, m = (c >> 3) & 15, c & 7
    x = np.where(e > 0, (1 + m / 8.0) * 2.0 ** (e - 7.0), m / 8.0 * 2.0 ** -6)
    x = np.where((c & 127) == 127, np.nan, x)
    return np.where(c & 128, -x, x)


def round_random(x, words):
    """x >= 0 (float64, at most 448) up or down to a value of e4m3 by the words."""
    x = np.minimum(x, 448.0).astype(np.float32)
    low = x < np.float32(2.0 ** -6)
    bits = np.where(low, x + np.float32(2.0 ** -6), x).view(np.uint32).astype(np.int64)
    z = ((bits + (words << 4) + 8) & 0xFFF00000).astype(np.uint32).view(np.float32)
    return np.where(low, z - np.float32(2.0 ** -6), z).astype(float)


def adamw(p, g, m, v, t, lr, beta1, beta2, eps, decay):
    """The step of one tensor in float64 -> dict of p, m, v, r (the root of v): (value, bound)."""
    m1, v1 = beta1 * m + (1 - beta1) * g, beta2 * v + (1 - beta2) * g * g
    em = 4 * U * (np.abs(beta1 * m) + np.abs((1 - beta1) * g)) + 1e-44
    ev = 6 * U * (beta2 * v + (1 - beta2) * g * g) + 1e-44
    r = np.sqrt(v1)
    er = np.where(r > 0, ev / np.maximum(r, 1e-30), np.sqrt(ev)) / 2 + 2 * U * r
    up, down = m1 / (1 - beta1 ** t), r / np.sqrt(1 - beta2 ** t) + eps
    with np.errstate(all="ignore"):
        step = up / down
        estep = np.abs(step) * (8 * U + (er / np.sqrt(1 - beta2 ** t)) / down) + em / (1 - beta1 ** t) / down
    new = p - lr * (step + decay * p)
    ep = lr * (estep + 4 * U * (np.abs(step) + np.abs(decay * p))) + 2 * U * np.abs(p)
    return {"p": (new, ep), "m": (m1, em), "v": (v1, ev), "r": (r, er)}
