"""The recurrent block's operators in float64 numpy, from their formulas, with error bounds.

Each value comes with a bound on what float32 arithmetic may be off from it, carried through the same
formulas: U is float32's unit roundoff, and every elementary step adds a few U of the
magnitudes it combines (sigmoids: 8 U relative, for two hardware functions of 1 ulp each and the
roundings around them). `rounded` adds the output type's own half ulp.
"""
import numpy as np

U = 2.0 ** -24
HALF_ULP = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -9}


def rounded(value, bound, prec):
    """Bound after the one rounding of an output to `prec` (1e-37: below the normal range)."""
    return bound + HALF_ULP[prec] * (np.abs(value) + bound) * 1.0001 + 1e-37


def sigmoid(x):
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-x)), 1.0 / (1.0 + np.exp(x))


def scan(f, v, h0=None, reset=None, lengths=None, dy=None, dhT=None):
    """-> dict name -> (value, bound) of y, hT, df, dv, dh0 for float64 [B, T, D] inputs."""
    B, T, D = f.shape
    keep = np.ones((B, T)) if reset is None else (np.asarray(reset) == 0).astype(float)
    n = np.full(B, T) if lengths is None else np.clip(lengths, 0, T)
    zero = np.zeros((B, D))
    h, eh = (zero if h0 is None else h0).copy(), zero.copy()
    a, b = sigmoid(f)
    y, ey, before, eb = np.zeros_like(f), np.zeros_like(f), np.zeros_like(f), np.zeros_like(f)
    for t in range(T):
        on = (t < n)[:, None]
        k = keep[:, t, None] != 0
        before[:, t], eb[:, t] = np.where(k, h, 0.0), np.where(k, eh, 0.0)
        vt = np.where(on, v[:, t], 0.0)
        new = a[:, t] * before[:, t] + b[:, t] * vt
        enew = a[:, t] * eb[:, t] + 12 * U * (a[:, t] * np.abs(before[:, t]) + b[:, t] * np.abs(vt))
        h, eh = np.where(on, new, h), np.where(on, enew, eh)
        y[:, t], ey[:, t] = np.where(on, new, 0.0), np.where(on, enew, 0.0)
    out = {"y": (y, ey), "hT": (h, eh)}
    if dy is None and dhT is None:
        return out
    c, ec = (zero if dhT is None else dhT).copy(), zero.copy()
    df, edf, dv, edv = (np.zeros_like(f) for _ in range(4))
    for t in range(T - 1, -1, -1):
        on = (t < n)[:, None]
        k = keep[:, t, None] != 0
        d = np.where(on, 0.0 if dy is None else dy[:, t], 0.0)
        vt = np.where(on, v[:, t], 0.0)
        g = d + c
        eg = ec + 2 * U * np.abs(g)
        gap = before[:, t] - vt
        dv[:, t] = np.where(on, g * b[:, t], 0.0)
        edv[:, t] = np.where(on, eg * b[:, t] + 16 * U * np.abs(g) * b[:, t], 0.0)
        df[:, t] = np.where(on, g * a[:, t] * b[:, t] * gap, 0.0)
        s = a[:, t] * b[:, t]
        edf[:, t] = np.where(on, s * (np.abs(gap) * eg + (np.abs(g) + eg) * (eb[:, t] + 2 * U * (np.abs(before[:, t]) + np.abs(vt))))
                             + 32 * U * np.abs(df[:, t]), 0.0)
        cn = np.where(k, a[:, t] * g, 0.0)
        ecn = np.where(k, a[:, t] * eg + 16 * U * a[:, t] * np.abs(g), 0.0)
        c, ec = np.where(on, cn, c), np.where(on, ecn, ec)
    out.update(df=(df, edf), dv=(dv, edv), dh0=(c, ec))
    return out


def philox16(n, seed, step, tensor):
    """The first n 16-bit words of dropout's stream, by the published generator (SC'11)."""
    m = (n + 7) // 8
    u = np.uint64
    low = u(0xFFFFFFFF)
    i = np.arange(m, dtype=np.uint64)
    c = [i & low, np.full(m, step, np.uint64), u(5) + ((i >> u(32)) << u(8)), np.full(m, tensor, np.uint64)]
    k0, k1 = seed & 0xFFFFFFFF, seed >> 32
    for _ in range(10):
        p, q = c[0] * u(0xD2511F53), c[2] * u(0xCD9E8D57)
        c = [(q >> u(32)) ^ c[1] ^ u(k0), q & low, (p >> u(32)) ^ c[3] ^ u(k1), p & low]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    w = np.stack(c, 1)
    return np.stack([w & u(0xFFFF), w >> u(16)], 2).reshape(-1)[:n].astype(np.int64)


def drop_factor(shape, p, seed, step, tensor):
    d = round(float(np.float32(p)) * 65536)
    keep = philox16(int(np.prod(shape)), seed, step, tensor).reshape(shape) >= d
    return np.where(keep, 65536.0 / (65536 - d) if d < 65536 else 0.0, 0.0)


def _norm(x, kind, eps):
    if kind == "none":
        return x, np.ones((len(x), 1))
    c = x - x.mean(1, keepdims=True) if kind == "layer" else x
    r = 1.0 / np.sqrt((c * c).mean(1, keepdims=True) + eps)
    return c * r, r


def _norm_back(dn, n, r, kind):
    if kind == "none":
        return dn
    t = dn - n * (dn * n).mean(1, keepdims=True)
    return r * (t - dn.mean(1, keepdims=True) if kind == "layer" else t)


def gate(z, kind):
    if kind == "none":
        return np.ones_like(z), np.zeros_like(z)
    s, t = sigmoid(z)
    return (s, s * t) if kind == "sigmoid" else (z * s, s * (1.0 + z * t))


def block_norm(x, h=None, z=None, w_post=None, b_post=None, scale=None, w_pre=None, b_pre=None, post="rms", pre="rms",
               gate_kind="none", eps=1e-6, factor=None, valid=None, dx_out=None, du=None):
    """-> dict name -> (value, bound) of x_out, u and, with dx_out or du, all gradients."""
    R, D = x.shape
    live = np.ones(R, bool) if valid is None else np.asarray(valid) != 0
    row = live[:, None]
    one, zero = np.ones(D), np.zeros(D)
    wq, bq = (one if w_post is None else w_post), (zero if b_post is None else b_post)
    wp, bp, sc = (one if w_pre is None else w_pre), (zero if b_pre is None else b_pre), (one if scale is None else scale)
    x = np.where(row, x, 0.0)
    K = 64 * U   # statistics of up to some ten thousand columns in partial sums of a few dozen, and their use
    if h is not None:
        h = np.where(row, h, 0.0)
        n, rh = _norm(h, post, eps)
        en = K * (np.abs(n) + np.abs(h).max(1, keepdims=True) * rh) if post != "none" else 0.0 * n
        t = n * wq + bq if post != "none" else n
        et = np.abs(wq) * en + K * (np.abs(n * wq) + np.abs(bq)) if post != "none" else en
        gt, slope = gate(np.where(row, z, 0.0) if z is not None else np.zeros_like(x), gate_kind)
        f = np.ones_like(x) if factor is None else factor
        o = f * gt * t
        eo = f * np.abs(gt) * (et + K * np.abs(t))
        xo = x + sc * o
        ex = np.abs(sc) * eo + 4 * U * (np.abs(x) + np.abs(sc * o))
    else:
        xo, ex = x, np.zeros_like(x)
    m, rx = _norm(xo, pre, eps)
    em = rx * ex + K * (np.abs(m) + np.abs(xo).max(1, keepdims=True) * rx)
    em = em + (np.abs(m) + 1.0) * (ex * rx).max(1, keepdims=True)
    out = {"x_out": (xo * row, ex * row)}
    if pre != "none":
        out["u"] = ((m * wp + bp) * row, (np.abs(wp) * em + K * (np.abs(m * wp) + np.abs(bp))) * row)
    if dx_out is None and du is None:
        return out
    dxo = np.where(row, np.zeros_like(x) if dx_out is None else dx_out, 0.0)
    du = np.where(row, np.zeros_like(x) if du is None or pre == "none" else du, 0.0)
    back = _norm_back(du * wp, m, rx, pre) if pre != "none" else 0.0 * x
    d = dxo + back
    # Gradients: each a sum of products of a row's values; bounded by 256 U (and the relative error of the
    # normalised values) times the largest magnitude that enters it in the row.
    rel = 256 * U + (em.max(1, keepdims=True) / (1e-30 + np.abs(m).max(1, keepdims=True)) if pre != "none" else 0.0)
    size_d = np.abs(dxo) + rx * (np.abs(du * wp) + (1 + np.abs(m)) * np.abs(du * wp * (1 + np.abs(m))).mean(1, keepdims=True))
    ed = 4 * rel * (size_d if pre != "none" else np.abs(dxo))
    out["dx"] = (d * row, ed * row)
    sums = {"dw_pre": (du * m, np.abs(du) * em), "db_pre": (du, 0.0 * du)}
    if h is not None:
        gd = d * f
        eg = ed * f
        do = gd * sc
        dz = do * t * slope
        ez = np.abs(sc * slope) * (np.abs(t) * eg + np.abs(gd) * et) + 256 * U * np.abs(do * t) * (1 + np.abs(slope))
        dt = do * gt
        edt = np.abs(sc * gt) * eg + 256 * U * np.abs(dt)
        dn = dt * wq if post != "none" else dt
        edn = edt * np.abs(wq) if post != "none" else edt
        rel_h = 256 * U + (en.max(1, keepdims=True) / (1e-30 + np.abs(n).max(1, keepdims=True)) if post != "none" else 0.0)
        big = lambda q: rh * (q + (1 + np.abs(n)) * (q * (1 + np.abs(n))).mean(1, keepdims=True)) if post != "none" else q
        out["dh"] = (_norm_back(dn, n, rh, post) * row, (4 * rel_h * big(np.abs(dn)) + big(edn)) * row)
        if gate_kind != "none":
            out["dz"] = (dz * row, ez * row)
        sums.update(dw_post=(dt * n, np.abs(n) * edt + np.abs(dt) * en), db_post=(dt, edt),
                    dscale=(gd * gt * t, np.abs(gt * t) * eg + np.abs(gd * gt) * (et + K * np.abs(t))))
    for k, (v, e) in sums.items():
        v, e = v * row, e * row
        out[k] = (v.sum(0), e.sum(0) + (R + 64) * U * np.abs(v).sum(0) + 1e-37)
    return out


def quant_rows(x):
    """float32 rows -> (q, scale): the scale is a float32 number, the largest magnitude times the float32
    next to 1 / 127; the quotient rounds to float32 before it rounds to an integer, as the operator states it."""
    m = np.abs(x).max(1) if x.shape[1] else np.zeros(len(x), np.float32)
    s = (m.astype(np.float32) * (np.float32(1.0) / np.float32(127.0))).astype(np.float32)
    q = np.zeros(x.shape)
    with np.errstate(all="ignore"):
        on = s > 0
        on &= np.isfinite(m)
        q[on] = np.clip(np.rint((x[on].astype(np.float32) / s[on][:, None]).astype(np.float32)), -127, 127)
    return q, np.where(np.isfinite(m), s, np.float32("nan"))
