"""CPU oracle of the learner's operators between a decoder block's matrix products: causal attention over packed sequences, addition with RMSNorm,
norm and rotation of heads, each with its gradient - TEST INFRASTRUCTURE, not a product path.  Everything is float64, straight from the formulas."""
from __future__ import annotations

import numpy as np

E4M3_MAX = 448.0


# ------------------------------------------------------------------------------------------------ attention
def _spans(lens):
    a = 0
    for n in lens:
        yield a, a + int(n)
        a += int(n)


def attention(q, k, v, lens, scale):
    """(out [n, Hq, hd], lse [Hq, n], p: {(sequence, head): [len, len]})."""
    q, k, v = (np.asarray(t, dtype=np.float64) for t in (q, k, v))
    G = q.shape[1] // k.shape[1]
    out, lse, ps = np.zeros_like(q), np.zeros((q.shape[1], q.shape[0])), {}
    with np.errstate(all="ignore"):
        for b, (a, e) in enumerate(_spans(lens)):
            n = e - a
            if not n:
                continue
            for h in range(q.shape[1]):
                p = np.zeros((n, n))
                for i in range(n):                                     # a row sees its own past alone, whatever stands elsewhere
                    s = scale * (k[a:a + i + 1, h // G] @ q[a + i, h])
                    m = s.max()
                    w = np.exp(s - m)
                    lse[h, a + i] = m + np.log(w.sum())
                    p[i, :i + 1] = w / w.sum()
                    out[a + i, h] = p[i, :i + 1] @ v[a:a + i + 1, h // G]
                ps[b, h] = p
    return out, lse, ps


def attention_grad(q, k, v, dout, lens, scale):
    """(dq, dk, dv) and, for error bounds, the same sums over magnitudes."""
    q, k, v, dout = (np.asarray(t, dtype=np.float64) for t in (q, k, v, dout))
    G = q.shape[1] // k.shape[1]
    out, _, ps = attention(q, k, v, lens, scale)
    g = [np.zeros_like(t) for t in (q, k, v)]
    size = [np.zeros_like(t) for t in (q, k, v)]
    with np.errstate(all="ignore"):
        for b, (a, e) in enumerate(_spans(lens)):
            n = e - a
            for h in range(q.shape[1] if n else 0):
                j = h // G
                p, d, o = ps[b, h], dout[a:e, h], out[a:e, h]
                for i in range(n):
                    s = slice(a, a + i + 1)
                    dp = v[s, j] @ d[i]
                    t = p[i, :i + 1] * (dp - d[i] @ o[i])
                    # magnitudes: what the rounding of p, out, dout . v and D can reach
                    w = p[i, :i + 1] * (np.abs(v[s, j]) @ np.abs(d[i]) + np.abs(d[i]) @ np.abs(o[i]))
                    g[0][a + i, h] += scale * (t @ k[s, j])
                    size[0][a + i, h] += scale * (w @ np.abs(k[s, j]))
                    g[1][s, j] += scale * np.outer(t, q[a + i, h])
                    size[1][s, j] += scale * np.outer(w, np.abs(q[a + i, h]))
                    g[2][s, j] += np.outer(p[i, :i + 1], d[i])
                    size[2][s, j] += np.outer(p[i, :i + 1], np.abs(d[i]))
    return g, size


# ------------------------------------------------------------------------------------------------ addition and RMSNorm
def round_e4m3(x):
    """The nearest value of 4 exponent and 3 mantissa bits, ties to even, |x| <= 448."""
    x = np.asarray(x, dtype=np.float64)
    e = np.floor(np.log2(np.maximum(np.abs(x), 2.0 ** -6)))
    step = np.exp2(e - 3)
    return np.round(x / step) * step


def add_rmsnorm(x, residual, gain, eps):
    """(sum, out, rstd)."""
    h = np.asarray(x, dtype=np.float64)
    if residual is not None:
        h = h + np.asarray(residual, dtype=np.float64)
    with np.errstate(all="ignore"):
        rstd = 1.0 / np.sqrt((h * h).mean(axis=1) + float(np.float32(eps)))
        return h, h * rstd[:, None] * np.asarray(gain, dtype=np.float64), rstd


def add_rmsnorm_grad(dout, h, gain, rstd, dsum=None):
    """(dx, dgain)."""
    dout, h, gain, r = (np.asarray(t, dtype=np.float64) for t in (dout, h, gain, rstd))
    u = h * r[:, None]
    a = dout * gain
    dx = r[:, None] * (a - u * (a * u).mean(axis=1, keepdims=True))
    if dsum is not None:
        dx = dx + np.asarray(dsum, dtype=np.float64)
    return dx, (dout * u).sum(axis=0)


# ------------------------------------------------------------------------------------------------ norm and rotation of heads
def _turn(x, positions, theta, sign):
    half = x.shape[-1] // 2
    angle = np.asarray(positions, dtype=np.float64)[:, None] * theta ** (-2.0 * np.arange(half) / (2 * half))
    c, s = np.cos(angle)[:, None], sign * np.sin(angle)[:, None]
    lo, hi = x[..., :half], x[..., half:]
    return np.concatenate([lo * c - hi * s, hi * c + lo * s], axis=-1)


def norm_rope(x, gain, eps, theta, positions):
    """x: [n, heads, hd]; gain None: rotation alone."""
    n = np.asarray(x, dtype=np.float64)
    if gain is not None:
        n = n / np.sqrt((n * n).mean(axis=-1, keepdims=True) + float(np.float32(eps))) * np.asarray(gain, dtype=np.float64)
    return _turn(n, positions, theta, 1.0)


def norm_rope_grad(x, dout, gain, eps, theta, positions):
    """(dx, dgain or None)."""
    d = _turn(np.asarray(dout, dtype=np.float64), positions, theta, -1.0)
    if gain is None:
        return d, None
    x, gain = np.asarray(x, dtype=np.float64), np.asarray(gain, dtype=np.float64)
    r = 1.0 / np.sqrt((x * x).mean(axis=-1, keepdims=True) + float(np.float32(eps)))
    u = x * r
    a = d * gain
    return r * (a - u * (a * u).mean(axis=-1, keepdims=True)), (d * u).sum(axis=(0, 1))
