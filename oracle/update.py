"""CPU oracle of what closes a policy update: the draw from given numbers, the gradient of the objective, AdamW - TEST
INFRASTRUCTURE, not a product path.  Everything is float64; each function says what it computes."""
from __future__ import annotations

import numpy as np

BLOCK = 256
E4M3_MAX, E4M3_LEAST = 448.0, 2.0 ** -9
TINY = float(np.float32(1e-30))


# ------------------------------------------------------------------------------------------------ draw
def weights_of(row, temperature):
    """exp((l - max l) / T), T in the 32 bits in which calls give it, 1 for every largest logit; T = 0: 1 for those and 0 for the rest.  None: nothing can be drawn."""
    x = np.asarray(row, dtype=np.float64).copy()
    x[np.isnan(x)] = -np.inf
    m = x.max()
    if m == -np.inf:
        return None, x
    if temperature == 0:
        return (x == m).astype(np.float64), x
    with np.errstate(invalid="ignore", over="ignore"):
        w = np.exp((x - m) / float(np.float32(temperature)))
    return np.where(x == m, 1.0, np.nan_to_num(w, nan=0.0)), x


def draw_row(row, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, logp, slack).  slack: how near, relative to the kept mass, the draw or a cut came to a border at which another order of
    additions may decide otherwise."""
    w, x = weights_of(row, temperature)
    V = len(x)
    if w is None:
        return 0, -np.inf, np.inf
    if temperature == 0:
        return int(np.argmax(w)), 0.0, np.inf
    keep = np.ones(V, dtype=bool)
    slack = np.inf
    if 0 < top_k < V:
        keep &= x >= np.sort(x)[V - top_k]
    if top_p < 1:
        values = np.unique(x[keep])[::-1]
        mass = np.array([w[keep & (x == t)].sum() for t in values]) if len(values) < 64 else \
            np.bincount(np.searchsorted(-values, -x[keep]), weights=w[keep], minlength=len(values))
        c = mass.cumsum()
        target = float(np.float32(top_p)) * c[-1]
        at = int(np.argmax(c >= target))
        below = c[at - 1] if at else 0.0
        # the two sides of the cut; one that is exactly on it (equal weights) is decided alike by exact sums
        slack = min([abs(d) for d in (c[at] - target, target - below) if d != 0.0] + [np.inf]) / c[-1]
        keep &= x >= values[at]
    if min_p > 0:
        keep &= w >= float(np.float32(min_p))
    kw = np.where(keep, w, 0.0)
    c = kw.cumsum()
    u = min(max(float(u) if u == u else 0.0, 0.0), float(np.float32(0.99999994)))
    target = u * c[-1]
    tok = int(np.argmax(c > target))
    near = np.abs(np.concatenate([c[max(tok - 1, 0):tok], c[tok:tok + 1]]) - target)
    if target > 0:
        slack = min(slack, near.min() / c[-1])
    return tok, float(np.log(kw[tok]) - np.log(c[-1])), slack


# ------------------------------------------------------------------------------------------------ policy gradient
def objective(logits, targets, logp_old, adv, mask, temperature, clip_eps):
    """(J, logp, slope dJ/dlogp): rows that do not count have logp 0 and slope 0."""
    z = np.asarray(logits, dtype=np.float64) / float(temperature)
    n, V = z.shape
    logp, slope, J = np.zeros(n), np.zeros(n), 0.0
    for t in range(n):
        if targets[t] < 0 or (mask is not None and mask[t] == 0):
            continue
        m = z[t].max()
        with np.errstate(invalid="ignore"):
            lse = m + np.log(np.exp(z[t] - m).sum())
            logp[t] = z[t, targets[t]] - lse if targets[t] < V else np.nan
        A = float(adv[t])
        if logp_old is None:
            J, slope[t] = J + A * logp[t], A
            continue
        r = np.exp(logp[t] - float(logp_old[t]))
        rc = min(max(r, 1.0 - clip_eps), 1.0 + clip_eps) if r == r else r
        J += min(r * A, rc * A)
        slope[t] = r * A if r * A <= rc * A else 0.0 if r == r else np.nan
    return J, logp, slope


def policy_gradient(logits, targets, logp_old, adv, mask, temperature, clip_eps, scale):
    """(logp, gradient of -scale J in the logits, softmax, slope of -scale J)"""
    _, logp, slope = objective(logits, targets, logp_old, adv, mask, temperature, clip_eps)
    z = np.asarray(logits, dtype=np.float64) / float(temperature)
    with np.errstate(invalid="ignore"):
        p = np.exp(z - z.max(axis=1, keepdims=True))
        p /= p.sum(axis=1, keepdims=True)
    live = np.array([targets[t] >= 0 and (mask is None or mask[t] != 0) for t in range(len(targets))])
    p[~live] = 0.0
    s = scale * slope / float(temperature)
    grad = s[:, None] * p
    for t in np.flatnonzero(live):
        if targets[t] < z.shape[1]:
            grad[t, targets[t]] -= s[t]
    return logp, grad, p, s


# ------------------------------------------------------------------------------------------------ AdamW
def e4m3_value(code):
    """Values of 8-bit floats: sign, 4 exponent bits (bias 7), 3 mantissa bits; no infinities, 0x7F and 0xFF undefined."""
    c = np.asarray(code).astype(np.int64)
    e, f = (c >> 3) & 15, c & 7
    v = np.where(e == 0, f * 2.0 ** -9, (8 + f) * 2.0 ** (e - 10.0))
    v = np.where((c & 127) == 127, np.nan, v)
    return np.where(c & 128, -v, v)


def decode_state(codes, scale):
    n = len(codes)
    return e4m3_value(codes) * np.repeat(np.asarray(scale, dtype=np.float64), BLOCK)[:n]


def block_scale(x):
    """(what a block's codes are multiples of, the same for every element), from unrounded values"""
    n = len(x)
    pad = np.concatenate([np.abs(x), np.zeros(-n % BLOCK)]).reshape(-1, BLOCK).max(axis=1)
    s = np.where(pad > TINY, pad / E4M3_MAX, 0.0)
    return s, np.repeat(s, BLOCK)[:n]


def encode_off_by(x, scale_of):
    """How far a code's value may be from x: half a step of 4 significant bits, 2^-10 of the scale below 2^-6 of it."""
    with np.errstate(divide="ignore"):
        e = np.floor(np.log2(np.maximum(np.abs(x), 1e-300) / np.maximum(scale_of, 1e-300)))
    return scale_of * 2.0 ** (np.maximum(e, -6.0) - 4.0)


def adamw(tensors, lr, beta1, beta2, eps, weight_decay, step, grad_scale=1.0, max_norm=0.0):
    """tensors: dicts with p, g, m, v (float64 values) and decay.  -> (new dicts with p, m, v, their update, the norm)"""
    norm = np.sqrt(sum(float(((t["g"] * grad_scale) ** 2).sum()) for t in tensors))
    c = max_norm / norm if max_norm > 0 and norm > max_norm else 1.0
    out = []
    for t in tensors:
        g = t["g"] * grad_scale * c
        m = beta1 * t["m"] + (1 - beta1) * g
        v = beta2 * t["v"] + (1 - beta2) * g * g
        upd = lr * (m / (1 - beta1 ** step)) / (np.sqrt(v / (1 - beta2 ** step)) + eps)
        out.append({"p": t["p"] * (1 - lr * weight_decay * t["decay"]) - upd, "m": m, "v": v, "update": upd, "g": g})
    return out, norm
