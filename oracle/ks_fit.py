"""fp64 oracle of fitting gated efficiency heads (test infrastructure, like
``ks_oracle``; no code shared with the HIP library).

The gated block per family, z = w3 . (silu(W1 x) * (W2 x)) + b3; its gradients;
the loss on log eta (Sec. 5.3 trains the heads on log eta of measured kernels);
the AdamW step with states in 32 or 8 bits.  Beside values, ``block`` and
``gradients`` return bounds on what fp32 arithmetic in any order may be off."""
from __future__ import annotations

import numpy as np

EPS = 2.0 ** -24          # half a step of fp32, relative


def sigmoid(v):
    v = np.asarray(v, np.float64)
    e = np.exp(-np.abs(v))
    return np.where(v >= 0, 1.0 / (1.0 + e), e / (1.0 + e))


def block(x, w1, w2, w3, b3):
    """One family's rows: z and a dict of what the gradients need.  "err": bounds
    on the fp32 error of g, u, s, a and z.

    A projection of D products: D roundings of partial sums below the sum of
    magnitudes, and 2^-24 of each product (pieces left out).  s = 1 / (1 + 2^(-g log2 e)): the exponent is rounded twice (the
    constant and the product: relative 2 EPS of |g| log2 e, a relative
    2 |g| EPS of e^-g), the exponential and the reciprocal are within 2 EPS (one unit
    of the last place), the sum within EPS; the exponential's error counts (1 - s)."""
    x, w1, w2, w3 = (np.asarray(v, np.float64) for v in (x, w1, w2, w3))
    D, H = w1.shape[1], w1.shape[0]
    g, u = x @ w1.T, x @ w2.T
    eg, eu = ((D + 1) * EPS * (np.abs(x) @ np.abs(w).T) for w in (w1, w2))
    s = sigmoid(g)
    a = g * s
    es = s * ((1 - s) * (2 * np.abs(g) + 2) * EPS + 4 * EPS) + eg / 4      # |ds/dg| <= 1/4
    ea = np.abs(a) * ((1 - s) * (2 * np.abs(g) + 2) + 6) * EPS + 1.1 * eg    # |da/dg| <= 1.1
    y = a * u
    ey = ea * np.abs(u) + np.abs(a) * eu + ea * eu + 2 * EPS * np.abs(y)
    z = y @ w3 + b3
    ez = ey @ np.abs(w3) + (H + 2) * EPS * (np.abs(y) @ np.abs(w3) + abs(float(b3)))
    return z, {"g": g, "u": u, "s": s, "a": a, "y": y, "err": {"g": eg, "u": eu, "s": es, "a": ea, "y": ey, "z": ez}}


def gradients(x, w1, w2, w3, dz, k, terms):
    """Gradients of sum dz z from ``block``'s dict k: w1, w2, w3, b3, x, and bounds on
    their fp32 errors.  terms: additions in fp32 that one sum over rows goes through
    in a row.  What a unit makes of a row is summed in three exact pieces; the products
    of pieces left out are at most 2 2^-9 2^-16 = 2^-24 of it (a second piece is at most
    2^-9 of the number, the third 2^-7 of the second).  Rows whose dz is 0 add nothing, whatever
    they hold."""
    dz = np.asarray(dz, np.float64)
    on = dz != 0
    x = np.where(on[:, None], np.asarray(x, np.float64), 0.0)
    w1, w2, w3 = (np.asarray(v, np.float64) for v in (w1, w2, w3))
    z0 = {n: np.where(on[:, None], k[n], 0.0) for n in ("g", "u", "s", "a", "y")}
    e0 = {n: np.where(on[:, None], k["err"][n], 0.0) for n in ("g", "u", "s", "a", "y")}
    u, s, a, y = (z0[n] for n in ("u", "s", "a", "y"))
    t = s + a * (1 - s)                                   # silu'
    et = e0["s"] + e0["a"] * (1 - s) + np.abs(a) * e0["s"] + 4 * EPS * (np.abs(s) + np.abs(a))
    dy = dz[:, None] * w3
    du, dg = dy * a, dy * u * t
    edu = np.abs(dy) * e0["a"] + 4 * EPS * np.abs(du)
    edg = np.abs(dy) * (e0["u"] * np.abs(t) + np.abs(u) * et + e0["u"] * et) + 6 * EPS * np.abs(dg)
    val = {"w1": dg.T @ x, "w2": du.T @ x, "w3": (dz[:, None] * y).sum(0), "b3": dz.sum(), "x": dg @ w1 + du @ w2}
    ax, H = np.abs(x), w1.shape[0]
    long = (terms + 8) * EPS + 2.0 ** -24
    # (dw3 may come as W2 . sum dz a x: its terms are dW2's, weighted)
    err = {"w1": edg.T @ ax + long * (np.abs(dg).T @ ax), "w2": edu.T @ ax + long * (np.abs(du).T @ ax),
           "w3": (((np.abs(dz)[:, None] * (e0["a"] + (4 * EPS + long) * np.abs(a))).T @ ax) * np.abs(w2)).sum(1),
           "b3": (terms + 8) * EPS * np.abs(dz).sum(),
           "x": edg @ np.abs(w1) + edu @ np.abs(w2) + (2 * H + 8) * EPS * (np.abs(dg) @ np.abs(w1) + np.abs(du) @ np.abs(w2))}
    return val, err


def counted(eta, weight):
    """The rows' weights, 0 for those without a usable measurement."""
    eta = np.asarray(eta, np.float64)
    w = np.ones(len(eta)) if weight is None else np.asarray(weight, np.float64)
    with np.errstate(invalid="ignore"):
        return np.where(np.isfinite(eta) & (eta > 0) & np.isfinite(w) & (w > 0), w, 0.0)


def eta_loss(z, eta, weight, huber):
    """One family's loss and dz: sum w rho(r) / sum w, r = log(1 + e^-z) - log eta."""
    w = counted(eta, weight)
    if not (w > 0).any():
        return 0.0, np.zeros(len(w))
    on = w > 0
    zz = np.where(on, z, 0.0)
    r = np.logaddexp(0.0, -zz) - np.log(np.where(on, eta, 1.0))
    far = np.abs(r) > huber
    rho = np.where(far, huber * (np.abs(r) - huber / 2) if np.isfinite(huber) else 0.0, r * r / 2)
    slope = np.where(far, huber * np.sign(r) if np.isfinite(huber) else 0.0, r)
    return float((w * rho).sum() / w.sum()), -w / w.sum() * slope * sigmoid(-zz)


# --------------------------------------------------------------------------
# AdamW
# --------------------------------------------------------------------------
def round_to(v, mant, low):
    """Nearest values of a binary format with ``mant`` fraction bits and exponents
    from ``low`` on (below, its subnormals), ties to even; float64."""
    v = np.asarray(v, np.float64)
    _, e = np.frexp(v)
    step = np.ldexp(1.0, np.maximum(e - 1, low) - mant)
    return np.rint(v / step) * step


def encode(v, second):
    """States in 8 bits: the values (in multiples of the block's power of two) and
    the exponent byte of each 64 elements.  second: v (e5m2), else m (e4m3)."""
    v = np.asarray(v, np.float64)
    mant, low, lift = (2, -14, 14) if second else (3, -6, 7)
    n = len(v)
    pad = np.concatenate([v, np.zeros(-n % 64)]).reshape(-1, 64)
    top = np.where(np.isfinite(pad), np.abs(pad), 0.0).max(1)
    _, e = np.frexp(top)
    e = np.where(top > 0, e - 1 + 127 - lift, 1)
    e = np.maximum(e, 1).astype(np.int64)
    q = pad * np.exp2(127.0 - e)[:, None]
    if second:
        q = np.where((pad > 0) & (q < 2.0 ** -16), 2.0 ** -16, q)
    fin = np.isfinite(q)
    out = round_to(np.where(fin, q, 0.0), mant, low)
    out = np.where(fin, out, np.where(np.isposinf(q), np.inf if second else np.nan, np.nan))
    return out.reshape(-1)[:n], e


def decode(q, e, n):
    return (np.concatenate([q, np.zeros(-n % 64)]).reshape(-1, 64) * np.exp2(np.asarray(e, np.float64) - 127)[:, None]).reshape(-1)[:n]


def moments32(m, v, g, grad_scale, beta1, beta2):
    """m and v of the next step in fp32, each product and sum rounded by itself."""
    f = np.float32
    with np.errstate(all="ignore"):
        g = f(g) * f(grad_scale)
        return f(m) * f(beta1) + g * f(1 - beta1), f(v) * f(beta2) + (g * f(1 - beta2)) * g


def step(p, m, v, lr, weight_decay, beta1, beta2, eps, t):
    """The parameter after a step with the moments m, v already moved."""
    p, m, v = (np.asarray(a, np.float64) for a in (p, m, v))
    return p * (1 - lr * weight_decay) - lr * (m / (1 - beta1 ** t)) / (np.sqrt(v / (1 - beta2 ** t)) + eps)
