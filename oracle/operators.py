"""Slow float64 statements of the sequence and residual operators (gated linear recurrence, residual step with norms, dropout) with hand-written
backward passes, and magnitudes that bound the rounding errors of a float32 evaluation.  Nothing is rounded here."""
from __future__ import annotations

import numpy as np


def sigmoid(g):
    """sigmoid(g) and 1 - sigmoid(g), both without cancellation."""
    with np.errstate(over="ignore"):
        e = np.exp(-np.abs(g))
    small, big = e / (1 + e), 1 / (1 + e)
    return np.where(g < 0, small, big), np.where(g < 0, big, small)


# ------------------------------------------------------------------------------------------------ gated linear recurrence
def recurrence_forward(x, gate, y0, lengths, coupled):
    """x, gate [B, T, D]; y0 [B, D].  Returns y [B, T, D] (zero behind a length), yT [B, D] and the same recurrence of absolute values."""
    B, T, D = x.shape
    b, a = sigmoid(gate)
    y, mag = np.zeros((B, T, D)), np.zeros((B, T, D))
    yT, magT = np.array(y0, dtype=np.float64), np.abs(y0)
    for s in range(B):
        for t in range(int(lengths[s])):
            w = b[s, t] if coupled else 1.0
            yT[s] = np.where(a[s, t] == 0, 0, a[s, t] * yT[s]) + w * x[s, t]
            magT[s] = a[s, t] * magT[s] + w * np.abs(x[s, t])
            y[s, t], mag[s, t] = yT[s], magT[s]
    return y, yT, mag, magT


def recurrence_backward(x, gate, y, dy, dyT, y0, lengths, coupled):
    """Gradients at the given trajectory y.  Returns dx, dg [B, T, D] (zero behind a length), dy0 and magnitudes of the adjoint [B, T, D], [B, D]."""
    B, T, D = x.shape
    b, a = sigmoid(gate)
    dx, dg, lmag = np.zeros((B, T, D)), np.zeros((B, T, D)), np.zeros((B, T, D))
    r, rmag = np.array(dyT, dtype=np.float64), np.abs(dyT)
    for s in range(B):
        for t in range(int(lengths[s]) - 1, -1, -1):
            l, lm = dy[s, t] + r[s], np.abs(dy[s, t]) + rmag[s]
            before = y[s, t - 1] if t > 0 else y0[s]
            dx[s, t] = b[s, t] * l if coupled else l
            dg[s, t] = l * a[s, t] * b[s, t] * (x[s, t] - before if coupled else -before)
            lmag[s, t] = lm
            r[s], rmag[s] = a[s, t] * l, a[s, t] * lm
    return dx, dg, r, lmag, rmag


# ------------------------------------------------------------------------------------------------ dropout
def philox4x32(counter, key, rounds=10):
    """Philox4x32 (Salmon et al. 2011) in Python integers: four 32-bit words each."""
    c, k = list(counter), list(key)
    for _ in range(rounds):
        p, q = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(q >> 32) ^ c[1] ^ k[0], q & 0xffffffff, (p >> 32) ^ c[3] ^ k[1], p & 0xffffffff]
        k = [(k[0] + 0x9E3779B9) & 0xffffffff, (k[1] + 0xBB67AE85) & 0xffffffff]
    return c


def drop_threshold(p):
    return int(float(np.float32(p)) * 65536 + 0.5)


def drop_factors(rows, width, p, seed, step, site, first_row=0):
    """[rows, width]: 0 where dropped, the kept elements' factor elsewhere."""
    thr, groups = drop_threshold(p), (width + 7) // 8
    out = np.zeros((rows, groups * 8))
    for r in range(rows):
        for j in range(groups):
            G = (first_row + r) * groups + j
            w = philox4x32([G & 0xffffffff, G >> 32, step & 0xffffffff, site], [seed & 0xffffffff, (seed >> 32) & 0xffffffff])
            for i in range(8):
                bits = (w[i // 2] >> (16 * (i % 2))) & 0xffff
                out[r, 8 * j + i] = 65536.0 / (65536 - thr) if bits >= thr else 0.0
    return out[:, :width]


# ------------------------------------------------------------------------------------------------ residual step
def norm(v, kind, eps):
    """(normalised rows, mean [M], 1 / deviation [M])."""
    M = v.shape[0]
    if kind == "none":
        return v, np.zeros(M), np.ones(M)
    mean = v.mean(1) if kind == "meanvar" else np.zeros(M)
    d = v - mean[:, None]
    rstd = 1 / np.sqrt((d * d).mean(1) + eps)
    return d * rstd[:, None], mean, rstd


def norm_backward(dn, n, rstd, kind):
    if kind == "none":
        return dn
    out = dn - n * (dn * n).mean(1, keepdims=True)
    if kind == "meanvar":
        out = out - dn.mean(1, keepdims=True)
    return out * rstd[:, None]


def residual_forward(y, u, gate, w_post, scale, w_pre, h, post, pre, eps, factors):
    """Returns y', z and stats [M, 4]; u may be None, the weights and `factors` (dropout) arrays of ones."""
    M = y.shape[0]
    mu, ru = np.zeros(M), np.ones(M)
    if u is not None:
        n, mu, ru = norm(u, post, eps)
        v = n * w_post * (sigmoid(gate)[0] if gate is not None else 1.0)
        y = y + np.where(factors == 0, 0, h * scale * v * factors)
    n, my, ry = norm(y, pre, eps)
    return y, n * w_pre, np.stack([mu, ru, my, ry], 1)


def residual_backward(y_new, u, gate, w_post, scale, w_pre, h, post, pre, eps, factors, dy, dz):
    """Gradients of <dy, y'> + <dz, z> with respect to y, u, gate and the weights, at the given y' = y_new."""
    n2, _, ry = norm(y_new, pre, eps)
    a = dy + norm_backward(dz * w_pre, n2, ry, pre)
    out = dict(dy=a, dw_pre=(dz * n2).sum(0))
    if u is None:
        return out
    n, _, ru = norm(u, post, eps)
    sig, cosig = sigmoid(gate) if gate is not None else (1.0, 0.0)
    t = np.where(factors == 0, 0, h * a * factors)
    out["dscale"] = (t * n * w_post * sig).sum(0)
    t = t * scale
    if gate is not None:
        out["dgate"] = t * n * w_post * sig * cosig
    t = t * sig
    out["dw_post"] = (t * n).sum(0)
    out["du"] = norm_backward(t * w_post, n, ru, post)
    return out
