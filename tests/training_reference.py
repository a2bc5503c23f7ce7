"""Rotary positions with head norms, cross entropy and AdamW in 64 bits on the CPU, from their definitions, with bounds of what the kernels may be off.

The bounds count the kernels' roundings: u is half a unit in the last place of the storage type, relative, EPS that of fp32 (2^-24).  fp32 sums of n terms are within n EPS of
the sum of the terms' magnitudes."""
from __future__ import annotations

import numpy as np

from operator_reference import EPS, TINY, U


# ------------------------------------------------------------------ rotary
def tokens(batch, length, positions=None, starts=None, lens=None):
    """(counts, position, place) of every token."""
    i = np.arange(length)[None, :].repeat(batch, 0)
    counts = np.ones((batch, length), bool) if lens is None else i < np.clip(np.asarray(lens), 0, length)[:, None]
    place = i if starts is None else i + np.asarray(starts, np.int64)[:, None]
    return counts, place if positions is None else np.asarray(positions, np.int64), place


def pairs_of(rotated, neighbours):
    j = np.arange(rotated // 2)
    return (2 * j, 2 * j + 1) if neighbours else (j, rotated // 2 + j)


def turned(x, angle, neighbours):
    """x [...][heads][head_dim], angle [...][pairs]"""
    a, b = pairs_of(2 * angle.shape[-1], neighbours)
    c, s = np.cos(angle)[..., None, :], np.sin(angle)[..., None, :]
    y = x.copy()
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
    return y


def spread(x, rotated, neighbours):
    """The magnitudes that went into each element of a turned head."""
    a, b = pairs_of(rotated, neighbours)
    y = np.abs(x)
    both = y[..., a] + y[..., b]
    y[..., a] = y[..., b] = both
    return y


def head_norm(x, kind, eps):
    if kind == "none":
        return x, np.ones(x.shape[:-1] + (1,))
    x = x - x.mean(-1, keepdims=True) if kind == "layer" else x
    dev = np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    return x / dev, dev


def rotary(x, angle, *, neighbours, norm, eps, weight=None, bias=None, dtype, d=None, there=None):
    """Of queries or keys [batch][length][heads][head_dim]: {name: (values, bounds)} of "y" and, with the gradient d of it, of "dx", "weight" and "bias"; `there`
    [batch][length]: which tokens have a part in the sums."""
    D, rotated = x.shape[-1], 2 * angle.shape[-1]
    u = U[dtype]
    hat, dev = head_norm(x, norm, eps)
    w, b = (np.ones(D) if weight is None else weight), (np.zeros(D) if bias is None else bias)
    y0 = hat if norm == "none" else hat * w + b
    # what a norm's subtraction of the mean adds: the mean is off by D roundings of the elements' size
    size = np.abs(y0) + (0.0 if norm == "none" else (np.abs(x).mean(-1, keepdims=True) + np.abs(x)) / dev * np.abs(w) + np.abs(b))
    y = turned(y0, angle, neighbours)
    out = {"y": (y, u * np.abs(y) * (1 + u) + EPS * (D + 32) * spread(size, rotated, neighbours) + TINY[dtype])}
    if d is None:
        return out
    back = turned(d, -angle, neighbours)
    eback = EPS * 16 * spread(d, rotated, neighbours)
    if norm == "none":
        return dict(out, dx=(back, u * np.abs(back) * (1 + u) + eback + TINY[dtype]))
    e = back * w
    along, mean = (e * hat).mean(-1, keepdims=True), (e.mean(-1, keepdims=True) if norm == "layer" else 0.0)
    dx = (e - hat * along - mean) / dev
    # magnitudes: of the gradient, of hat with what the mean's subtraction leaves in it, and of the means of their products
    fat = spread(d, rotated, neighbours) * np.abs(w) * 2
    hat_size = (np.abs(x).mean(-1, keepdims=True) + np.abs(x)) / dev
    much = (fat + hat_size * (fat * hat_size).mean(-1, keepdims=True) + fat.mean(-1, keepdims=True)) / dev
    out["dx"] = (dx, u * np.abs(dx) * (1 + u) + EPS * (2 * D + 64) * much + TINY[dtype])
    t = there[..., None, None]
    n = there.sum() * x.shape[2]
    out["weight"] = ((back * hat * t).sum((0, 1, 2)), EPS * (n + D + 64) * (2 * spread(d, rotated, neighbours) * hat_size * t).sum((0, 1, 2)) + 1e-30)
    out["bias"] = ((back * t).sum((0, 1, 2)), EPS * (n + 64) * (spread(d, rotated, neighbours) * t).sum((0, 1, 2)) + 1e-30)
    return out


# ------------------------------------------------------------------ cross entropy
def cross_entropy(H, W, targets, *, smoothing=0.0, z_loss=0.0, weights=None, scale=1.0, dtype="f32"):
    """{name: (values, bounds)} of losses, logs, dH and dW.  Arrays in float64."""
    n, V, D = len(H), len(W), H.shape[1]
    u = U[dtype]
    counts = (targets >= 0) & (targets < V)
    rows = np.nonzero(counts)[0]
    z = {k: np.zeros(s) for k, s in (("losses", n), ("logs", n), ("dH", H.shape), ("dW", W.shape))}
    e = {k: np.zeros_like(a) for k, a in z.items()}
    g = scale * (np.ones(n) if weights is None else weights)
    if len(rows):
        h, t, g = H[rows], targets[rows], g[rows, None]
        at = np.arange(len(rows))
        s = h @ W.T
        es = EPS * (D + 4) * (np.abs(h) @ np.abs(W).T)
        es_row = es.max(1, keepdims=True)
        top = s.max(1, keepdims=True)
        L = top + np.log(np.exp(s - top).sum(1, keepdims=True))
        eL = es_row + EPS * (V / 16 + 64 + 2 * np.abs(L) + 2 * np.abs(top))
        mean = s.mean(1, keepdims=True)
        z["logs"][rows], e["logs"][rows] = L[:, 0], eL[:, 0]
        hit = s[at, t][:, None]
        z["losses"][rows] = (L - (1 - smoothing) * hit - smoothing * mean + z_loss * L * L)[:, 0]
        e["losses"][rows] = (eL * (1 + 2 * z_loss * np.abs(L)) + es[at, t][:, None] + smoothing * (es_row + EPS * (V / 16 + 64) * np.abs(s).mean(1, keepdims=True))
                             + 4 * EPS * (np.abs(L) + np.abs(hit) + np.abs(mean) + z_loss * L * L))[:, 0]
        p = np.exp(s - L)
        rise = 1 + 2 * z_loss * L
        one = np.zeros_like(s)
        one[at, t] = 1.0
        dz = (p * rise - (1 - smoothing) * one - smoothing / V) * g
        ep = p * (es + eL + EPS * 32)                                        # of p in fp32
        edz = ((ep + u * p * (1 - one)) * np.abs(rise) + p * 2 * z_loss * eL + 4 * EPS * (p * np.abs(rise) + one + smoothing / V)) * np.abs(g) + u * np.abs(dz)
        # What lies below the smallest numbers.  Exponentials of both 16-bit types are fp16 numbers, whose steps are no smaller than 2^-24, in units of 2^-15 of the largest of their piece: off by
        # 2^-25 2^-15 of a probability of at most 1, and as much again for its factors' roundings.
        if dtype != "f32":
            edz += 2.0 ** -39 * np.abs(rise * g)
        if dtype == "f16":                                                   # dz: 2^-25 in units of 2^-13 of the largest, and the factors' roundings
            edz += 2.0 ** -37 * (np.abs(g) * (2 + 2 * z_loss * np.abs(L))).max()
        z["dH"][rows], z["dW"] = dz @ W, dz.T @ h
        e["dH"][rows] = edz @ np.abs(W) + EPS * (V + 4) * (np.abs(dz) @ np.abs(W))
        e["dW"] = edz.T @ np.abs(h) + EPS * (len(rows) + 4) * (np.abs(dz).T @ np.abs(h))
        for k in ("dH", "dW"):
            e[k] = e[k] * (1 + u) + u * np.abs(z[k]) + TINY[dtype]
    return {k: (z[k], e[k]) for k in z}


# ------------------------------------------------------------------ AdamW
def m_values(codes):
    """e4m3: sign, 4 bits of exponent from 2^-6 on (0: multiples of 2^-9), 3 of mantissa."""
    c = np.asarray(codes, np.int64)
    e, f = (c >> 3) & 15, (c & 7).astype(float)
    return np.where(e > 0, np.ldexp(1 + f / 8, e - 7), f / 512) * np.where(c > 127, -1.0, 1.0)


def v_values(codes):
    c = np.asarray(codes, np.int64)
    return np.where(c > 0, np.ldexp(1 + (c & 7) / 8.0, (c >> 3) - 31), 0.0)


def of_blocks(scale, n):
    return np.repeat(np.asarray(scale, float), 256)[:n]


def adamw(p, g, m, v, *, rate, decay, beta1, beta2, eps, step, grad_scale=1.0):
    """float64: (p, m, v) after a step, and the update's magnitude: of m that of its two terms, which are rounded before they cancel."""
    g = g * grad_scale
    size = beta1 * np.abs(m) + (1 - beta1) * np.abs(g)
    m, v = beta1 * m + (1 - beta1) * g, beta2 * v + (1 - beta2) * g * g
    to = rate / (1 - beta1 ** step) / (np.sqrt(v / (1 - beta2 ** step)) + eps)
    return p - rate * decay * p - to * m, m, v, to * size + rate * decay * np.abs(p)
