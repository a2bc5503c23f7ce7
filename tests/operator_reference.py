"""The operators of a training step in 64 bits on the CPU, from their definitions, with bounds of what the kernels may be off.

The bounds follow the roundings that the kernels make: operands of the second products (probabilities, gradients of scores) and results are
rounded to the storage type once each, everything else is fp32.  `u` is half a unit in the last place of the storage type, relative; EPS that of
fp32 (2^-24)."""
from __future__ import annotations

import math

import numpy as np

EPS = 2.0 ** -24
U = {"f32": EPS, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}       # relative, of the nearest value (bounds; most are half of it)
LEAST = 2.0 ** -126                                          # of fp32's normal numbers: a probability below it is zero
TINY = {"f32": 1e-37, "f16": 2.0 ** -24, "bf16": 1e-37}      # spacing below the normal numbers


def philox(counter, key, rounds=7):
    """Philox4x32 of four Python or numpy integers below 2^32 (broadcast): four words."""
    c = [np.asarray(x, dtype=np.uint64) for x in counter]
    k = [int(x) for x in key]
    low, half = np.uint64(0xFFFFFFFF), np.uint64(32)
    for _ in range(rounds):
        p, q = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(q >> half) ^ c[1] ^ np.uint64(k[0]), q & low, (p >> half) ^ c[3] ^ np.uint64(k[1]), p & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def limit_of(p):
    return min(int(math.floor(float(np.float32(p)) * 65536.0 + 0.5)), 65535)


def keep_factors(counter, seed, p):
    """Factors of eight elements for each counter, in a new last axis."""
    c = philox(counter, (seed & 0xFFFFFFFF, seed >> 32 & 0xFFFFFFFF))
    w = np.stack(np.broadcast_arrays(*c), axis=-1)
    words = np.stack([w & np.uint64(0xFFFF), w >> np.uint64(16)], axis=-1).reshape(w.shape[:-1] + (8,))
    t = limit_of(p)
    return np.where(words >= t, 65536.0 / (65536 - t), 0.0)


def keep_matrix(rows, width, seed, offset, p):
    blocks = (width + 7) // 8
    n = np.arange(rows * blocks, dtype=np.uint64)
    f = keep_factors((n & np.uint64(0xFFFFFFFF), n >> np.uint64(32), 0, offset), seed, p)
    return f.reshape(rows, blocks * 8)[:, :width]


def keep_probabilities(batch_head, q_len, k_len, seed, offset, p):
    block, row = np.arange((k_len + 7) // 8, dtype=np.uint64)[None, :], np.arange(q_len, dtype=np.uint64)[:, None]
    return keep_factors((block, row, batch_head, offset), seed, p).reshape(q_len, -1)[:, :k_len]


def attention(Q, K, V, *, scale, causal, q_lens=None, k_lens=None, dropout=0.0, seed=0, offset=0, dO=None, dtype="f32"):
    """Arrays [batch][position][head][dim] in float64.  Returns {name: (values, bounds)} of O and L and, with dO, of dQ, dK and dV."""
    B, Sq, H, D = Q.shape
    Sk, Hk = K.shape[1], K.shape[2]
    u = U[dtype]
    z = {n: np.zeros(s) for n, s in (("O", Q.shape), ("dQ", Q.shape), ("dK", K.shape), ("dV", V.shape))}
    e = {n: np.zeros_like(a) for n, a in z.items()}
    L, eL = np.full((B, H, Sq), -np.inf), np.zeros((B, H, Sq))
    add = {n: np.zeros_like(a) for n, a in z.items()}           # bounds before the last rounding
    floor = 0.0
    if dO is not None and dtype == "f16":                       # what the operands' scaling leaves below the smallest fp16 number
        floor = 2.0 ** -36 * np.sqrt((dO ** 2).sum(-1).max() * (V ** 2).sum(-1).max()) / max(1e-9, 1.0 - dropout)
    for b in range(B):
        nq = Sq if q_lens is None else min(max(int(q_lens[b]), 0), Sq)
        nk = Sk if k_lens is None else min(max(int(k_lens[b]), 0), Sk)
        if nq == 0 or nk == 0:
            continue
        seen = np.ones((nq, nk), bool) if not causal else (np.arange(nk)[None, :] - nk <= np.arange(nq)[:, None] - nq)
        for h in range(H):
            g = h // (H // Hk)
            q, k, v = Q[b, :nq, h], K[b, :nk, g], V[b, :nk, g]
            s = np.where(seen, scale * (q @ k.T), -np.inf)
            rows = seen.any(1)
            top = np.where(rows, s.max(1, initial=-np.inf), 0.0)
            p = np.where(seen, np.exp(s - top[:, None]), 0.0)
            total = p.sum(1)
            p = p / np.where(rows, total, 1.0)[:, None]
            L[b, h, :nq] = np.where(rows, top + np.log(np.where(rows, total, 1.0)), -np.inf)
            # a score's error: D products summed in fp32, then the scale and the shift by a maximum, each a rounding of numbers of this size
            es = EPS * ((D + 4) * scale * (np.abs(q) @ np.abs(k).T) + 4 * np.abs(top)[:, None] + 16)
            es_row = np.where(seen, es, 0.0).max(1)
            eL[b, h, :nq] = es_row + EPS * (nk + 8 + 2 * np.abs(np.where(rows, L[b, h, :nq], 0.0)))
            ep = 2 * (es + es_row[:, None]) + EPS * (nk + 8)     # relative, of a probability
            keep = keep_probabilities(b * H + h, nq, nk, seed, offset, dropout) if dropout > 0 else 1.0
            pd = p * keep
            z["O"][b, :nq, h] = pd @ v
            add["O"][b, :nq, h] = (pd * (u + ep + EPS * (nk + 4)) + LEAST * seen) @ np.abs(v)
            if dO is None:
                continue
            d = dO[b, :nq, h]
            z["dV"][b, :nk, g] += pd.T @ d
            add["dV"][b, :nk, g] += (pd * (u + ep + EPS * (nq + 4)) + LEAST * seen).T @ np.abs(d)
            dp = (d @ v.T) * keep
            edp = EPS * (D + 4) * (np.abs(d) @ np.abs(v).T) * keep
            delta = (p * dp).sum(1)
            eO = add["O"][b, :nq, h] + u * np.abs(z["O"][b, :nq, h]) + TINY[dtype]
            edelta = (np.abs(d) * eO).sum(1) + EPS * (D + 4) * (np.abs(d) * np.abs(z["O"][b, :nq, h])).sum(1)
            ds = p * (dp - delta[:, None])
            eds = p * (ep * np.abs(dp - delta[:, None]) + edp + edelta[:, None] + 4 * EPS * (np.abs(dp) + np.abs(delta)[:, None])) + u * np.abs(ds)
            eds += LEAST * (np.abs(dp) + np.abs(delta)[:, None])
            eds = np.where(seen, eds * (1 + u) + floor, 0.0)
            z["dQ"][b, :nq, h] = scale * (ds @ k)
            add["dQ"][b, :nq, h] = scale * ((eds + EPS * (nk + 4) * np.abs(ds)) @ np.abs(k))
            z["dK"][b, :nk, g] += scale * (ds.T @ q)
            add["dK"][b, :nk, g] += scale * ((eds + EPS * (nq + 4) * np.abs(ds)).T @ np.abs(q))
    out = {n: (z[n], add[n] * (1 + u) + u * np.abs(z[n]) + TINY[dtype]) for n in (("O",) if dO is None else ("O", "dQ", "dK", "dV"))}
    out["L"] = (L, eL)
    return out


def residual_norm(x, f, *, post, pre, eps, a, b, w_post=None, b_post=None, gate=None, w_pre=None, b_pre=None, keep=1.0, dy=None, dh=None):
    """Arrays in float64, [rows][width]; `keep`: dropout's factors.  Returns values by name."""
    one, zero = np.ones(x.shape[1]), np.zeros(x.shape[1])
    w_post, w_pre, gate = (one if v is None else v for v in (w_post, w_pre, gate))
    b_post, b_pre = (zero if v is None else v for v in (b_post, b_pre))

    def norm(v, kind):
        if kind == "none":
            return v, np.ones((len(v), 1))
        v = v - v.mean(1, keepdims=True) if kind == "layer" else v
        dev = np.sqrt((v * v).mean(1, keepdims=True) + eps)
        return v / dev, dev

    def back(d, hat, dev, kind):
        if kind == "none":
            return d
        inner = d - hat * (d * hat).mean(1, keepdims=True)
        return (inner - (d.mean(1, keepdims=True) if kind == "layer" else 0.0)) / dev

    f_hat, f_dev = norm(f, post)
    u = keep * (f_hat * w_post + b_post if post != "none" else f_hat)
    y = a * x + b * gate * u
    y_hat, y_dev = norm(y, pre)
    out = {"y": y, "h": y_hat * w_pre + b_pre if pre != "none" else y_hat, "f_dev": f_dev, "y_dev": y_dev}
    if dy is not None:
        e = dh if pre == "none" else dh * w_pre
        total = dy + back(e, y_hat, y_dev, pre)
        du = b * total * gate * keep
        out.update(dx=a * total, df=back(du * w_post if post != "none" else du, f_hat, f_dev, post), total=total, du=du,
                   pre_weight=(dh * y_hat).sum(0), pre_bias=dh.sum(0), gate=(b * total * u).sum(0), post_weight=(du * f_hat).sum(0), post_bias=du.sum(0))
    return out
