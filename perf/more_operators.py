"""What a training step needs around attention, norms and the compressed update, as cases that can be timed.

Between the joint projection of queries, keys and values and attention stand the norms of each head and the rotation by position;
behind the last norm stands the loss over the vocabulary, with whose gradient the backward pass begins; and the parameters that
have no projector (embeddings, norms, biases) take an ordinary optimizer step.  Every case is one pass of one operator:

  rotary         Qr = rotate(norm(Q)), Kr = rotate(norm(K)), head by head.  Pair j of a head, elements (j, rotated / 2 + j) or, with
                 "neighbours", (2 j, 2 j + 1), turns by position * frequency[j]; elements from `rotated` on stay.  Token i of text b has
                 position start[b] + i or the one given, counts when i < lens[b], and with "cache" its key and value go to place start[b] + i
                 of the text's cache.  With "train" also the gradients of Q, K and of the norms' weights from those of Qr and Kr.
  cross_entropy  z = H W^T, loss = log(sum exp z) - (1 - smoothing) z_target - smoothing mean(z) + z_loss log(sum exp z)^2, row by row; a row
                 whose target is outside the vocabulary does not count: loss 0, no gradient.  With "train" also the gradients of H and W of
                 the sum of weight * loss.
  adamw          m = beta1 m + (1 - beta1) g, v = beta2 v + (1 - beta2) g^2, p -= rate (decay p + (m / c1) / (sqrt(v / c2) + eps)) with
                 c = 1 - beta^step (Loshchilov and Hutter, "Decoupled weight decay regularization", ICLR 2019), over many tensors, with
                 states in fp32 or in 8 bits: blocks of 256 elements that share an fp32 scale, m as e4m3 (largest 448), v without sign as 5
                 bits of exponent and 3 of mantissa (code 0 is 0, others 2^(code / 8 - 31) (1 + code % 8 / 8), largest 1.875, and what is not
                 0 is at least the smallest).  Both are rounded to nearest, ties to even; the update takes m and v before that rounding.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

_TORCH = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_SIZE = {"f32": 4, "f16": 2, "bf16": 2}
_CODE = {"f32": 0, "f16": 1, "bf16": 2}
_EPS = 1e-5
_BLOCK = 256                    # elements that share a scale
_BETA1, _BETA2, _ADAM_EPS, _STEP, _RATE = 0.9, 0.95, 1e-8, 100, 5e-5


def _rotary(name, train, dtype, batch, length, heads, kv_heads, head_dim, rotated, norm="none", bias=False, neighbours=False, ragged=False, cache=0, far=0):
    c = {"op": "rotary", "train": train, "dtype": dtype, "batch": batch, "length": length, "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim,
         "rotated": rotated, "norm": norm, "bias": bias, "neighbours": neighbours, "ragged": ragged, "cache": cache, "far": far}
    return dict(c, name=name) if name else c


def _loss(name, train, dtype, rows, width, vocab, smoothing=0.0, z_loss=0.0, left_out=0.0):
    c = {"op": "cross_entropy", "train": train, "dtype": dtype, "rows": rows, "width": width, "vocab": vocab, "smoothing": smoothing, "z_loss": z_loss,
         "left_out": left_out}
    return dict(c, name=name) if name else c


def _adamw(name, dtype, grad, states, tensors, elements, master=False, odd=False):
    c = {"op": "adamw", "dtype": dtype, "grad": grad, "states": states, "tensors": tensors, "elements": elements, "master": master, "odd": odd}
    return dict(c, name=name) if name else c


def listed():
    return [
        # a 6.7B-style layer (32 heads of 128) on a batch of texts of 1024 tokens: norms of queries and keys, rotation, and back
        _rotary("rotary_layer_bf16", True, "bf16", 4, 1024, 32, 32, 128, 128, norm="rms"),
        # generating: single tokens, keys and values straight into caches of 4096 positions
        _rotary("rotary_token_bf16", False, "bf16", 8, 1, 32, 8, 128, 128, norm="rms", ragged=True, cache=4096),
        # a padded batch with shared key heads; a part of each head turns, neighbours together; norms with means, weights and biases
        _rotary("rotary_ragged_f16", True, "f16", 3, 777, 16, 4, 80, 32, norm="layer", bias=True, neighbours=True, ragged=True),
        # documents packed one behind the other, with positions of their own, far from the beginning
        _rotary("rotary_far_f32", False, "f32", 1, 16384, 16, 16, 64, 64, far=1000000),
        # the smallest layer of the configurations (256 wide) under a small vocabulary, in fp32: launches and latency
        _loss("loss_small_f32", True, "f32", 64, 256, 1000),
        # a 6.7B-style model's last layer: 4 x 1024 tokens, 4096 wide
        _loss("loss_layer_bf16", True, "bf16", 4096, 4096, 32000),
        # fine-tuning on answers: two rows of five are prompt or padding and do not count; nothing divides a tile
        _loss("loss_ragged_f16", True, "f16", 3001, 1000, 50021, smoothing=0.1, left_out=0.4),
        # evaluation over a large vocabulary
        _loss("loss_eval_bf16", False, "bf16", 8192, 2048, 128000, z_loss=1e-4),
        # the norms of a model's layers: 64 short tensors whose gradients are fp32
        _adamw("adamw_norms_bf16", "bf16", "f32", "f32", 64, 4096),
        # an embedding of 32000 x 4096 with an fp32 copy, states in fp32
        _adamw("adamw_embedding_bf16", "bf16", "bf16", "f32", 1, 131072000, master=True),
        # the same with states in 8 bits
        _adamw("adamw_8bit_bf16", "bf16", "bf16", "8bit", 1, 131072000),
        # tensors of odd sizes, states in 8 bits
        _adamw("adamw_8bit_odd_f32", "f32", "f32", "8bit", 9, 2999999, odd=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rotary", "cross_entropy", "adamw"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if op == "rotary":
        while True:
            kv_heads = rng.choice([1, 2, 4, 8, 16, 32])
            heads, dim = kv_heads * rng.choice([1, 1, 2, 4]), rng.choice([32, 64, 64, 80, 96, 128, 128, 128])
            kind = rng.choice(["train", "train", "forward", "token", "cache"])
            norm = rng.choice(["none", "rms", "rms", "layer"])
            length = rng.randint(1, 4) if kind == "token" else _log_int(rng, 5, 16384)
            cache = length + _log_int(rng, 16, 4096) if kind in ("token", "cache") else 0
            c = _rotary(None, kind == "train", dtype, rng.choice([1, 1, 2, 3, 4, 8]), length, heads, kv_heads, dim, rng.choice([dim, dim, dim // 16 * 8]), norm=norm,
                        bias=norm == "layer" or (norm == "rms" and rng.random() < 0.2), neighbours=rng.random() < 0.4, ragged=cache > 0 or rng.random() < 0.4, cache=cache,
                        far=rng.choice([0, 0, 100000]) if not cache else 0)
            if heads <= 64 and work(c)["bytes"] <= 5e8 and c["batch"] * cache * kv_heads * dim <= 1 << 26:
                return c
    if op == "cross_entropy":
        while True:
            train = rng.random() < 0.7
            c = _loss(None, train, dtype, _log_int(rng, 16, 8192), _log_int(rng, 8, 512) * 8, _log_int(rng, 500, 130000), smoothing=rng.choice([0.0, 0.0, 0.1]),
                      z_loss=rng.choice([0.0, 0.0, 1e-4]), left_out=rng.choice([0.0, 0.0, 0.1, 0.5]))
            if work(c)["flops"] <= (4e11 if dtype == "f32" else 3.2e12):
                return c
    states = rng.choice(["f32", "8bit"])
    tensors = rng.choice([1, 1, 3, 9, 40, 200])
    return _adamw(None, dtype, rng.choice([dtype, dtype, "f32"]), states, tensors, max(1, _log_int(rng, 1000, 100000000) // tensors), master=dtype != "f32" and rng.random() < 0.4,
                  odd=rng.random() < 0.5)


def _sizes(c):
    """Elements of each tensor."""
    return [max(1, c["elements"] // (k + 1) - k) if c["odd"] else c["elements"] for k in range(c["tensors"])]


def _lens(c, seed):
    """(starts, lens), lists, or None each where there are none."""
    if not c["ragged"]:
        return None, None
    g = np.random.default_rng(seed)
    lens = [c["length"]] + [int(x) for x in g.integers(c["length"] // 4 + 1, c["length"] + 1, c["batch"] - 1)]
    starts = [c["cache"] - c["length"]] + [int(x) for x in g.integers(0, c["cache"] - c["length"] + 1, c["batch"] - 1)] if c["cache"] else None
    return starts, lens


def work(c):
    z = _SIZE[c["dtype"]]
    if c["op"] == "rotary":
        # what another seed's lengths would need differs a little; these stand for all
        tokens = sum(_lens(c, 1)[1]) if c["ragged"] else c["batch"] * c["length"]
        one = tokens * (c["heads"] + c["kv_heads"]) * c["head_dim"]
        values = tokens * c["kv_heads"] * c["head_dim"] if c["cache"] else 0
        normed = c["norm"] != "none"
        # forward: read and written; backward: the gradients read and written, and what was normed read again
        return {"bytes": z * ((2 + 2 * c["train"]) * one + 2 * values), "flops": one * ((12 if normed else 6) + c["train"] * (24 if normed else 6))}
    if c["op"] == "cross_entropy":
        n, d, v = round(c["rows"] * (1 - c["left_out"])), c["width"], c["vocab"]
        return {"bytes": (1 + c["train"]) * (n * d + v * d) * z + 4 * n, "flops": 2 * n * d * v * (3 if c["train"] else 1) + 6 * n * v}
    n = sum(_sizes(c))
    state = 2 * (4 if c["states"] == "f32" else 1 + 4 / _BLOCK)
    return {"bytes": n * (2 * z - (z if c["master"] else 0) + _SIZE[c["grad"]] + 2 * state + (8 if c["master"] else 0)), "flops": 16 * n}


# ------------------------------------------------------------------ inputs
def prepare(c, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    t = _TORCH[c["dtype"]]

    def normal(*shape):
        return torch.randn(*shape, device="cuda", generator=gen)

    s = dict(c)
    if c["op"] == "rotary":
        B, n, H, Hk, D = (c[k] for k in ("batch", "length", "heads", "kv_heads", "head_dim"))
        joint = normal(B, n, H + 2 * Hk, D)
        joint[..., : max(1, D // 32)] *= 6.0                     # a few large channels, as projections have them
        s["Q"], s["K"], s["V"] = joint.to(t).split([H, Hk, Hk], dim=2)
        s["Qr"] = torch.zeros(B, n, H, D, device="cuda", dtype=t)
        if c["cache"]:
            s["Kr"], s["Vr"] = (normal(B, c["cache"], Hk, D).to(t) for _ in range(2))
        else:
            s["Kr"], s["Vr"], s["V"] = torch.zeros(B, n, Hk, D, device="cuda", dtype=t), None, None
        s["frequencies"] = (10000.0 ** (-torch.arange(0, c["rotated"], 2, device="cuda", dtype=torch.float64) / c["rotated"])).float()
        starts, lens = _lens(c, seed)
        s["starts"], s["lens"] = (None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda") for x in (starts, lens))
        s["positions"] = None
        if c["far"]:                                             # texts of about 1000 tokens that each begin somewhere
            i = torch.arange(n, device="cuda")
            begin = torch.randint(0, c["far"], (B, n // 1000 + 1), device="cuda", generator=gen)
            s["positions"] = (begin[:, i // 1000] + i % 1000).to(torch.int32)
        for k in ("q", "k"):
            s[k + "_weight"] = None if c["norm"] == "none" else (1.0 + 0.2 * normal(D)).to(t)
            s[k + "_bias"] = (0.1 * normal(D)).to(t) if c["bias"] else None
        if c["train"]:
            s["dQr"], s["dKr"] = normal(B, n, H, D).to(t), normal(B, n, Hk, D).to(t)
            s["dQ"], s["dK"], _ = torch.zeros(B, n, H + 2 * Hk, D, device="cuda", dtype=t).split([H, Hk, Hk], dim=2)
            for k in ("q_weight", "k_weight", "q_bias", "k_bias"):
                s["d" + k] = None if s[k] is None else torch.empty(D, device="cuda")
    elif c["op"] == "cross_entropy":
        n, d, v = c["rows"], c["width"], c["vocab"]
        W = normal(v, d) / math.sqrt(d)
        targets = torch.randint(0, v, (n,), device="cuda", generator=gen)
        known = torch.rand(n, 1, device="cuda", generator=gen) * 8.0      # some targets are likely and some are not
        s["H"], s["W"] = (2.0 * normal(n, d) + known * W[targets]).to(t), W.to(t)
        if c["left_out"]:
            targets[torch.rand(n, device="cuda", generator=gen) < c["left_out"]] = -100
        s["targets"], s["losses"] = targets, torch.empty(n, device="cuda")
        if c["train"]:
            s["weights"] = (0.5 + torch.rand(n, device="cuda", generator=gen)) / n
            s["dH"], s["dW"] = torch.empty_like(s["H"]), torch.empty_like(s["W"])
    else:
        # tensors are pieces of flat buffers, each from a multiple of 256 elements on; what is between them is 0 and stays so
        sizes = _sizes(c)
        s["sizes"], s["firsts"], total = sizes, [], 0
        for n in sizes:
            s["firsts"].append(total)
            total += -(-n // _BLOCK) * _BLOCK
        lengths = [b - a for a, b in zip(s["firsts"], s["firsts"][1:] + [total])]
        s["decays"] = [0.1 if k % 2 == 0 else 0.0 for k in range(len(sizes))]
        inside = torch.ones(total, dtype=torch.bool, device="cuda")
        for n, first, length in zip(sizes, s["firsts"], lengths):
            inside[first + n: first + length] = False
        p = normal(total).mul_(0.02).mul_(inside)
        s["param"] = p.to(t)
        s["master"] = p if c["master"] else None
        spread = torch.exp(1.5 * normal(total // 64 + 1)).repeat_interleave(64)[:total].mul_(inside)    # gradients differ in size from row to row
        s["grad"] = (normal(total).mul_(spread).mul_(1e-3)).to(_TORCH[c["grad"]])
        m, v = normal(total).mul_(spread).mul_(2e-4), (normal(total).square_().add_(0.1)).mul_(spread).mul_(spread).mul_(1e-6)
        if c["states"] == "f32":
            s["m"], s["v"], s["m_scale"], s["v_scale"] = m, v, None, None
        else:
            s["m"], s["m_scale"] = _encode_m(m)
            s["v"], s["v_scale"] = _encode_v(v)
        s["grad_scale"] = torch.full((1,), 0.7, device="cuda")   # of clipping
        s["decay"] = torch.tensor(s["decays"], device="cuda").repeat_interleave(torch.tensor(lengths, device="cuda")) if len(sizes) > 1 else torch.full((1,), s["decays"][0], device="cuda")
    return s


# ------------------------------------------------------------------ 8 bits
def _encode_m(m):
    """(codes as uint8, scales) of e4m3 in blocks."""
    b = m.view(-1, _BLOCK)
    scale = b.abs().amax(dim=1) / 448.0
    y = torch.where(scale[:, None] > 0, b / torch.where(scale > 0, scale, 1.0)[:, None], 0.0)
    return y.float().clamp_(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8).view(-1), scale.float()


def _decode_m(codes, scale, t):
    return (codes.view(torch.float8_e4m3fn).to(t).view(-1, _BLOCK) * scale.to(t)[:, None]).view(-1)


def _encode_v(v):
    b = v.view(-1, _BLOCK)
    scale = b.amax(dim=1) / 1.875
    y = torch.where(scale[:, None] > 0, b / torch.where(scale > 0, scale, 1.0)[:, None], 0.0).float()
    bits = y.view(torch.int32)
    code = ((bits + 0x7FFFF + ((bits >> 20) & 1)) >> 20) - (127 - 31) * 8
    return torch.where(y > 0, code.clamp(1, 255), 0).to(torch.uint8).view(-1), scale.float()


def _code_values(codes, t):
    """The values that codes of v stand for, without their scale."""
    c = codes.to(torch.int32)
    return torch.where(c > 0, ((c + (127 - 31) * 8) << 20).view(torch.float32), 0.0).to(t)


def _decode_v(codes, scale, t):
    return (_code_values(codes, t).view(-1, _BLOCK) * scale.to(t)[:, None]).view(-1)


# ------------------------------------------------------------------ the plain forms
def _counted(s):
    """Which tokens count, and the position of each: [batch][length]."""
    i = torch.arange(s["length"], device="cuda")[None, :]
    counts = (i < s["lens"][:, None]) if s["lens"] is not None else (i < s["length"]).expand(s["batch"], -1)
    at = i + s["starts"][:, None] if s["starts"] is not None else i.expand(s["batch"], -1)
    return counts, at, at if s["positions"] is None else s["positions"]


def _turn(s, x, cos, sin):
    """Pairs of a float32 [batch][length][heads][head_dim], turned."""
    r = s["rotated"]
    if s["neighbours"]:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        turned = torch.stack([a * cos - b * sin, a * sin + b * cos], dim=-1).flatten(-2)
    else:
        a, b = x[..., : r // 2], x[..., r // 2: r]
        turned = torch.cat([a * cos - b * sin, a * sin + b * cos], dim=-1)
    return torch.cat([turned, x[..., r:]], dim=-1)


def _head_norm(x, kind):
    """(normed heads, one over their deviation)"""
    if kind == "none":
        return x, None
    x = x - x.mean(dim=-1, keepdim=True) if kind == "layer" else x
    factor = torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + _EPS)
    return x * factor, factor


def _plain_rotary(s):
    t = s["Q"].dtype
    counts, at, position = _counted(s)
    angle = (position.double()[:, :, None] * s["frequencies"].double())[:, :, None, :]
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    there = counts[:, :, None, None]
    out = {}
    for k in ("q", "k"):
        x = torch.where(there, s[k.upper()].float(), 0.0)
        hat, factor = _head_norm(x, s["norm"])
        w, b = (None if s[k + name] is None else s[k + name].float() for name in ("_weight", "_bias"))
        y = hat if w is None else hat * w
        turned = _turn(s, y if b is None else y + b, cos, sin).to(t)
        into = s[k.upper() + "r"]
        if k == "k" and s["cache"]:
            text, token = counts.nonzero(as_tuple=True)
            place = at[text, token]
            into[text, place] = turned[text, token]
            s["Vr"][text, place] = s["V"][text, token]
            out["Kr"], out["Vr"] = into, s["Vr"]
        else:
            out[k.upper() + "r"] = torch.where(there, turned, into)
        if s["train"]:
            d = _turn(s, torch.where(there, s["d" + k.upper() + "r"].float(), 0.0), cos, -sin)
            dy = d if w is None else d * w
            if s["norm"] != "none":
                if w is not None:
                    out["d" + k + "_weight"] = (d * hat).double().sum(dim=(0, 1, 2)).float()
                if b is not None:
                    out["d" + k + "_bias"] = d.double().sum(dim=(0, 1, 2)).float()
                inner = dy - hat * (dy * hat).mean(dim=-1, keepdim=True)
                dy = factor * (inner - dy.mean(dim=-1, keepdim=True) if s["norm"] == "layer" else inner)
            out["d" + k.upper()] = torch.where(there, dy, 0.0).to(t)
    return out


def _plain_loss(s):
    t, V = s["H"].dtype, s["vocab"]
    counts = (s["targets"] >= 0) & (s["targets"] < V)
    target = torch.where(counts, s["targets"], 0)[:, None]
    h, w = s["H"].float(), s["W"].float()
    z = torch.matmul(h, w.t())
    top = z.amax(dim=1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(dim=1, keepdim=True)
    L = top + torch.log(total)
    losses = L - (1 - s["smoothing"]) * z.gather(1, target)
    if s["smoothing"]:
        losses = losses - s["smoothing"] * z.mean(dim=1, keepdim=True)
    if s["z_loss"]:
        losses = losses + s["z_loss"] * L * L
    out = {"losses": torch.where(counts, losses.squeeze(1), 0.0)}
    if s["train"]:
        dz = e / total
        if s["z_loss"]:
            dz = dz * (1.0 + 2.0 * s["z_loss"] * L)
        if s["smoothing"]:
            dz = dz - s["smoothing"] / V
        dz = dz.scatter_add(1, target, torch.full_like(L, s["smoothing"] - 1.0))
        dz = dz * torch.where(counts, s["weights"], 0.0)[:, None]
        out["dH"], out["dW"] = torch.matmul(dz, w).to(t), torch.matmul(dz.t().contiguous(), h).to(t)
    return out


def _plain_adamw(s):
    # what is rounded to 8 bits is computed in 64: values next to a border
    f = torch.float32 if s["states"] == "f32" else torch.float64
    g = s["grad"].to(f) * s["grad_scale"].to(f)
    m = s["m"] if s["states"] == "f32" else _decode_m(s["m"], s["m_scale"], f)
    v = s["v"] if s["states"] == "f32" else _decode_v(s["v"], s["v_scale"], f)
    m = _BETA1 * m + (1 - _BETA1) * g
    v = _BETA2 * v + (1 - _BETA2) * g * g
    p = (s["master"] if s["master"] is not None else s["param"]).to(f)
    step = (m / (1 - _BETA1 ** _STEP)) / (torch.sqrt(v / (1 - _BETA2 ** _STEP)) + _ADAM_EPS)
    p = p - _RATE * (s["decay"].to(f) * p + step)
    s["param"].copy_(p.float())
    if s["master"] is not None:
        s["master"].copy_(p)
    for k, x, encode in (("m", m, _encode_m), ("v", v, _encode_v)):
        if s["states"] == "f32":
            s[k].copy_(x)
        else:
            codes, scale = encode(x)
            s[k].copy_(codes)
            s[k + "_scale"].copy_(scale)
    return _adamw_state(s)


def _adamw_state(s):
    """What a step leaves; the 8-bit states as the values that their codes stand for, beside the scales."""
    out = {k: s[k] for k in ("param", "master", "m", "v", "m_scale", "v_scale") if s[k] is not None}
    if s["states"] == "8bit":
        out["m"], out["v"] = s["m"].view(torch.float8_e4m3fn), _code_values(s["v"], torch.bfloat16)
    return out


# ------------------------------------------------------------------ the framework's operators
def _scratch(s, key, count):
    """Scratch that a program keeps from pass to pass."""
    if key not in s:
        s[key] = torch.empty(max(int(count), 16), dtype=torch.uint8, device="cuda")
    return s[key]


def _own_rotary(s):
    import paper_2406_10181_amd as lsp
    stream, code = torch.cuda.current_stream(), _CODE[s["dtype"]]
    p = lsp.rotary_problem(s["Q"], s["K"], s["Qr"], s["Kr"], V=s["V"], Vr=s["Vr"], frequencies=s["frequencies"], neighbours=s["neighbours"], positions=s["positions"],
                           starts=s["starts"], lens=s["lens"], norm=s["norm"], q_weight=s["q_weight"], k_weight=s["k_weight"], q_bias=s["q_bias"], k_bias=s["k_bias"], eps=_EPS)
    lsp.lsp_rotary_forward(p, code, stream)
    out = {"Qr": s["Qr"], "Kr": s["Kr"]}
    if s["cache"]:
        out["Vr"] = s["Vr"]
    if s["train"]:
        names = ("q_weight", "k_weight", "q_bias", "k_bias")
        g = lsp.rotary_gradients(s["dQr"], s["dKr"], s["dQ"], s["dK"], **{k: s["d" + k] for k in names})
        nbytes = lsp.lsp_rotary_backward_workspace_bytes(p, code)
        lsp.lsp_rotary_backward(p, g, code, _scratch(s, "ws", nbytes), nbytes, stream)
        out.update({"dQ": s["dQ"], "dK": s["dK"]}, **{"d" + k: s["d" + k] for k in names if s["d" + k] is not None})
    return out


def _own_loss(s):
    import paper_2406_10181_amd as lsp
    stream, code = torch.cuda.current_stream(), _CODE[s["dtype"]]
    p = lsp.cross_entropy_problem(s["H"], s["W"], s["targets"], s["losses"], smoothing=s["smoothing"], z_loss=s["z_loss"])
    if not s["train"]:
        nbytes = lsp.lsp_cross_entropy_forward_workspace_bytes(p, code)
        lsp.lsp_cross_entropy_forward(p, code, _scratch(s, "ws", nbytes), nbytes, stream)
        return {"losses": s["losses"]}
    nbytes = lsp.lsp_cross_entropy_backward_workspace_bytes(p, code)
    lsp.lsp_cross_entropy_backward(p, lsp.cross_entropy_gradients(s["dH"], s["dW"], weights=s["weights"]), code, _scratch(s, "ws", nbytes), nbytes, stream)
    return {"losses": s["losses"], "dH": s["dH"], "dW": s["dW"]}


def _own_adamw(s):
    import paper_2406_10181_amd as lsp
    if "items" not in s:                                         # addresses, which a program keeps as long as its parameters
        def piece(k, first, n, per=1):
            return None if s[k] is None else s[k][first // per: -(-(first + n) // per)]
        s["items"] = lsp.adamw_items([dict(
            param=piece("param", a, n), grad=piece("grad", a, n), m=piece("m", a, n), v=piece("v", a, n), m_scale=piece("m_scale", a, n, _BLOCK),
            v_scale=piece("v_scale", a, n, _BLOCK), master=piece("master", a, n), decay=d) for a, n, d in zip(s["firsts"], s["sizes"], s["decays"])])
    lsp.lsp_adamw(s["items"], rate=_RATE, beta1=_BETA1, beta2=_BETA2, eps=_ADAM_EPS, step=_STEP, grad_scale=s["grad_scale"], stream=torch.cuda.current_stream())
    return _adamw_state(s)


def run(s):
    if own:
        return {"rotary": _own_rotary, "cross_entropy": _own_loss, "adamw": _own_adamw}[s["op"]](s)
    return {"rotary": _plain_rotary, "cross_entropy": _plain_loss, "adamw": _plain_adamw}[s["op"]](s)


# ------------------------------------------------------------------ the same in 64 bits, from the definitions
def exact(c, seed):
    s = prepare(c, seed)
    return {"rotary": _exact_rotary, "cross_entropy": _exact_loss, "adamw": _exact_adamw}[c["op"]](s)


def _exact_rotary(s):
    """Pairs as complex numbers times numbers of length one; the gradients by torch's differentiation of that."""
    f64 = torch.float64
    lens = [s["length"]] * s["batch"] if s["lens"] is None else s["lens"].tolist()
    out = {k: s[k].to(f64).clone() for k in ("Qr", "Kr")}
    if s["cache"]:
        out["Vr"] = s["Vr"].to(f64).clone()
    if s["train"]:
        out["dQ"], out["dK"] = (torch.zeros(s[k].shape, dtype=f64, device="cuda") for k in ("Q", "K"))
    r = s["rotated"]
    vectors = {k: s[k].to(f64).requires_grad_() for k in ("q_weight", "k_weight", "q_bias", "k_bias") if s[k] is not None}

    def head(x, k, turn):
        if s["norm"] != "none":
            x = x - x.mean(-1, keepdim=True) if s["norm"] == "layer" else x
            x = x / (x.pow(2).mean(-1, keepdim=True) + _EPS).sqrt()
            x = x * vectors[k + "_weight"] + vectors.get(k + "_bias", 0.0)
        pairs = x[..., :r].unflatten(-1, (-1, 2) if s["neighbours"] else (2, -1))
        pairs = pairs if s["neighbours"] else pairs.transpose(-1, -2)
        z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
        return torch.cat([(z if s["neighbours"] else z.transpose(-1, -2)).flatten(-2), x[..., r:]], dim=-1)

    total = 0.0
    for b, n in enumerate(lens):
        first = 0 if s["starts"] is None else int(s["starts"][b])
        position = torch.arange(first, first + n, device="cuda") if s["positions"] is None else s["positions"][b, :n]
        angle = torch.outer(position.to(f64), s["frequencies"].to(f64))
        turn = torch.polar(torch.ones_like(angle), angle)[:, None, :]
        at = first if s["cache"] else 0
        for k in ("q", "k"):
            x = s[k.upper()][b, :n].to(f64).requires_grad_()
            y = head(x, k, turn)
            where = slice(0, n) if k == "q" else slice(at, at + n)
            out[k.upper() + "r"][b, where] = y.detach()
            if s["train"]:
                (y * s["d" + k.upper() + "r"][b, :n].to(f64)).sum().backward()
                out["d" + k.upper()][b, :n] = x.grad
        if s["cache"]:
            out["Vr"][b, at: at + n] = s["V"][b, :n].to(f64)
    if s["train"]:
        out.update({"d" + k: x.grad for k, x in vectors.items()})
    return out


def _exact_loss(s):
    f64, V = torch.float64, s["vocab"]
    w = s["W"].to(f64)
    out = {"losses": torch.zeros(s["rows"], dtype=f64, device="cuda")}
    if s["train"]:
        out["dH"], out["dW"] = torch.zeros(s["H"].shape, dtype=f64, device="cuda"), torch.zeros(w.shape, dtype=f64, device="cuda")
    rows = ((s["targets"] >= 0) & (s["targets"] < V)).nonzero().squeeze(1)
    for some in rows.split(1024):
        h, y = s["H"][some].to(f64), s["targets"][some]
        z = h.mm(w.t().contiguous())
        L = torch.logsumexp(z, dim=1)
        want = torch.full_like(z, s["smoothing"] / V)            # the distribution that the loss compares with
        want[torch.arange(len(some), device="cuda"), y] += 1.0 - s["smoothing"]
        out["losses"][some] = L - (want * z).sum(dim=1) + s["z_loss"] * L.square()
        if s["train"]:
            d = (torch.softmax(z, dim=1) * (1.0 + 2.0 * s["z_loss"] * L[:, None]) - want) * s["weights"][some].to(f64)[:, None]
            out["dH"][some] = d.mm(w)
            out["dW"] += d.t().contiguous().mm(h)
    return out


def _exact_adamw(s):
    f64 = torch.float64
    g = s["grad"].to(f64) * float(s["grad_scale"])
    if s["states"] == "f32":
        m, v = s["m"].to(f64), s["v"].to(f64)
    else:
        # codes read bit by bit: sign, 4 bits of exponent from 2^-6 on (0: multiples of 2^-9), 3 of mantissa; and without sign
        code = s["m"].to(torch.int64)
        e, f = (code >> 3) & 15, (code & 7).to(f64)
        m = torch.where(e > 0, torch.ldexp(1.0 + f / 8.0, e - 7), f / 512.0) * torch.where(code > 127, -1.0, 1.0) * s["m_scale"].to(f64).repeat_interleave(_BLOCK)
        code = s["v"].to(torch.int64)
        v = torch.where(code > 0, torch.ldexp(1.0 + (code & 7).to(f64) / 8.0, (code >> 3) - 31), 0.0) * s["v_scale"].to(f64).repeat_interleave(_BLOCK)
    m, v = m + (1 - _BETA1) * (g - m), v + (1 - _BETA2) * (g * g - v)
    p = (s["param"] if s["master"] is None else s["master"]).to(f64)
    p = p * (1.0 - _RATE * s["decay"].to(f64)) - _RATE * m / (1 - _BETA1 ** _STEP) / ((v / (1 - _BETA2 ** _STEP)).sqrt() + _ADAM_EPS)
    out = {"param": p}
    if s["master"] is not None:
        out["master"] = p
    if s["states"] == "f32":
        return dict(out, m=m, v=v)
    for k, x, largest, least in (("m", m, 448.0, -6), ("v", v, 1.875, -31)):
        scale = x.abs().view(-1, _BLOCK).amax(dim=1) / largest
        y = x / torch.where(scale > 0, scale, 1.0).repeat_interleave(_BLOCK)
        e = torch.frexp(y)[1].to(torch.int64) - 1                # y = 1.f 2^e
        step = torch.ldexp(torch.ones_like(y), e.clamp(min=least) - 3)
        y = torch.round(y / step) * step                         # (to even)
        if k == "v":
            y = torch.where(x > 0, y.clamp(min=1.125 * 2.0 ** -31), 0.0)
        out[k], out[k + "_scale"] = y, scale
    return out
