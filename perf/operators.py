"""The operators of a transformer block's training step that stand beside compress and apply, as cases that can be timed.

LSP-Offload's loop (Alg. 1, Alg. 3) takes the weight gradients of a layer as given.  What makes them on the GPU, apart from
plain matrix products, is here: attention and its backward pass, the norms and the gated residual between two blocks, and
dropout.  Every case is one pass of one operator:

  attention   O = softmax(scale Q K^T + mask) V with the logarithm L of the softmax's sums; with "train" also dQ, dK, dV from dO, the
              probabilities computed again.  Key j is visible to query i of batch b when j < k_lens[b], i < q_lens[b] and, if
              causal, j - k_lens[b] <= i - q_lens[b].  A query that sees no key has O = 0, L = -inf and no gradient.  Query head h
              reads key head h / (heads / kv_heads).  Dropout acts on the probabilities.
  norm        u = norm(f) (norm after a block), y = residual_scale x + branch_scale gate * drop(u) (residual), h = norm(y) (norm
              before the next block); with "train" also the gradients of x, f, the weights, biases and the gate from those of y and h.
  dropout     y = drop(x); its backward pass is the same call on the gradient.

Dropout's mask is a function of (seed, offset, place) and is never stored: Philox4x32 with 7 rounds (Salmon, Moraes, Dror and
Shaw, SC 2011) under the key `seed` turns a counter into eight 16-bit words, one for each of eight elements that follow one
another along the last axis; an element is kept, and scaled by 65536 / (65536 - t), when its word is at least
t = round(65536 p).  The counter is (block of eight keys, query, batch * heads + head, offset) in attention, and
(number of the block of eight, 64 bits, 0, offset) elsewhere, each row starting a new block.
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


def _attention(name, train, dtype, batch, heads, kv_heads, q_len, k_len, head_dim, causal=False, ragged=False, dropout=0.0):
    c = {"op": "attention", "train": train, "dtype": dtype, "batch": batch, "heads": heads, "kv_heads": kv_heads, "q_len": q_len,
         "k_len": k_len, "head_dim": head_dim, "causal": causal, "ragged": ragged, "dropout": dropout}
    return dict(c, name=name) if name else c


def _norm(name, train, dtype, rows, width, post, pre, gate=False, dropout=0.0):
    c = {"op": "norm", "train": train, "dtype": dtype, "rows": rows, "width": width, "post": post, "pre": pre, "gate": gate,
         "dropout": dropout}
    return dict(c, name=name) if name else c


def _dropout(name, dtype, rows, width, dropout):
    c = {"op": "dropout", "dtype": dtype, "rows": rows, "width": width, "dropout": dropout}
    return dict(c, name=name) if name else c


def listed():
    return [
        # the smallest layer of the configurations (256 wide) on a short text, in fp32: launches and latency
        _attention("attention_small_f32", True, "f32", 2, 4, 4, 64, 64, 64, causal=True),
        # a 6.7B-style layer (32 heads of 128) on a batch of texts of 1024 tokens, the longest of the paper's fine-tuning
        _attention("attention_layer_bf16", True, "bf16", 4, 32, 32, 1024, 1024, 128, causal=True),
        # one long text, half the heads
        _attention("attention_long_bf16", True, "bf16", 1, 16, 16, 8192, 8192, 128, causal=True),
        # a batch padded to its longest text, with shared key heads and dropout on the probabilities; nothing divides a tile
        _attention("attention_ragged_f16", True, "f16", 4, 16, 4, 777, 777, 80, causal=True, ragged=True, dropout=0.1),
        # evaluation of an encoder: every token sees every other
        _attention("attention_encoder_f16", False, "f16", 8, 16, 16, 2048, 2048, 64),
        # generating for an evaluation: single tokens against caches of different length
        _attention("attention_token_bf16", False, "bf16", 8, 32, 8, 1, 8192, 128, ragged=True),
        # a 256-wide layer's normalised input from residual and block output, with dropout
        _norm("norm_small_f32", True, "f32", 128, 256, "none", "layer", dropout=0.1),
        # a 6.7B-style layer: 4 x 1024 tokens, norms on both sides of the block, gate
        _norm("norm_layer_bf16", True, "bf16", 4096, 4096, "rms", "rms", gate=True),
        # odd rows and columns
        _norm("norm_ragged_f16", True, "f16", 3001, 2999, "layer", "layer", gate=True, dropout=0.1),
        # evaluation over many tokens of a wide model
        _norm("norm_wide_bf16", False, "bf16", 16384, 8192, "rms", "rms"),
        # the hidden layer of a 6.7B-style MLP
        _dropout("dropout_mlp_bf16", "bf16", 4096, 11008, 0.1),
        # rows of odd length
        _dropout("dropout_odd_f32", "f32", 301, 2999, 0.25),
    ]


_MOST_FLOPS = 10e11        # attention: less than attention_long_bf16 takes
_MOST_ELEMENTS = 1 << 26   # norm, dropout
_NOT_DRAWN = 3072          # a size that no configuration here has


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attention"] * 6 + ["norm"] * 4 + ["dropout"] * 2)
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    dropout = rng.choice([0.0, 0.0, 0.1, 0.25])
    if op == "attention":
        while True:
            kind = rng.choice(["train", "train", "train", "forward", "token"])
            k_len = _log_int(rng, 33, 8192)
            q_len = k_len if kind != "token" else rng.randint(1, 4)
            if kind != "token" and rng.random() < 0.2:
                q_len = _log_int(rng, 17, k_len)                # texts that go on from others, or attention from one text to another
            kv_heads = rng.choice([1, 2, 4, 8, 16])
            heads = kv_heads * rng.choice([1, 1, 2, 4])
            c = _attention(None, kind == "train", dtype, rng.choice([1, 1, 2, 3, 4, 8]), heads, kv_heads, q_len, k_len,
                           rng.choice([32, 64, 64, 80, 96, 128, 128, 128]), causal=rng.random() < 0.7, ragged=rng.random() < 0.4,
                           dropout=dropout if kind == "train" else 0.0)
            pairs = c["batch"] * heads * q_len * k_len
            if heads <= 32 and _NOT_DRAWN not in (q_len, k_len) and work(c)["flops"] <= (_MOST_FLOPS / 8 if dtype == "f32" else _MOST_FLOPS) and pairs <= (1 << 27 if c["dropout"] else 1 << 30):
                return c
    while True:
        rows, width = _log_int(rng, 64, 16384), _log_int(rng, 128, 8192 if op == "norm" else 16384)
        if rng.random() < 0.7:
            width = width // 64 * 64
        if rows * width <= _MOST_ELEMENTS and _NOT_DRAWN not in (rows, width):
            break
    if op == "dropout":
        return _dropout(None, dtype, rows, width, dropout or 0.1)
    post, pre = rng.choice([("none", "layer"), ("none", "rms"), ("rms", "rms"), ("layer", "layer")])
    return _norm(None, rng.random() < 0.7, dtype, rows, width, post, pre, gate=rng.random() < 0.5, dropout=dropout)


def _lengths(c, seed):
    """(q_lens, k_lens), lists, or None each where every text has the full length."""
    if not c["ragged"]:
        return None, None
    g = np.random.default_rng(seed)
    k = [c["k_len"]] + [int(x) for x in g.integers(c["k_len"] // 4 + 1, c["k_len"] + 1, c["batch"] - 1)]
    # padded texts: as many queries as keys are left out; where queries go on from a cache, all of them count
    q = [x for x in k] if c["q_len"] == c["k_len"] else [c["q_len"]] * c["batch"]
    return q, k


def _visible(c, lens):
    """Pairs of a query and a key that it sees, over all batches, of one head."""
    total = 0
    for b in range(c["batch"]):
        q = c["q_len"] if lens[0] is None else lens[0][b]
        k = c["k_len"] if lens[1] is None else lens[1][b]
        total += int(np.clip(np.arange(q, dtype=np.int64) + (k - q) + 1, 0, k).sum()) if c["causal"] else q * k
    return total


def work(c):
    z = _SIZE[c["dtype"]]
    if c["op"] == "attention":
        # what another seed's lengths would need differs a little; these stand for all
        pairs = _visible(c, _lengths(c, 1)) * c["heads"]
        q = c["batch"] * c["q_len"] * c["heads"] * c["head_dim"] * z
        kv = 2 * c["batch"] * c["k_len"] * c["kv_heads"] * c["head_dim"] * z
        if c["ragged"] and c["q_len"] != c["k_len"]:
            kv = kv * sum(_lengths(c, 1)[1]) // (c["batch"] * c["k_len"])
        L = 4 * c["batch"] * c["heads"] * c["q_len"]
        both = 2 if c["train"] else 1                            # O, dQ, dK, dV written and Q, K, V, dO read once
        return {"bytes": both * (2 * q + kv) + L, "flops": pairs * c["head_dim"] * (14 if c["train"] else 4)}
    n = c["rows"] * c["width"]
    if c["op"] == "dropout":
        return {"bytes": 2 * n * z, "flops": 2 * n}
    # forward: x, f read, y, h written; backward: the gradients of y and h read, those of x and f written
    return {"bytes": (8 if c["train"] else 4) * n * z, "flops": (40 if c["train"] else 12) * n}


# ------------------------------------------------------------------ inputs
def prepare(c, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    t = _TORCH[c["dtype"]]

    def normal(*shape):
        return torch.randn(*shape, device="cuda", generator=gen)

    s = dict(c, seed=int(seed) * 0x9E3779B1 + 12345, offset=int(seed) % 1000)
    if c["op"] == "attention":
        B, H, Hk, Sq, Sk, D = (c[k] for k in ("batch", "heads", "kv_heads", "q_len", "k_len", "head_dim"))
        if Sq == Sk:                                             # one projection made all three: views into its output
            qkv = normal(B, Sq, H + 2 * Hk, D)
            qkv[:, :, :H] *= 1.5                                 # scores wide enough for probabilities that differ
            qkv = qkv.to(t)
            s["Q"], s["K"], s["V"] = qkv.split([H, Hk, Hk], dim=2)
            grads = torch.empty_like(qkv).split([H, Hk, Hk], dim=2)
        else:
            s["Q"], s["K"], s["V"] = (normal(B, Sq, H, D) * 1.5).to(t), normal(B, Sk, Hk, D).to(t), normal(B, Sk, Hk, D).to(t)
            grads = [torch.empty_like(s[k]) for k in "QKV"]
        s["O"], s["L"] = torch.empty(B, Sq, H, D, device="cuda", dtype=t), torch.empty(B, H, Sq, device="cuda")
        lens = _lengths(c, seed)
        s["q_lens"], s["k_lens"] = (None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda") for x in lens)
        if c["train"]:
            s["dO"] = normal(B, Sq, H, D).to(t)
            s["dQ"], s["dK"], s["dV"] = grads
    elif c["op"] == "norm":
        n, w = c["rows"], c["width"]
        x = normal(n, w)
        x[:, torch.randperm(w, device="cuda", generator=gen)[: max(1, w // 200)]] *= 20.0   # a residual stream's few large channels
        s["x"], s["f"] = x.to(t), (normal(n, w) * 0.7 + 0.1).to(t)
        s["y"], s["h"], s["stats"] = torch.empty_like(s["x"]), torch.empty_like(s["x"]), torch.empty(4, n, device="cuda")
        for side in ("post", "pre"):
            s[side + "_w"] = None if c[side] == "none" else (1.0 + 0.1 * normal(w)).to(t)
            s[side + "_b"] = (0.1 * normal(w)).to(t) if c[side] == "layer" else None
        s["g"] = (0.5 + 0.1 * normal(w)).to(t) if c["gate"] else None
        s["residual_scale"], s["branch_scale"] = 1.0, 0.7
        if c["train"]:
            s["dy"], s["dh"] = normal(n, w).to(t), normal(n, w).to(t)
            s["dx"], s["df"] = torch.empty_like(s["x"]), torch.empty_like(s["x"])
            for k in ("post_w", "post_b", "pre_w", "pre_b", "g"):
                s["d" + k] = None if s[k] is None else torch.empty(w, device="cuda")
    else:
        s["x"] = normal(c["rows"], c["width"]).to(t)
        s["y"] = torch.empty_like(s["x"])
    return s


# ------------------------------------------------------------------ the plain forms
def _words(c0, c1, c2, c3, seed):
    """Philox4x32-7 of counters given as int64 tensors (broadcast against one another): eight 16-bit words in a new last axis.
    The product of two 32-bit numbers is right modulo 2^64 in int64, whose upper half the mask makes unsigned again."""
    low = 0xFFFFFFFF
    k0, k1 = seed & low, (seed >> 32) & low
    for _ in range(7):                                           # the generator's rounds
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((b >> 32) & low) ^ c1 ^ k0, b & low, ((a >> 32) & low) ^ c3 ^ k1, a & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    w = torch.stack(torch.broadcast_tensors(c0, c1, c2, c3), dim=-1)
    return torch.stack([w & 0xFFFF, w >> 16], dim=-1).flatten(-2)


def _threshold(p):
    return int(math.floor(65536.0 * p + 0.5))


def _drop(x, s):
    """drop() of a float32 matrix."""
    if s["dropout"] == 0.0:
        return x
    rows, width = x.shape
    blocks = (width + 7) // 8
    number = torch.arange(rows * blocks, device=x.device)
    zero = torch.zeros((), dtype=torch.int64, device=x.device)
    words = _words(number & 0xFFFFFFFF, number >> 32, zero, zero + s["offset"], s["seed"]).view(rows, blocks * 8)[:, :width]
    t = _threshold(s["dropout"])
    return torch.where(words >= t, x * (65536.0 / (65536 - t)), 0.0)


def _plain_attention(s):
    t, H, Sq, Sk = s["Q"].dtype, s["heads"], s["q_len"], s["k_len"]
    group = H // s["kv_heads"]
    scale = 1.0 / math.sqrt(s["head_dim"])
    q = s["Q"].float().transpose(1, 2)
    k = s["K"].float().transpose(1, 2).repeat_interleave(group, dim=1)
    v = s["V"].float().transpose(1, 2).repeat_interleave(group, dim=1)
    B = q.shape[0]
    i, j = torch.arange(Sq, device=q.device).view(1, Sq, 1), torch.arange(Sk, device=q.device).view(1, 1, Sk)
    nq = Sq if s["q_lens"] is None else s["q_lens"].view(B, 1, 1)
    nk = Sk if s["k_lens"] is None else s["k_lens"].view(B, 1, 1)
    hidden = (i >= nq) | (j >= nk)
    if s["causal"]:
        hidden = hidden | (j - nk > i - nq)
    hidden = hidden.unsqueeze(1)
    scores = (torch.matmul(q, k.transpose(2, 3)) * scale).masked_fill(hidden, -math.inf)
    top = scores.amax(dim=-1, keepdim=True)
    e = torch.exp(scores - torch.where(top == -math.inf, 0.0, top))
    total = e.sum(dim=-1, keepdim=True)
    L = (top + torch.log(total)).squeeze(-1)
    p = e / torch.where(total == 0.0, 1.0, total)
    keep = None
    if s["dropout"] > 0.0:
        c0 = torch.arange((Sk + 7) // 8, device=q.device)
        c2 = torch.arange(B * H, device=q.device).view(B, H, 1, 1)
        words = _words(c0, i.view(1, 1, Sq, 1), c2, torch.full_like(c2, s["offset"]), s["seed"]).flatten(-2)[..., :Sk]
        limit = _threshold(s["dropout"])
        keep = torch.where(words >= limit, 65536.0 / (65536 - limit), 0.0).float()
    pd = p if keep is None else p * keep
    O = torch.matmul(pd, v)
    out = {"O": O.transpose(1, 2).to(t), "L": L}
    if s["train"]:
        dO = torch.where((i >= nq).unsqueeze(1), 0.0, s["dO"].float().transpose(1, 2))
        dV = torch.matmul(pd.transpose(2, 3), dO)
        dP = torch.matmul(dO, v.transpose(2, 3))
        if keep is not None:
            dP = dP * keep
        dS = p * (dP - (dO * O).sum(dim=-1, keepdim=True)) * scale
        dK = torch.matmul(dS.transpose(2, 3), q)
        shared = (B, s["kv_heads"], group, Sk, s["head_dim"])
        out["dQ"] = torch.matmul(dS, k).transpose(1, 2).to(t)
        out["dK"] = dK.view(shared).sum(dim=2).transpose(1, 2).to(t)
        out["dV"] = dV.view(shared).sum(dim=2).transpose(1, 2).to(t)
    return out


def _normed(x, kind):
    """(normalised rows, their mean, one over their deviation) of a float32 matrix; mean and factor are None where a kind has none."""
    if kind == "none":
        return x, None, None
    mean = x.mean(dim=1, keepdim=True) if kind == "layer" else None
    x = x - mean if kind == "layer" else x
    factor = torch.rsqrt((x * x).mean(dim=1, keepdim=True) + _EPS)
    return x * factor, mean, factor


def _affine(x, w, b):
    x = x if w is None else x * w
    return x if b is None else x + b


def _norm_back(d, hat, factor, kind):
    """The gradient of the rows that _normed was given, from that of its result."""
    if kind == "none":
        return d
    inner = d - hat * (d * hat).mean(dim=1, keepdim=True)
    return factor * (inner - d.mean(dim=1, keepdim=True) if kind == "layer" else inner)


def _plain_norm(s):
    t = s["x"].dtype
    w = {k: None if s[k] is None else s[k].float() for k in ("post_w", "post_b", "pre_w", "pre_b", "g")}
    x, f = s["x"].float(), s["f"].float()
    f_hat, _, f_factor = _normed(f, s["post"])
    u = _drop(_affine(f_hat, w["post_w"], w["post_b"]), s)
    y = s["residual_scale"] * x + s["branch_scale"] * (u if w["g"] is None else u * w["g"])
    y_hat, _, y_factor = _normed(y, s["pre"])
    out = {"y": y.to(t), "h": _affine(y_hat, w["pre_w"], w["pre_b"]).to(t)}
    if s["train"]:
        dy, dh = s["dy"].float(), s["dh"].float()
        total = dy + _norm_back(dh if w["pre_w"] is None else dh * w["pre_w"], y_hat, y_factor, s["pre"])
        branch = s["branch_scale"] * total
        du = _drop(branch if w["g"] is None else branch * w["g"], s)
        out["dx"] = (s["residual_scale"] * total).to(t)
        out["df"] = _norm_back(du if w["post_w"] is None else du * w["post_w"], f_hat, f_factor, s["post"]).to(t)
        out["dpre_w"] = None if w["pre_w"] is None else (dh * y_hat).sum(dim=0)
        out["dpre_b"] = None if w["pre_b"] is None else dh.sum(dim=0)
        out["dg"] = None if w["g"] is None else (branch * u).sum(dim=0)
        out["dpost_w"] = None if w["post_w"] is None else (du * f_hat).sum(dim=0)
        out["dpost_b"] = None if w["post_b"] is None else du.sum(dim=0)
    return {k: v for k, v in out.items() if v is not None}


# ------------------------------------------------------------------ the framework's operators
def _scratch(s, key, count):
    """Scratch that a program keeps from pass to pass."""
    if key not in s:
        s[key] = torch.empty(max(int(count), 16), dtype=torch.uint8, device="cuda")
    return s[key]


def _own_attention(s):
    import paper_2406_10181_amd as lsp
    stream, code = torch.cuda.current_stream(), _CODE[s["dtype"]]
    p = lsp.attention_problem(s["Q"], s["K"], s["V"], s["O"], s["L"], q_lens=s["q_lens"], k_lens=s["k_lens"],
                              scale=1.0 / math.sqrt(s["head_dim"]), causal=s["causal"], dropout=s["dropout"], seed=s["seed"], offset=s["offset"])
    nbytes = lsp.lsp_attention_forward_workspace_bytes(p, code)
    lsp.lsp_attention_forward(p, code, _scratch(s, "forward_ws", nbytes), nbytes, stream)
    if not s["train"]:
        return {"O": s["O"], "L": s["L"]}
    nbytes = lsp.lsp_attention_backward_workspace_bytes(p, code)
    lsp.lsp_attention_backward(p, lsp.attention_gradients(s["dO"], s["dQ"], s["dK"], s["dV"]), code,
                               _scratch(s, "backward_ws", nbytes), nbytes, stream)
    return {k: s[k] for k in ("O", "L", "dQ", "dK", "dV")}


def _own_norm(s):
    import paper_2406_10181_amd as lsp
    stream, code = torch.cuda.current_stream(), _CODE[s["dtype"]]
    p = lsp.residual_norm_problem(s["x"], s["f"], s["y"], s["h"], s["stats"], post=s["post"], post_weight=s["post_w"], post_bias=s["post_b"],
                                  gate=s["g"], pre=s["pre"], pre_weight=s["pre_w"], pre_bias=s["pre_b"], eps=_EPS,
                                  residual_scale=s["residual_scale"], branch_scale=s["branch_scale"],
                                  dropout=s["dropout"], seed=s["seed"], offset=s["offset"])
    lsp.lsp_residual_norm_forward(p, code, stream)
    if not s["train"]:
        return {"y": s["y"], "h": s["h"]}
    g = lsp.residual_norm_gradients(s["dy"], s["dh"], s["dx"], s["df"], post_weight=s["dpost_w"], post_bias=s["dpost_b"], gate=s["dg"],
                                    pre_weight=s["dpre_w"], pre_bias=s["dpre_b"])
    nbytes = lsp.lsp_residual_norm_backward_workspace_bytes(p, code)
    lsp.lsp_residual_norm_backward(p, g, code, _scratch(s, "ws", nbytes), nbytes, stream)
    names = ("y", "h", "dx", "df", "dpre_w", "dpre_b", "dg", "dpost_w", "dpost_b")
    return {k: s[k] for k in names if s[k] is not None}


def _own_dropout(s):
    import paper_2406_10181_amd as lsp
    lsp.lsp_dropout(s["x"], s["y"], s["rows"], s["width"], s["dropout"], s["seed"], s["offset"], _CODE[s["dtype"]], torch.cuda.current_stream())
    return {"y": s["y"]}


def run(s):
    if own:
        return {"attention": _own_attention, "norm": _own_norm, "dropout": _own_dropout}[s["op"]](s)
    if s["op"] == "dropout":
        return {"y": _drop(s["x"].float(), s).to(s["x"].dtype)}
    return _plain_attention(s) if s["op"] == "attention" else _plain_norm(s)


# ------------------------------------------------------------------ the same in 64 bits, from the definitions
def _exact_keep(counter, seed, p):
    """Factors of dropout, on the host: counter is four uint64 arrays that can be broadcast; eight factors in a new last axis."""
    c = [np.asarray(x, np.uint64) for x in counter]
    key = [np.uint64(seed & 0xFFFFFFFF), np.uint64(seed >> 32 & 0xFFFFFFFF)]
    half, low = np.uint64(32), np.uint64(0xFFFFFFFF)
    for r in range(7):
        m0, m1 = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        k0 = np.uint64((int(key[0]) + r * 0x9E3779B9) & 0xFFFFFFFF)
        k1 = np.uint64((int(key[1]) + r * 0xBB67AE85) & 0xFFFFFFFF)
        c = [(m1 >> half) ^ c[1] ^ k0, m1 & low, (m0 >> half) ^ c[3] ^ k1, m0 & low]
    words = np.stack(np.broadcast_arrays(*c), axis=-1).astype(np.uint32)
    words = np.ascontiguousarray(words).view("<u2")
    t = round(p * 65536 - 1e-9)
    return np.where(words >= t, 65536.0 / (65536.0 - t), 0.0)


def _exact_rows_keep(s, rows, width):
    blocks = -(-width // 8)
    n = np.arange(rows * blocks, dtype=np.uint64)
    keep = _exact_keep((n & np.uint64(0xFFFFFFFF), n >> np.uint64(32), 0, s["offset"]), s["seed"], s["dropout"])
    return torch.from_numpy(keep.reshape(rows, blocks * 8)[:, :width].copy()).cuda()


def exact(c, seed):
    s = prepare(c, seed)
    if c["op"] == "dropout":
        return {"y": s["x"].double() * _exact_rows_keep(s, c["rows"], c["width"])}
    return _exact_attention(s) if c["op"] == "attention" else _exact_norm(s)


def _exact_attention(s):
    B, H, Sq, Sk, D = (s[k] for k in ("batch", "heads", "q_len", "k_len", "head_dim"))
    group = H // s["kv_heads"]
    f64 = torch.float64
    O, L = torch.zeros(B, Sq, H, D, dtype=f64, device="cuda"), torch.full((B, H, Sq), -math.inf, dtype=f64, device="cuda")
    dQ, dK, dV = (torch.zeros(s[k].shape, dtype=f64, device="cuda") for k in "QKV")
    for b in range(B):
        nq = Sq if s["q_lens"] is None else int(s["q_lens"][b])
        nk = Sk if s["k_lens"] is None else int(s["k_lens"][b])
        first = max(0, nq - nk) if s["causal"] else 0            # the first query that sees a key
        if nk == 0 or first >= nq:
            continue
        for h in range(H):
            q, k, v = s["Q"][b, first:nq, h].double(), s["K"][b, :nk, h // group].double(), s["V"][b, :nk, h // group].double()
            z = q.mm(k.t().contiguous()) / math.sqrt(D)
            if s["causal"]:
                z += torch.full((nq - first, nk), -math.inf, dtype=f64, device="cuda").triu(diagonal=nk - nq + first + 1)
            L[b, h, first:nq] = torch.logsumexp(z, dim=1)
            p = torch.softmax(z, dim=1)
            del z
            keep = 1.0
            if s["dropout"] > 0:
                block, row = np.arange(-(-nk // 8), dtype=np.uint64)[None, :], np.arange(first, nq, dtype=np.uint64)[:, None]
                keep = torch.from_numpy(_exact_keep((block, row, b * H + h, s["offset"]), s["seed"], s["dropout"]).reshape(nq - first, -1)[:, :nk].copy()).cuda()
            O[b, first:nq, h] = (p * keep).mm(v)
            if s["train"]:
                g = s["dO"][b, first:nq, h].double()
                dV[b, :nk, h // group] += (p * keep).t().mm(g)
                dp = g.mm(v.t().contiguous()) * keep
                dz = p * (dp - (p * dp).sum(dim=1, keepdim=True)) / math.sqrt(D)
                dQ[b, first:nq, h] = dz.mm(k)
                dK[b, :nk, h // group] += dz.t().mm(q)
    out = {"O": O, "L": L}
    return dict(out, dQ=dQ, dK=dK, dV=dV) if s["train"] else out


def _exact_norm(s):
    f64 = torch.float64
    rows, width = s["rows"], s["width"]
    one = torch.ones(width, dtype=f64, device="cuda")

    def vector(key, other):
        return other if s[key] is None else s[key].double()

    def statistics(a, kind):
        """(centred rows, deviation)"""
        a = a - a.sum(dim=1, keepdim=True) / width if kind == "layer" else a
        return a, torch.sqrt(a.pow(2).sum(dim=1, keepdim=True) / width + _EPS)

    def gradient(d, a, dev, kind):
        """d/da of sum(d * centred(a) / dev(a))"""
        if kind == "none":
            return d
        e = d / dev - a * (d * a).sum(dim=1, keepdim=True) / (width * dev.pow(3))
        return e - e.sum(dim=1, keepdim=True) / width if kind == "layer" else e

    keep = _exact_rows_keep(s, rows, width) if s["dropout"] > 0 else 1.0
    x, f = s["x"].double(), s["f"].double()
    fc, fd = (f, 1.0) if s["post"] == "none" else statistics(f, s["post"])
    u = (fc / fd * vector("post_w", one) + vector("post_b", 0.0 * one)) * keep
    g = vector("g", one) * s["branch_scale"]
    y = s["residual_scale"] * x + g * u
    yc, yd = (y, 1.0) if s["pre"] == "none" else statistics(y, s["pre"])
    out = {"y": y, "h": yc / yd * vector("pre_w", one) + vector("pre_b", 0.0 * one)}
    if s["train"]:
        dh = s["dh"].double()
        dy = s["dy"].double() + gradient(dh * vector("pre_w", one), yc, yd, s["pre"])
        du = dy * g * keep
        out["dx"] = s["residual_scale"] * dy
        out["df"] = gradient(du * vector("post_w", one), fc, fd, s["post"])
        for name, there, value in (("dpre_w", s["pre_w"], dh * yc / yd), ("dpre_b", s["pre_b"], dh),
                                   ("dg", s["g"], s["branch_scale"] * dy * u),
                                   ("dpost_w", s["post_w"], du * fc / fd), ("dpost_b", s["post_b"], du)):
            if there is not None:
                out[name] = value.sum(dim=0)
    return out
