"""A small language model trained with all of this library: the block of block_step.py with rotary positions and norms of query and key heads, an embedding, and the cross
entropy over a vocabulary behind it.  The block's four matrices take LSP-Offload's step (compress, the update in the subspace, decompress-apply); what has no projector --
the embedding, the vocabulary's matrix, the norms -- takes AdamW, one call for all of it, with states in 8 bits.

    python examples/language_step.py [--steps K] [--dtype bf16] ...

The text is a made-up one in which each word says what the next one is likely to be.  After the steps some words are generated, one at a time, over a cache that the rotary call
fills and attention reads."""
from __future__ import annotations

import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from block_step import DTYPE, Block, Subspace, lsp


class Model(Block):
    """Embedding, block and loss for a batch of texts of one length; descriptors and workspaces are made once."""

    def __init__(self, vocab=1000, batch=4, length=128, dtype="bf16", **block):
        self.vocab = vocab
        self.base = 10000.0
        super().__init__(batch=batch, length=length, dtype=dtype, **block)
        g = torch.Generator().manual_seed(self.seed + 7)
        t = DTYPE[dtype]
        self.embedding = torch.randn(vocab, self.width, generator=g).to(t).cuda()
        self.head = (torch.randn(vocab, self.width, generator=g) / math.sqrt(self.width)).to(t).cuda()
        self.head_grad = torch.empty_like(self.head)
        self.targets = torch.empty(self.rows, dtype=torch.int64, device="cuda")
        self.losses = torch.empty(self.rows, device="cuda")
        self.loss = lsp.cross_entropy_problem(self.h[2], self.head, self.targets, self.losses)
        self.loss_grads = lsp.cross_entropy_gradients(self.dh, self.head_grad, scale=1.0 / self.rows)
        n = lsp.lsp_cross_entropy_backward_workspace_bytes(self.loss, self.code)
        self.loss_room = (torch.empty(max(n, 16), dtype=torch.uint8, device="cuda"), n)

    def _describe(self):
        super()._describe()
        new = lambda heads, length=self.length: torch.empty(self.batch, length, heads, self.head_dim, dtype=DTYPE[self.dtype], device="cuda")
        if not hasattr(self, "head_norms"):
            self.head_norms = {k: torch.ones(self.head_dim, dtype=DTYPE[self.dtype], device="cuda") for k in ("q", "k")}
            self.head_norm_grads = {k: torch.empty(self.head_dim, device="cuda") for k in ("q", "k")}
            self.frequencies = (self.base ** (-torch.arange(0, self.head_dim, 2, dtype=torch.float64) / self.head_dim)).float().cuda()
            self.qr, self.kr = new(self.heads), new(self.kv_heads)
            self.under = torch.empty_like(self.x[0])
        q, k, v = self.heads_of(self.qkv)
        self.norms_of_heads = dict(frequencies=self.frequencies, norm="rms", q_weight=self.head_norms["q"], k_weight=self.head_norms["k"])
        self.rotary = lsp.rotary_problem(q, k, self.qr, self.kr, **self.norms_of_heads)
        dq, dk, _ = self.heads_of(self.dqkv)
        self.rotary_grads = lsp.rotary_gradients(dq, dk, dq, dk, q_weight=self.head_norm_grads["q"], k_weight=self.head_norm_grads["k"])
        n = lsp.lsp_rotary_backward_workspace_bytes(self.rotary, self.code)
        self.rotary_room = (torch.empty(max(n, 16), dtype=torch.uint8, device="cuda"), n)
        self.attention = lsp.attention_problem(self.qr, self.kr, v, self.o, self.logs, q_lens=self.k_lens, k_lens=self.k_lens, scale=1 / math.sqrt(self.head_dim), causal=True,
                                               dropout=self.dropout, seed=self.seed)
        # the first norm again, with its input and what goes on apart, as its backward pass wants them
        self.first = lsp.residual_norm_problem(self.x[0], self.x[0], self.under, self.h[0], self.stats[0], pre="rms", pre_weight=self.norms[0], branch_scale=0.0)
        self.first_grads = lsp.residual_norm_gradients(self.dx[0], self.dh, self.dx[1], self.df, pre_weight=self.norm_grads[0])

    def turn(self):
        lsp.lsp_rotary_forward(self.rotary, self.code, self.stream)

    def turn_back(self):
        lsp.lsp_rotary_backward(self.rotary, self.rotary_grads, self.code, *self.rotary_room, self.stream)

    def forward_backward(self, words, targets, step=0):
        """words, targets: [batch][length].  The mean loss, and all gradients by name."""
        w, code, s = self.weights, self.code, self.stream
        self.x[0].copy_(self.embedding[words.reshape(-1)])
        self.targets.copy_(targets.reshape(-1))
        self.forward(step)
        lsp.lsp_cross_entropy_backward(self.loss, self.loss_grads, code, *self.loss_room, s)
        grads = self.backward(self.dh, step)
        torch.mm(self.dqkv, w["qkv"], out=self.dh)
        lsp.lsp_residual_norm_backward(self.first, self.first_grads, code, *self.norm_room, s)
        embedding = torch.zeros(self.vocab, self.width, device="cuda").index_add_(0, words.reshape(-1), self.dx[1].float())
        grads.update({f"norm {i}": self.norm_grads[i] for i in range(3)}, head=self.head_grad, embedding=embedding, q=self.head_norm_grads["q"], k=self.head_norm_grads["k"])
        return self.losses.mean(), grads

    def others(self):
        """The parameters that have no projector, by the names of their gradients."""
        return {**{f"norm {i}": t for i, t in enumerate(self.norms)}, "head": self.head, "embedding": self.embedding, **self.head_norms}

    def generate(self, words, count):
        """`count` more words behind words [batch][length]: each the likeliest, from one query a text over a cache of keys and values."""
        w, code, b, room = self.weights, self.code, self.batch, words.shape[1] + count
        t = DTYPE[self.dtype]
        new = lambda *shape: torch.empty(*shape, dtype=t, device="cuda")
        K, V = (torch.zeros(b, room, self.kv_heads, self.head_dim, dtype=t, device="cuda") for _ in range(2))
        out, stats = list(words.t()), torch.empty(4, b, device="cuda")
        for i in range(room - 1):
            x = self.embedding[out[i]]
            h, q, o, logs = torch.empty_like(x), new(b, 1, self.heads, self.head_dim), new(b, 1, self.heads, self.head_dim), torch.empty(b, self.heads, 1, device="cuda")
            lsp.lsp_residual_norm_forward(lsp.residual_norm_problem(x, x, x, h, stats, pre="rms", pre_weight=self.norms[0], branch_scale=0.0), code, self.stream)
            joint = (h @ w["qkv"].t()).view(b, 1, -1, self.head_dim)
            starts = torch.full((b,), i, dtype=torch.int32, device="cuda")
            q0, k0, v0 = joint.split([self.heads, self.kv_heads, self.kv_heads], dim=2)
            lsp.lsp_rotary_forward(lsp.rotary_problem(q0, k0, q, K, V=v0, Vr=V, starts=starts, **self.norms_of_heads), code, self.stream)
            p = lsp.attention_problem(q, K, V, o, logs, k_lens=starts + 1, scale=1 / math.sqrt(self.head_dim), causal=True)
            n = lsp.lsp_attention_forward_workspace_bytes(p, code)
            scratch = torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")
            lsp.lsp_attention_forward(p, code, scratch, n, self.stream)
            f = o.view(b, -1) @ w["out"].t()
            lsp.lsp_residual_norm_forward(lsp.residual_norm_problem(x, f, x, h, stats, pre="rms", pre_weight=self.norms[1]), code, self.stream)
            f = (h @ w["up"].t()).relu_() @ w["down"].t()
            lsp.lsp_residual_norm_forward(lsp.residual_norm_problem(x, f, x, h, stats, pre="rms", pre_weight=self.norms[2]), code, self.stream)
            self.last = h                                                     # (what the vocabulary is asked with)
            if i + 1 >= words.shape[1]:
                out.append((h @ self.head.t()).argmax(1))
        return torch.stack(out, dim=1)


class Optimizer:
    """AdamW for what has no projector: gradients in fp32 buffers of their own, states in 8 bits."""

    def __init__(self, parameters, rate):
        self.rate, self.step, self.grads, items = rate, 0, {}, []
        for name, p in parameters.items():
            n = p.numel()
            self.grads[name] = torch.empty(p.shape, device="cuda")
            states = {k: torch.zeros(n, dtype=torch.uint8, device="cuda") for k in ("m", "v")}
            scales = {k: torch.zeros((n + 255) // 256, device="cuda") for k in ("m_scale", "v_scale")}
            master = p.float() if p.dtype != torch.float32 else None
            items.append(dict(param=p, grad=self.grads[name], master=master, decay=0.01 if p.dim() > 1 else 0.0, **states, **scales))
        self.kept, self.items = items, lsp.adamw_items(items)

    def apply(self, grads, stream):
        self.step += 1
        for name, g in self.grads.items():
            g.copy_(grads[name])
        norm = torch.linalg.vector_norm(torch.stack([torch.linalg.vector_norm(g) for g in self.grads.values()]))
        lsp.lsp_adamw(self.items, rate=self.rate, step=self.step, grad_scale=(1.0 / (norm + 1e-6)).clamp_(max=1.0), stream=stream)


def text(model, generator):
    """[batch][length + 1]: word n is followed by 3 n + 1 modulo the vocabulary, in nine cases of ten."""
    words = [torch.randint(0, model.vocab, (model.batch,), generator=generator)]
    for _ in range(model.length):
        guess = torch.randint(0, model.vocab, (model.batch,), generator=generator)
        words.append(torch.where(torch.rand(model.batch, generator=generator) < 0.9, (3 * words[-1] + 1) % model.vocab, guess))
    return torch.stack(words, dim=1).cuda()


def train(model, steps=8, r=128, d=4, rate=0.2, adam_rate=3e-3):
    g = torch.Generator().manual_seed(model.seed + 1)
    spaces = {k: Subspace(w, r, d, model.code, g) for k, w in model.weights.items()}
    optimizer = Optimizer(model.others(), adam_rate)
    losses = []
    for step in range(steps):
        words = text(model, g)
        loss, grads = model.forward_backward(words[:, :-1], words[:, 1:], step)
        losses.append(float(loss))
        for name, space in spaces.items():
            received = space.compress(grads[name].contiguous(), model.stream).cpu()
            space.apply((rate * received).cuda(), model.stream)
        optimizer.apply(grads, model.stream)
    return losses


def main():
    a = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("steps", 40), ("vocab", 1000), ("batch", 8), ("length", 128), ("heads", 8), ("kv-heads", 4), ("head-dim", 64), ("hidden", 2048), ("subspace", 128), ("entries", 4)):
        a.add_argument("--" + name, type=int, default=value)
    a.add_argument("--dropout", type=float, default=0.0)
    a.add_argument("--dtype", choices=sorted(DTYPE), default="bf16")
    o = a.parse_args()
    model = Model(o.vocab, o.batch, o.length, o.dtype, heads=o.heads, kv_heads=o.kv_heads, head_dim=o.head_dim, hidden=o.hidden, dropout=o.dropout)
    for step, loss in enumerate(train(model, o.steps, o.subspace, o.entries)):
        print(f"step {step}: loss {loss:.5f}")
    words = model.generate(text(model, torch.Generator().manual_seed(5))[:, :4], 6)
    print("words:", words[0].tolist())


if __name__ == "__main__":
    main()
