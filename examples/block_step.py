"""One transformer block trained with LSP-Offload's step: attention, norms with the residual, and dropout of this library between the block's
products (torch's), its four weight gradients through compress, the update in the subspace, and decompress-apply back into the weights.

    python examples/block_step.py [--steps K] [--dtype bf16] ...

The block is pre-norm: h = norm(x); x += drop(attention(h W_qkv) W_out); h = norm(x); x += drop(drop(relu(h W_up)) W_down); h = norm(x), every
"x += ...; h = norm(x)" one call.  The data are random, the loss is the mean square of h against a random target.  After the steps the last
position is computed once more as a decoder does it: one query over a cache of keys and values."""
from __future__ import annotations

import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2406_10181_amd as lsp

DTYPE = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


class Block:
    """Weights, buffers, descriptors and workspaces of one block for a batch of fixed size; made once, used by every step."""

    def __init__(self, batch=4, length=256, heads=8, kv_heads=4, head_dim=64, hidden=2048, dtype="bf16", dropout=0.1, seed=1):
        assert heads % kv_heads == 0 and head_dim % 8 == 0
        self.batch, self.length, self.heads, self.kv_heads, self.head_dim, self.dropout, self.seed = batch, length, heads, kv_heads, head_dim, dropout, seed
        self.rows, self.width, self.hidden, self.dtype, self.code = batch * length, heads * head_dim, hidden, dtype, lsp.DTYPE_CODE[dtype]
        g = torch.Generator().manual_seed(seed)
        new = lambda *shape: torch.empty(*shape, dtype=DTYPE[dtype], device="cuda")
        joint = (heads + 2 * kv_heads) * head_dim
        shapes = {"qkv": (joint, self.width), "out": (self.width, self.width), "up": (hidden, self.width), "down": (self.width, hidden)}
        self.weights = {k: (torch.randn(m, n, generator=g) / math.sqrt(n)).to(DTYPE[dtype]).cuda() for k, (m, n) in shapes.items()}
        self.norms = [torch.ones(self.width, dtype=DTYPE[dtype], device="cuda") for _ in range(3)]
        self.norm_grads = [torch.empty(self.width, device="cuda") for _ in range(3)]
        self.x = [new(self.rows, self.width) for _ in range(3)]             # the residual stream before, inside and behind the block
        self.h = [new(self.rows, self.width) for _ in range(3)]             # its norms
        self.stats = [torch.empty(4, self.rows, device="cuda") for _ in range(3)]
        self.qkv, self.dqkv = new(self.rows, joint), new(self.rows, joint)
        self.o, self.do = (new(batch, length, heads, head_dim) for _ in range(2))
        self.logs = torch.empty(batch, heads, length, device="cuda")
        self.a, self.f = new(self.rows, self.width), new(self.rows, self.width)
        self.act, self.dact = new(self.rows, hidden), new(self.rows, hidden)
        self.dx = [new(self.rows, self.width) for _ in range(2)]
        self.da, self.df, self.dh = (new(self.rows, self.width) for _ in range(3))
        self.k_lens = torch.full((batch,), length, dtype=torch.int32, device="cuda")
        self._describe()

    @property
    def stream(self):
        """The stream of torch's products, whichever it is at the call."""
        return torch.cuda.current_stream()

    def heads_of(self, joint):
        """Views of a joint projection [rows][...] as Q, K and V with heads."""
        t = joint.view(self.batch, self.length, -1, self.head_dim)
        return t.split([self.heads, self.kv_heads, self.kv_heads], dim=2)

    def _describe(self):
        drop = dict(dropout=self.dropout, seed=self.seed)
        q, k, v = self.heads_of(self.qkv)
        self.attention = lsp.attention_problem(q, k, v, self.o, self.logs, q_lens=self.k_lens, k_lens=self.k_lens, scale=1 / math.sqrt(self.head_dim), causal=True, **drop)
        self.attention_grads = lsp.attention_gradients(self.do, *self.heads_of(self.dqkv))
        norm = lambda i, x, f, y, **more: lsp.residual_norm_problem(x, f, y, self.h[i], self.stats[i], pre="rms", pre_weight=self.norms[i], **more)
        self.residual = [norm(0, self.x[0], self.x[0], self.x[0], branch_scale=0.0), norm(1, self.x[0], self.a, self.x[1], **drop), norm(2, self.x[1], self.f, self.x[2], **drop)]
        # from the back: the gradients of x[2] and h[2] give those of x[1] and f, then those of x[1] and h[1] give those of x[0] and a
        self.residual_grads = {2: lsp.residual_norm_gradients(self.dx[0], self.dh, self.dx[1], self.df, pre_weight=self.norm_grads[2]),
                               1: lsp.residual_norm_gradients(self.dx[1], self.dh, self.dx[0], self.da, pre_weight=self.norm_grads[1])}
        take = lambda n: (torch.empty(max(n, 16), dtype=torch.uint8, device="cuda"), n)
        self.forward_room = take(lsp.lsp_attention_forward_workspace_bytes(self.attention, self.code))
        self.backward_room = take(lsp.lsp_attention_backward_workspace_bytes(self.attention, self.code))
        self.norm_room = take(lsp.lsp_residual_norm_backward_workspace_bytes(self.residual[1], self.code))

    def number(self, problem, offset):
        """Masks of this step: every place that drops takes an offset of its own."""
        problem.offset = offset
        return problem

    def forward(self, step=0):
        """x[0] to h[2]."""
        w, code, s = self.weights, self.code, self.stream
        lsp.lsp_residual_norm_forward(self.residual[0], code, s)
        torch.mm(self.h[0], w["qkv"].t(), out=self.qkv)
        lsp.lsp_attention_forward(self.number(self.attention, 4 * step), code, *self.forward_room, s)
        torch.mm(self.o.view(self.rows, -1), w["out"].t(), out=self.a)
        lsp.lsp_residual_norm_forward(self.number(self.residual[1], 4 * step + 1), code, s)
        torch.mm(self.h[1], w["up"].t(), out=self.act).relu_()
        lsp.lsp_dropout(self.act, self.act, self.rows, self.hidden, self.dropout, self.seed, 4 * step + 2, code, s)
        torch.mm(self.act, w["down"].t(), out=self.f)
        lsp.lsp_residual_norm_forward(self.number(self.residual[2], 4 * step + 3), code, s)
        return self.h[2]

    def backward(self, grad, step=0):
        """From the gradient of h[2] to those of the weights, by name; the masks are made again."""
        w, code, s = self.weights, self.code, self.stream
        self.dh.copy_(grad)
        self.dx[0].zero_()
        lsp.lsp_residual_norm_backward(self.number(self.residual[2], 4 * step + 3), self.residual_grads[2], code, *self.norm_room, s)
        grads = {"down": self.df.t() @ self.act}
        torch.mm(self.df, w["down"], out=self.dact)
        lsp.lsp_dropout(self.dact, self.dact, self.rows, self.hidden, self.dropout, self.seed, 4 * step + 2, code, s)
        self.dact.mul_(self.act > 0)                                          # (dropped or cut off: both are zero in `act` and get none)
        grads["up"] = self.dact.t() @ self.h[1]
        torch.mm(self.dact, w["up"], out=self.dh)
        lsp.lsp_residual_norm_backward(self.number(self.residual[1], 4 * step + 1), self.residual_grads[1], code, *self.norm_room, s)
        grads["out"] = self.da.t() @ self.o.view(self.rows, -1)
        torch.mm(self.da, w["out"], out=self.do.view(self.rows, -1))
        lsp.lsp_attention_backward(self.number(self.attention, 4 * step), self.attention_grads, code, *self.backward_room, s)
        grads["qkv"] = self.dqkv.t() @ self.h[0]
        return grads

    def last_position(self):
        """h[2] of the last position of every text without dropout, from one query a text over the keys and values that forward() left in `qkv`:
        a cache that is a view, read by a call for single tokens."""
        w, code, s, b = self.weights, self.code, self.stream, self.batch
        last = lambda t: t.view(b, self.length, -1)[:, -1]
        q, k, v = self.heads_of(self.qkv)
        o = torch.empty(b, 1, self.heads, self.head_dim, dtype=q.dtype, device="cuda")
        logs = torch.empty(b, self.heads, 1, device="cuda")
        p = lsp.attention_problem(q[:, -1:], k, v, o, logs, k_lens=self.k_lens, scale=1 / math.sqrt(self.head_dim), causal=True)
        n = lsp.lsp_attention_forward_workspace_bytes(p, code)
        room = torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")
        lsp.lsp_attention_forward(p, code, room, n, s)
        x, h, stats = last(self.x[0]).clone(), torch.empty(b, self.width, dtype=q.dtype, device="cuda"), torch.empty(4, b, device="cuda")
        f = o.view(b, -1) @ w["out"].t()
        lsp.lsp_residual_norm_forward(lsp.residual_norm_problem(x, f, x, h, stats, pre="rms", pre_weight=self.norms[1]), code, s)
        f = (h @ w["up"].t()).relu_() @ w["down"].t()
        lsp.lsp_residual_norm_forward(lsp.residual_norm_problem(x, f, x, h, stats, pre="rms", pre_weight=self.norms[2]), code, s)
        return h


class Subspace:
    """A weight's (d, r)-sparse projectors with random values, their plan, and the calls of a step."""

    def __init__(self, weight, r, d, code, generator):
        self.weight, self.r, self.d, self.code = weight, r, d, code
        self.m, self.n = weight.shape
        sparse = lambda rows: (torch.rand(rows, r, generator=generator).argsort(1)[:, :d].int().cuda().contiguous(),
                               (torch.randn(rows, d, generator=generator) * math.sqrt(r / (rows * d))).cuda())     # columns of length one in the mean
        (self.pi, self.pv), (self.qi, self.qv) = sparse(self.m), sparse(self.n)
        size = lsp.lsp_plan_bytes(self.m, self.n, r, d)
        self.plan = torch.empty(size, dtype=torch.uint8, device="cuda")
        lsp.lsp_plan_build(self.pi, self.pv, self.qi, self.qv, self.m, self.n, r, d, self.plan, size, torch.cuda.current_stream())
        self.room = torch.empty(lsp.lsp_compress_planned_workspace_bytes(self.m, self.n, r, d), dtype=torch.uint8, device="cuda")
        self.S = torch.empty(r, r, device="cuda")

    def compress(self, gradient, stream):
        lsp.lsp_compress_planned(gradient, self.plan, self.m, self.n, self.r, self.d, self.S, self.code, self.room, self.room.numel(), stream)
        return self.S

    def apply(self, delta, stream):
        self.S.copy_(delta)
        lsp.lsp_decompress_apply(self.weight, self.S, self.pi, self.pv, self.qi, self.qv, self.m, self.n, self.r, self.d, self.code, stream)


def train(block, steps=8, r=128, d=4, rate=0.5):
    """`steps` steps on one batch; the losses.  The update in the subspace is made on the CPU: plain gradient descent stands for the optimizer there."""
    g = torch.Generator().manual_seed(block.seed + 1)
    draw = lambda: torch.randn(block.rows, block.width, generator=g).to(DTYPE[block.dtype]).cuda()
    block.x[0].copy_(draw())
    target = draw().float()
    spaces = {k: Subspace(w, r, d, block.code, g) for k, w in block.weights.items()}
    losses = []
    for step in range(steps):
        off = block.forward(step).float() - target
        losses.append(float(off.square().mean()))
        for name, gradient in block.backward(off * (2.0 / block.rows), step).items():                # (of the loss times the width: fp16 keeps it)
            received = spaces[name].compress(gradient.contiguous(), block.stream).cpu()
            spaces[name].apply((rate * received).cuda(), block.stream)
    return losses


def main():
    a = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("steps", 8), ("batch", 4), ("length", 256), ("heads", 8), ("kv-heads", 4), ("head-dim", 64), ("hidden", 2048), ("subspace", 128), ("entries", 4)):
        a.add_argument("--" + name, type=int, default=value)
    a.add_argument("--dropout", type=float, default=0.1)
    a.add_argument("--rate", type=float, default=0.5)
    a.add_argument("--dtype", choices=sorted(DTYPE), default="bf16")
    o = a.parse_args()
    block = Block(o.batch, o.length, o.heads, o.kv_heads, o.head_dim, o.hidden, o.dtype, o.dropout)
    for step, loss in enumerate(train(block, o.steps, o.subspace, o.entries, o.rate)):
        print(f"step {step}: loss {loss:.5f}")
    block.dropout = 0.0
    block._describe()
    whole = block.forward().view(o.batch, o.length, -1)[:, -1].float()
    print(f"last position from the cache: off by {float((block.last_position().float() - whole).abs().max()):.4f} at most, of values up to {float(whole.abs().max()):.2f}")


if __name__ == "__main__":
    main()
