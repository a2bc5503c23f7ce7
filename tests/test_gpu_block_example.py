"""The example's block: its gradients against automatic differentiation in 64 bits with the same masks, its steps, and its last position by one query.

Bounds, of a tensor's norm: each of the twelve stages in a row is off by a sum of at most 512 terms in fp32, 512 * 2^-24; in 16 bits by two roundings."""
import math
import os
import sys

import pytest
import torch

import operator_reference as ref

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import block_step

pytestmark = pytest.mark.gpu
STAGES = 12


def _bound(dtype):
    return STAGES * (512 * ref.EPS + (0.0 if dtype == "f32" else 2 * ref.U[dtype]))


def _reference(block, x, grad, step):
    """h[2] and the gradients by name, float64 on the CPU."""
    B, S, H, Hk, D, p, seed = block.batch, block.length, block.heads, block.kv_heads, block.head_dim, block.dropout, block.seed
    w = {k: t.double().cpu().requires_grad_() for k, t in block.weights.items()}
    n = [t.double().cpu().requires_grad_() for t in block.norms]
    matrix = lambda width, place: torch.from_numpy(ref.keep_matrix(B * S, width, seed, 4 * step + place, p))
    norm = lambda v, i: v / (v.square().mean(1, keepdim=True) + 1e-5).sqrt() * n[i]
    q, k, v = (norm(x, 0) @ w["qkv"].t()).view(B, S, -1, D).split([H, Hk, Hk], dim=2)
    k, v = (t.repeat_interleave(H // Hk, dim=2) for t in (k, v))
    scores = torch.einsum("bqhd,bkhd->bhqk", q, k) / math.sqrt(D)
    scores = scores.masked_fill(torch.ones(S, S, dtype=torch.bool).triu(1), -math.inf)
    keep = torch.stack([torch.from_numpy(ref.keep_probabilities(i, S, S, seed, 4 * step, p)) for i in range(B * H)]).view(B, H, S, S)
    o = torch.einsum("bhqk,bkhd->bqhd", scores.softmax(-1) * keep, v).reshape(B * S, -1)
    x = x + matrix(block.width, 1) * (o @ w["out"].t())
    act = matrix(block.hidden, 2) * (norm(x, 1) @ w["up"].t()).relu()
    x = x + matrix(block.width, 3) * (act @ w["down"].t())
    h = norm(x, 2)
    h.backward(grad)
    return h.detach(), {**{k: t.grad for k, t in w.items()}, **{f"norm {i}": n[i].grad for i in (1, 2)}}


@pytest.mark.parametrize("heads,kv_heads,head_dim,length", [(4, 2, 32, 37), (2, 2, 64, 130)])
def test_gradients(heads, kv_heads, head_dim, length):
    block = block_step.Block(2, length, heads, kv_heads, head_dim, 200, "f32", 0.2)
    g = torch.Generator().manual_seed(3)
    x, grad = (torch.randn(block.rows, block.width, generator=g) for _ in range(2))
    block.x[0].copy_(x)
    for step in (0, 5):
        h = block.forward(step).clone()
        got = block.backward(grad.cuda(), step)
        got.update({f"norm {i}": block.norm_grads[i] for i in (1, 2)})
        want_h, want = _reference(block, x.double(), grad.double(), step)
        for name, value in (("h", want_h), *want.items()):
            off = (h if name == "h" else got[name]).double().cpu() - value
            assert off.norm() <= _bound("f32") * value.norm(), (step, name, float(off.norm() / value.norm()))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_steps(dtype):
    losses = block_step.train(block_step.Block(batch=2, length=100, hidden=512, dtype=dtype), steps=4, r=64)
    assert all(math.isfinite(x) for x in losses) and losses[-1] < losses[0], losses


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_last_position(dtype):
    block = block_step.Block(batch=3, length=300, hidden=512, dtype=dtype, dropout=0.0)
    block.x[0].copy_(torch.randn(block.rows, block.width, generator=torch.Generator().manual_seed(4)))
    whole = block.forward().view(3, 300, -1)[:, -1].double()
    off = block.last_position().double() - whole
    assert off.norm() <= _bound(dtype) * whole.norm(), float(off.norm() / whole.norm())
