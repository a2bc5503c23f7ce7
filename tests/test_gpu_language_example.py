"""The language model of the examples: its gradients against automatic differentiation in 64 bits, its steps in every type, and its words one at a time against all at once.

Bounds, of a tensor's norm: each of the sixteen stages in a row is off by a sum of at most 512 terms in fp32, 512 * 2^-24; in 16 bits by two roundings."""
import math
import os
import sys

import pytest
import torch

import operator_reference as ref

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import language_step

pytestmark = pytest.mark.gpu
STAGES = 16


def _bound(dtype):
    return STAGES * (512 * ref.EPS + (0.0 if dtype == "f32" else 2 * ref.U[dtype]))


def _reference(m, words, targets, step):
    """(mean loss, gradients by name), float64 on the CPU."""
    B, S, H, Hk, D, p, seed = m.batch, m.length, m.heads, m.kv_heads, m.head_dim, m.dropout, m.seed
    leaf = lambda t: t.double().cpu().requires_grad_()
    w, n = {k: leaf(t) for k, t in m.weights.items()}, [leaf(t) for t in m.norms]
    E, head, hn = leaf(m.embedding), leaf(m.head), {k: leaf(t) for k, t in m.head_norms.items()}
    matrix = lambda width, place: torch.from_numpy(ref.keep_matrix(B * S, width, seed, 4 * step + place, p)) if p else 1.0
    rms = lambda v, weight: v / (v.square().mean(-1, keepdim=True) + 1e-5).sqrt() * weight
    angle = torch.outer(torch.arange(S, dtype=torch.float64), m.frequencies.double().cpu())
    turn = torch.polar(torch.ones_like(angle), angle)[None, :, None, :]

    def turned(v):
        z = torch.view_as_real(torch.complex(*v.chunk(2, dim=-1)) * turn)
        return torch.cat([z[..., 0], z[..., 1]], dim=-1)

    x = E[words.cpu().reshape(-1)]
    q, k, v = (rms(x, n[0]) @ w["qkv"].t()).view(B, S, -1, D).split([H, Hk, Hk], dim=2)
    q, k = turned(rms(q, hn["q"])), turned(rms(k, hn["k"]))
    k, v = (t.repeat_interleave(H // Hk, dim=2) for t in (k, v))
    scores = torch.einsum("bqhd,bkhd->bhqk", q, k) / math.sqrt(D)
    scores = scores.masked_fill(torch.ones(S, S, dtype=torch.bool).triu(1), -math.inf)
    keep = torch.stack([torch.from_numpy(ref.keep_probabilities(i, S, S, seed, 4 * step, p)) for i in range(B * H)]).view(B, H, S, S) if p else 1.0
    o = torch.einsum("bhqk,bkhd->bqhd", scores.softmax(-1) * keep, v).reshape(B * S, -1)
    x = x + matrix(m.width, 1) * (o @ w["out"].t())
    x = x + matrix(m.width, 3) * ((matrix(m.hidden, 2) * (rms(x, n[1]) @ w["up"].t()).relu()) @ w["down"].t())
    loss = torch.nn.functional.cross_entropy(rms(x, n[2]) @ head.t(), targets.cpu().reshape(-1))
    loss.backward()
    return float(loss.detach()), {**{k: t.grad for k, t in w.items()}, **{f"norm {i}": n[i].grad for i in range(3)}, "head": head.grad, "embedding": E.grad, "q": hn["q"].grad, "k": hn["k"].grad}


@pytest.mark.parametrize("heads,kv_heads,head_dim,length,dropout", [(4, 2, 32, 37, 0.2), (2, 2, 64, 130, 0.0)])
def test_gradients(heads, kv_heads, head_dim, length, dropout):
    m = language_step.Model(301, 2, length, "f32", heads=heads, kv_heads=kv_heads, head_dim=head_dim, hidden=200, dropout=dropout)
    g = torch.Generator().manual_seed(3)
    for t in [*m.norms, *m.head_norms.values()]:
        t.copy_(1 + 0.2 * torch.randn(t.shape, generator=g))
    for step in (0, 3):
        words = language_step.text(m, g)
        loss, got = m.forward_backward(words[:, :-1], words[:, 1:], step)
        want_loss, want = _reference(m, words[:, :-1], words[:, 1:], step)
        assert abs(float(loss) - want_loss) <= _bound("f32") * want_loss
        assert set(want) == set(got)
        for name, value in want.items():
            off = got[name].double().cpu() - value
            assert off.norm() <= _bound("f32") * value.norm(), (step, name, float(off.norm() / value.norm()))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_steps(dtype):
    m = language_step.Model(500, 2, 100, dtype, heads=4, kv_heads=2, head_dim=32, hidden=512, dropout=0.1)
    before = {k: t.clone() for k, t in {**m.weights, **m.others()}.items()}
    losses = language_step.train(m, steps=3, r=64)
    assert all(math.isfinite(x) for x in losses), losses
    assert all(bool(torch.isfinite(t).all()) and not torch.equal(before[k], t) for k, t in {**m.weights, **m.others()}.items())


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_words_one_at_a_time(dtype):
    """The last position's hidden state, over a cache filled word by word, against the whole text at once."""
    m = language_step.Model(300, 3, 40, dtype, heads=4, kv_heads=2, head_dim=64, hidden=300, dropout=0.0)
    words = language_step.text(m, torch.Generator().manual_seed(4))
    m.x[0].copy_(m.embedding[words[:, :-1].reshape(-1)])
    whole = m.forward().view(3, 40, -1)[:, -1].double()
    out = m.generate(words[:, :40], 1)
    off = m.last.double() - whole
    assert off.norm() <= _bound(dtype) * whole.norm(), float(off.norm() / whole.norm())
    assert torch.equal(out[:, :40], words[:, :40]) and out.shape == (3, 41)
