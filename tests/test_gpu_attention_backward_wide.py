"""Backward of wide heads, where values stay in LDS and 32 queries are worked on at a time, and of more workgroups than run at once.

Elements against the bounds of the other sizes.  And in 16 bits the norms of the errors: a rounding is off by half a unit in the last place at most, and O and
dV have two that are independent of one another (probabilities, result), dQ and dK three (O, gradients of scores, result), so with random inputs, whose
sums are as random as their errors, by no more than the root of so many squares of that, of the tensor's norm."""
import math

import numpy as np
import pytest

import operator_reference as ref
from test_gpu_attention import Call, _check, _problem

pytestmark = pytest.mark.gpu


def _against_reference(dtype, B, H, Hk, Sq, Sk, D, seed=1, **options):
    Q, K, V, dO = _problem(dtype, B, H, Hk, Sq, Sk, D, seed)
    options = {**dict(scale=1.0 / math.sqrt(D), causal=True), **options}
    got = Call(dtype, Q, K, V, dO, **options).run()
    f = [t.double().numpy() for t in (Q, K, V, dO)]
    want = ref.attention(*f[:3], dO=f[3], dtype=dtype, **options)
    _check(got, want, (dtype, B, H, Hk, Sq, Sk, D, options))
    if dtype == "f32":
        return
    for name, roundings in (("O", 2), ("dV", 2), ("dQ", 3), ("dK", 3)):
        value = want[name][0]
        off = np.linalg.norm(got[name].double().cpu().numpy() - value) / np.linalg.norm(value)
        assert off <= math.sqrt(roundings) * ref.U[dtype] / 2, (name, off)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("D", [96, 104, 120, 128])
@pytest.mark.parametrize("B,H,Hk,Sq,Sk", [(2, 4, 2, 300, 300), (1, 6, 2, 130, 517), (3, 2, 1, 517, 130), (2, 4, 1, 257, 257)])
def test_shared_heads_and_dropout(dtype, D, B, H, Hk, Sq, Sk):
    _against_reference(dtype, B, H, Hk, Sq, Sk, D)
    _against_reference(dtype, B, H, Hk, Sq, Sk, D, seed=3, dropout=0.2, causal=False, offset=5)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("dropout", [0.0, 0.1])
def test_texts_that_end_early(dtype, dropout):
    """Tiles without queries, without keys, and with some of both."""
    _against_reference(dtype, 5, 4, 2, 400, 400, 128, q_lens=[400, 129, 1, 0, 333], k_lens=[400, 129, 200, 400, 31], dropout=dropout)


@pytest.mark.parametrize("dtype,D,Hk,S", [("bf16", 128, 16, 640), ("f16", 128, 4, 640), ("bf16", 64, 16, 640), ("f16", 80, 4, 777), ("f32", 64, 8, 520)])
@pytest.mark.parametrize("dropout", [0.0, 0.1])
def test_more_workgroups_than_run_at_once(dtype, D, Hk, S, dropout):
    """64 heads of five tiles and more each, of queries and of keys: every XCD goes through several tiles of several heads."""
    _against_reference(dtype, 4, 16, Hk, S, S, D, dropout=dropout, seed=9)
