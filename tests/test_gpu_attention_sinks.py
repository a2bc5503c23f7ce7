"""One key with nearly all the weight and no value (a sink): the result consists of the other keys' probabilities, 2^-17 to 2^-23 of the largest each.

References and bounds as for the other sizes: a probability's rounding is relative to itself, however small it is beside the others."""
import math

import pytest
import torch

from test_gpu_attention import Call, _check, _normal
import operator_reference as ref

pytestmark = pytest.mark.gpu


def _sink(dtype, B, H, Hk, Sq, Sk, D, gap, at, backward):
    """Key `at` of every head scores `gap`, the others about half at most; values are of a size that leaves results among fp16's normal numbers."""
    Q, K, V = (_normal(seed, "f32", *shape) for seed, shape in ((1, (B, Sq, H, D)), (2, (B, Sk, Hk, D)), (3, (B, Sk, Hk, D))))
    Q[..., 0] = 1.0
    K *= 0.4 / math.sqrt(D)
    K[..., 0] = 0.0
    K[:, at] = 0.0
    K[:, at, :, 0] = gap
    V *= 64.0
    V[:, at] = 0.0
    dO = _normal(4, "f32", B, Sq, H, D) if backward else None
    return [None if t is None else t.to(Q.dtype if dtype == "f32" else {"f16": torch.float16, "bf16": torch.bfloat16}[dtype]) for t in (Q, K, V, dO)]


def _against_reference(dtype, B, H, Hk, Sq, Sk, D, gap, at=0, backward=False, heads=None, **options):
    Q, K, V, dO = _sink(dtype, B, H, Hk, Sq, Sk, D, gap, at, backward)
    options = {**dict(scale=1.0, causal=True), **options}
    got = Call(dtype, Q, K, V, dO, **options).run()
    f = [None if t is None else t.double().numpy() for t in (Q, K, V, dO)]
    for h in heads or [None]:                                       # (of long texts some heads are compared)
        if h is not None:
            g = h // (H // Hk)
            f = [t.double().numpy()[:, :, i:i + 1] for t, i in ((Q, h), (K, g), (V, g))] + [None]
        part = {n: t if h is None else t[:, :, h:h + 1] if n == "O" else t[:, h:h + 1] for n, t in got.items()}
        _check(part, ref.attention(*f[:3], dO=f[3], dtype=dtype, **options), (dtype, B, H, Hk, Sq, Sk, D, gap, at, options))


GAPS = [12.0, 14.0, 16.0]


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("gap", GAPS)
@pytest.mark.parametrize("D,at,causal", [(64, 0, True), (128, 0, True), (64, 299, False), (32, 150, False)])
def test_prompts(dtype, gap, D, at, causal):
    _against_reference(dtype, 2, 2, 1, 300, 300, D, gap, at, backward=True, causal=causal)


@pytest.mark.parametrize("gap", GAPS)
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("Sk,at", [(200, 0), (1024, 0), (3000, 2999), (3000, 1500)])
def test_few_queries(dtype, gap, Sk, at):
    """In one part of the keys and in several: the sink is in one of them, the others' weights are small beside it."""
    _against_reference(dtype, 1, 8, 2, 1, Sk, 128, gap, at, causal=False)
    _against_reference(dtype, 2, 4, 1, 5, Sk, 64, gap, at, causal=False, k_lens=[Sk, Sk - 1] if at < Sk - 1 else None)


@pytest.mark.parametrize("gap", GAPS)
@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_parts_of_the_keys(dtype, gap):
    """Few tiles of rows and long texts: the keys are shared by workgroups, in tiles of several query heads and of one."""
    _against_reference(dtype, 1, 4, 2, 40, 1700, 64, gap, causal=False)
    _against_reference(dtype, 1, 2, 2, 100, 1700, 128, gap, 1699, causal=False)


@pytest.mark.parametrize("gap", GAPS)
def test_with_dropout(gap):
    _against_reference("f16", 1, 2, 2, 200, 200, 64, gap, backward=True, dropout=0.3, seed=5)


@pytest.mark.parametrize("gap", GAPS)
def test_wide_heads_over_long_texts(gap):
    """Workgroups of eight waves."""
    _against_reference("f16", 2, 16, 4, 2048, 2048, 128, gap, heads=(0, 15))
