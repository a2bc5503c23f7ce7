"""Attention where the choice of kernels changes: wide heads over long texts, few rows with and without a split of the keys, tiles shared by workgroups.

References and bounds as for the other sizes; of the long texts some heads are compared."""
import math

import pytest
import torch

import operator_reference as ref
import paper_2406_10181_amd as L
from test_gpu_attention import _CODE, Call, _against_reference, _check, _normal, _problem

pytestmark = pytest.mark.gpu


def _heads_of(got, Q, K, V, dtype, heads, **options):
    """O and L of some heads of every text against the reference of these heads alone."""
    group = Q.shape[2] // K.shape[2]
    for h in heads:
        q, k, v = (t[:, :, i:i + 1].double().numpy() for t, i in ((Q, h), (K, h // group), (V, h // group)))
        want = ref.attention(q, k, v, dtype=dtype, **options)
        _check({"O": got["O"][:, :, h:h + 1], "L": got["L"][:, h:h + 1]}, want, (dtype, h, options))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("causal,D,Sq,Sk,lens", [(True, 128, 2048, 2048, None), (False, 80, 1801, 2111, None), (True, 128, 2300, 2048, None), (True, 96, 2048, 2049, [2049, 700]),
                                                 (False, 128, 300, 2500, [0, 2047])])
def test_wide_heads_over_long_texts(dtype, causal, D, Sq, Sk, lens):
    """Workgroups of eight waves where there are enough of them: rows in front of the keys, odd lengths, texts that end early."""
    H = {2048: 16, 1801: 16, 2300: 16, 300: 64}[Sq]
    Q, K, V, _ = _problem(dtype, 2, H, H // 4, Sq, Sk, D, backward=False)
    options = dict(scale=1.0 / math.sqrt(D), causal=causal, k_lens=lens)
    got = Call(dtype, Q, K, V, **options).run()
    _heads_of(got, Q, K, V, dtype, (0, H - 1), **options)


def test_wide_heads_over_long_texts_with_dropout():
    """Head 0 of the one text has the reference's counters."""
    Q, K, V, _ = _problem("bf16", 1, 32, 8, 2048, 2048, 128, backward=False)
    options = dict(scale=0.09, causal=True, dropout=0.1, seed=9, offset=2)
    got = Call("bf16", Q, K, V, **options).run()
    _heads_of(got, Q, K, V, "bf16", (0,), **options)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("D", [8, 24, 64, 72, 96, 120, 128])
@pytest.mark.parametrize("B,H,Hk,Sq,Sk", [(2, 8, 2, 1, 31), (1, 32, 1, 1, 257), (3, 4, 4, 7, 33), (1, 6, 2, 10, 1025), (40, 32, 32, 1, 65)])
def test_rows_of_one_tile(dtype, D, B, H, Hk, Sq, Sk):
    """Up to 32 rows a key head: one part of the keys and several, parts that end inside a tile, head dimensions round the tiles' widths."""
    for causal in (False, True):
        _against_reference(dtype, B, H, Hk, Sq, Sk, D, backward=False, causal=causal, k_lens=None if B == 1 else [Sk - 3 * b % Sk for b in range(B)])


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_one_token_of_a_long_cache(dtype):
    """One query a text, caches filled to different lengths, the empty one and those that leave whole parts without keys among them; the cache is a
    view, and what lies behind the lengths is not a number."""
    B, H, Hk, S, D, lens = 6, 16, 4, 5000, 128, [5000, 1, 0, 4097, 129, 2500]
    Q, K, V, _ = _problem(dtype, B, H, Hk, 1, S, D, backward=False)
    for b, n in enumerate(lens):
        K[b, n:], V[b, n:] = float("nan"), float("inf")
    joint = torch.stack([K, V], dim=2)                              # keys and values of a position side by side
    options = dict(scale=1.0 / math.sqrt(D), causal=True, k_lens=lens)
    got = Call(dtype, Q, joint[:, :, 0], joint[:, :, 1], **options).run()
    _heads_of(got, Q, K.nan_to_num(0, 0, 0), V.nan_to_num(0, 0, 0), dtype, range(0, H, 5), **options)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("B,H,Hk,Sq,Sk", [(1, 2, 1, 40, 1700), (1, 4, 1, 900, 60), (1, 1, 1, 1030, 1030)])
def test_tiles_shared_by_workgroups(dtype, B, H, Hk, Sq, Sk):
    """Few tiles, long sums: parts of dQ, of dK and dV, and of all of them are added in a launch of their own."""
    _against_reference(dtype, B, H, Hk, Sq, Sk, 64, causal=True)
    _against_reference(dtype, B, H, Hk, Sq, Sk, 40, dropout=0.25, seed=3, k_lens=[Sk - 11])


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_the_choice_of_kernel_is_no_part_of_the_result(dtype):
    """A text's rows are the same, within both calls' bounds, whether they come one at a time, some at a time or together."""
    H, S, D = 4, 700, 64
    Q, K, V, _ = _problem(dtype, 1, H, 2, S, S, D, backward=False)
    options = dict(scale=0.125, causal=True)
    whole = Call(dtype, Q, K, V, **options).run()["O"].double().cpu()
    want = ref.attention(*(t.double().numpy() for t in (Q, K, V)), dtype=dtype, **options)["O"][1]
    for first, last in ((699, 700), (650, 661), (300, 400), (0, 1)):
        part = Call(dtype, Q[:, first:last].contiguous(), K[:, :last].contiguous(), V[:, :last].contiguous(), **options).run()["O"].double().cpu()
        off = (part - whole[:, first:last]).abs().numpy()
        assert (off <= 2 * want[:, first:last]).all(), (first, last)


def test_workspace_queries_name_what_each_choice_takes():
    """No split, no workspace; a split of one token's keys takes some."""
    Q, K, V, _ = _problem("bf16", 1, 8, 2, 1, 5000, 128, backward=False)
    call = Call("bf16", Q, K, V, scale=1.0)
    p = L.attention_problem(call.Q, call.K, call.V, call.O, call.L, scale=1.0)
    assert L.lsp_attention_forward_workspace_bytes(p, _CODE["bf16"]) > 0
    Q, K, V = (_normal(1, "bf16", 2, 2048, h, 128) for h in (16, 4, 4))
    call = Call("bf16", Q, K, V, scale=1.0)
    p = L.attention_problem(call.Q, call.K, call.V, call.O, call.L, scale=1.0)
    assert L.lsp_attention_forward_workspace_bytes(p, _CODE["bf16"]) == 0
