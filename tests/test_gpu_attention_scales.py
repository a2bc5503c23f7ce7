"""Attention with scales at the ends of fp32: every key alike, and the largest that is taken."""
import pytest

import operator_reference as ref
import paper_2406_10181_amd as L
from test_gpu_attention import Call, _against_reference, _check, _problem
from test_operator_refusals import FAKE, attention, gradients


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("scale", [1e-37, 1e-38, 1e-42])
def test_scales_that_leave_no_difference(dtype, scale):
    """Probabilities are 1 / keys, L is the logarithm of their number: in whole tiles, in parts of the keys, and for single tokens."""
    for B, H, Hk, Sq, Sk, D in ((1, 2, 1, 100, 300, 64), (1, 2, 2, 40, 1700, 64), (2, 8, 2, 1, 1500, 128), (1, 2, 2, 3, 20, 32)):
        _against_reference(dtype, B, H, Hk, Sq, Sk, D, backward=Sk < 1000, scale=scale, causal=True)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_largest_scales(dtype):
    """Scores of ordinary size from queries and keys that are nearly nothing."""
    scale = 2.0 ** 127
    Q, K, V, _ = _problem(dtype, 1, 2, 1, 70, 150, 32, backward=False)
    Q, K = (Q.float() * 2.0 ** -64).to(Q.dtype), (K.float() * 2.0 ** -63).to(K.dtype)
    got = Call(dtype, Q, K, V, scale=scale).run()
    f = [t.double().numpy() for t in (Q, K, V)]
    _check(got, ref.attention(*f, dtype=dtype, scale=scale, causal=False), (dtype, scale))


@pytest.mark.parametrize("scale", [2.4e38, 3.4e38])
def test_scales_whose_powers_of_two_are_out_of_range(scale):
    """CPU: the kernels take powers of two, of scale * log2(e)."""
    p = attention(scale=scale)
    assert L.lsp_attention_forward(p, 2, FAKE, 1 << 30, None, check=False) == -10
    assert L.lsp_attention_backward(p, gradients(), 2, FAKE, 1 << 30, None, check=False) == -10
