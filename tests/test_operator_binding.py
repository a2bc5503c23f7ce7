"""CPU-only: the descriptors of the training operators are made of tensors that belong together; every other call of theirs would write past one of them."""
import pytest
import torch

import paper_2406_10181_amd as L

F32, F16, BF16, F64 = torch.float32, torch.float16, torch.bfloat16, torch.float64


def _attention(dtype=BF16, L_dtype=F32):
    q, k = torch.zeros(2, 5, 4, 16, dtype=dtype), torch.zeros(2, 7, 2, 16, dtype=dtype)
    return L.attention_problem(q, k, k, q, torch.zeros(2, 4, 5, dtype=L_dtype), scale=1.0)


def _gradients(do=BF16, dq=BF16, dk=BF16, dv=BF16):
    t = lambda length, heads, dtype: torch.zeros(2, length, heads, 16, dtype=dtype)
    return L.attention_gradients(t(5, 4, do), t(5, 4, dq), t(7, 2, dk), t(7, 2, dv))


def _norm(dtype=BF16, stats=F32):
    x = torch.zeros(3, 8, dtype=dtype)
    return L.residual_norm_problem(x, x, x.clone(), x.clone(), torch.zeros(4, 3, dtype=stats), post="rms", pre="layer")


def _norm_gradients(dy=BF16, dh=BF16, dx=BF16, df=BF16, **vectors):
    t = lambda dtype: None if dtype is None else torch.zeros(3, 8, dtype=dtype)
    return L.residual_norm_gradients(t(dy), t(dh), t(dx), t(df), **{k: torch.zeros(8, dtype=d) for k, d in vectors.items()})


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_types_that_belong_together(dtype):
    _attention(dtype), _norm(dtype)
    _gradients(dtype, dtype, dtype, dtype)
    _norm_gradients(dtype, dtype, dtype, dtype, post_weight=F32, post_bias=F32, gate=F32, pre_weight=F32, pre_bias=F32)
    _norm_gradients(dtype, None, dtype, dtype)


@pytest.mark.parametrize("other", [F16, BF16, F64, torch.int32])
def test_what_is_kept_in_fp32_is_fp32(other):
    """The kernels store fp32 there, whatever the type of the rest."""
    with pytest.raises(ValueError):
        _attention(L_dtype=other)
    with pytest.raises(ValueError):
        _norm(stats=other)
    for name in ("post_weight", "post_bias", "gate", "pre_weight", "pre_bias"):
        with pytest.raises(ValueError):
            _norm_gradients(**{name: other})


@pytest.mark.parametrize("other", [F32, F16])
def test_gradients_are_of_one_type(other):
    for name in ("do", "dq", "dk", "dv"):
        with pytest.raises(ValueError):
            _gradients(**{name: other})
    for name in ("dy", "dh", "dx", "df"):
        with pytest.raises(ValueError):
            _norm_gradients(**{name: other})


@pytest.mark.parametrize("other", [F64, torch.int16, torch.int32])
def test_types_without_a_kernel(other):
    for make in (lambda: _attention(other), lambda: _norm(other), lambda: _gradients(other, other, other, other), lambda: _norm_gradients(other, other, other, other)):
        with pytest.raises(ValueError):
            make()
