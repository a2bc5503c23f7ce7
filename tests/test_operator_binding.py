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


CODE = {F32: 0, F16: 1, BF16: 2}
FAKE, ROOM = 0x1000, 1 << 30                 # never followed: these calls fail before any HIP call


def _attention_back(problem, gradients, dtype=2):
    return L.lsp_attention_backward(problem, gradients, dtype, FAKE, ROOM, None, check=False)


def _norm_back(problem, gradients, dtype=2):
    return L.lsp_residual_norm_backward(problem, gradients, dtype, FAKE, ROOM, None, check=False)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_the_calls_type_is_the_tensors(dtype):
    p, n = _attention(dtype), _norm(dtype)
    for code in {0, 1, 2, 3} - {CODE[dtype]}:
        with pytest.raises(ValueError):
            L.lsp_attention_forward(p, code, FAKE, ROOM, None, check=False)
        with pytest.raises(ValueError):
            _attention_back(p, _gradients(dtype, dtype, dtype, dtype), code)
        with pytest.raises(ValueError):
            L.lsp_residual_norm_forward(n, code, None, check=False)
        with pytest.raises(ValueError):
            _norm_back(n, _norm_gradients(dtype, dtype, dtype, dtype), code)


@pytest.mark.parametrize("other", [F32, F16])
def test_gradients_are_of_the_problems_type(other):
    with pytest.raises(ValueError):
        _attention_back(_attention(BF16), _gradients(other, other, other, other))
    with pytest.raises(ValueError):
        _norm_back(_norm(BF16), _norm_gradients(other, other, other, other))


@pytest.mark.parametrize("q,k", [((2, 4, 4, 16), (2, 7, 2, 16)), ((2, 5, 4, 16), (2, 6, 2, 16)), ((1, 5, 4, 16), (1, 7, 2, 16)), ((2, 5, 2, 16), (2, 7, 2, 16)), ((2, 5, 4, 16), (2, 7, 1, 16)),
                                 ((2, 5, 4, 8), (2, 7, 2, 8)), ((2, 5, 4, 24), (2, 7, 2, 24)), ((2, 5, 4, 16), (1, 7, 2, 16))])
def test_gradients_have_the_problems_shapes(q, k):
    a, b = torch.zeros(q, dtype=BF16), torch.zeros(k, dtype=BF16)
    with pytest.raises(ValueError):
        _attention_back(_attention(), L.attention_gradients(a, a, b, b))


@pytest.mark.parametrize("shape", [(2, 8), (4, 8), (3, 7), (3, 16)])
def test_norm_gradients_have_the_problems_shape(shape):
    t = torch.zeros(shape, dtype=BF16)
    with pytest.raises(ValueError):
        _norm_back(_norm(), L.residual_norm_gradients(t, t, t, t))


def test_descriptors_of_another_kind():
    a, g, n, m = _attention(), _gradients(), _norm(), _norm_gradients()
    for call in (lambda: L.lsp_attention_forward(n, 2, FAKE, ROOM, None, check=False), lambda: L.lsp_residual_norm_forward(a, 2, None, check=False),
                 lambda: _attention_back(a, m), lambda: _attention_back(g, g), lambda: _norm_back(n, g), lambda: _norm_back(m, m)):
        with pytest.raises(TypeError):
            call()


def test_descriptors_keep_what_they_were_made_of():
    """Fields may be changed between calls (offsets are); what is compared is what the structure says then."""
    p = _attention()
    p.offset = 7
    p.k_len = 6
    with pytest.raises(ValueError):
        _attention_back(p, _gradients())


def test_lengths_are_where_the_other_tensors_are():
    """Lists of lengths begin on the host; the kernels would follow the address there."""
    q, logs = torch.zeros(2, 5, 4, 16), torch.zeros(2, 4, 5)

    class Elsewhere:
        """Lengths that say of themselves that they are on device 0."""
        def __init__(self):
            self.t = torch.ones(2, dtype=torch.int32)

        def __getattr__(self, name):
            return getattr(self.t, name)

        def get_device(self):
            return 0

    ok = torch.ones(2, dtype=torch.int32)
    L.attention_problem(q, q, q, q, logs, scale=1.0, q_lens=ok, k_lens=ok)
    for lens in (dict(q_lens=Elsewhere()), dict(k_lens=Elsewhere()), dict(q_lens=ok, k_lens=Elsewhere())):
        with pytest.raises(ValueError):
            L.attention_problem(q, q, q, q, logs, scale=1.0, **lens)


def test_sizes_beyond_32_bits_are_refused():
    """Views that repeat one position 2^32 + 2 times: not two positions."""
    q, k, logs = torch.zeros(1, 2, 1, 16), torch.zeros(1, 1, 1, 16).expand(1, (1 << 32) + 2, 1, 16), torch.zeros(1, 1, 2)
    p = L.attention_problem(q, k, k, q, logs, scale=1.0)
    assert L.lsp_attention_forward(p, 0, FAKE, ROOM, None, check=False) == -2
