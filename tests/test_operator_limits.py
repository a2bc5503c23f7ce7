"""CPU-only: problems at the border of what the training operators' launches hold, and outputs whose rows would share memory; refused before any HIP call."""
import ctypes

import pytest

from test_operator_refusals import FAKE, attention, gradients
import paper_2406_10181_amd as L

THREE = ctypes.c_int64 * 3
BIG = 1 << 40


def _forward(p, dtype=2):
    return L.lsp_attention_forward(p, dtype, FAKE, BIG, None, check=False)


def _backward(p, g, dtype=2):
    return L.lsp_attention_backward(p, g, dtype, FAKE, BIG, None, check=False)


def _tokens(batch, q_len=1, k_len=1, heads=1):
    """Short texts of one head, rows one behind the other."""
    strides = lambda length: THREE(length * heads * 8, heads * 8, 8)
    q, k = strides(q_len), strides(k_len)
    p = attention(batch=batch, heads=heads, kv_heads=heads, q_len=q_len, k_len=k_len, head_dim=8, q_stride=q, k_stride=k, v_stride=k, o_stride=q)
    return p, gradients(do_stride=q, dq_stride=q, dk_stride=k, dv_stride=k)


@pytest.mark.parametrize("dtype", [0, 1, 2])
def test_forward_launches_have_fewer_than_2_to_32_threads(dtype):
    """256 threads for every text and head."""
    for p in (_tokens(1 << 24)[0], _tokens(1 << 23, heads=2)[0], _tokens(1 << 24, 7, 3)[0]):
        assert _forward(p, dtype) == -2
        assert L.lsp_attention_forward_workspace_bytes(p, dtype) == 0


@pytest.mark.parametrize("dtype", [0, 1, 2])
@pytest.mark.parametrize("q_len,k_len", [(1, 1), (15, 1), (1, 15), (15, 15)])
def test_backward_launches_have_fewer_than_2_to_32_threads(dtype, q_len, k_len):
    """Twice as many: workgroups for queries and for keys are of one launch."""
    for batch in (1 << 23, (1 << 23) + 1):
        p, g = _tokens(batch, q_len, k_len)
        assert L.lsp_attention_backward_workspace_bytes(p, dtype) == 0
        assert _backward(p, g, dtype) == -2
    p, g = _tokens((1 << 23) - 1, q_len, k_len)
    assert L.lsp_attention_backward_workspace_bytes(p, dtype) > 0


def test_shared_key_heads_count_once():
    q, k = THREE(32, 32, 8), THREE(8, 8, 8)
    p = attention(batch=3 << 20, heads=4, kv_heads=1, q_len=1, k_len=1, head_dim=8, q_stride=q, k_stride=k, v_stride=k, o_stride=q)
    assert L.lsp_attention_backward_workspace_bytes(p, 2) > 0             # 12 * 2^20 + 3 * 2^20
    p.batch = 1 << 22
    assert L.lsp_attention_backward_workspace_bytes(p, 2) == 0            # 16 * 2^20 + 4 * 2^20


def test_parts_of_the_keys_keep_their_workspace():
    """Few texts, long caches: the limit counts the parts too, and they are few."""
    q, k = THREE(128, 128, 8), THREE(8192 * 8, 8, 8)
    p = attention(batch=4, heads=16, kv_heads=1, q_len=1, k_len=8192, head_dim=8, q_stride=q, k_stride=k, v_stride=k, o_stride=q)
    need = L.lsp_attention_forward_workspace_bytes(p, 2)
    assert need > 0 and L.lsp_attention_forward(p, 2, FAKE, need - 1, None, check=False) == -4


# (strides of batch, position and head; 2 texts of 100 positions, 4 query heads or 2 key heads of 64)
OVERLAPPING = [(1 << 20, 64, 64), (1 << 20, 256, 256), (1 << 20, 64, 128), (64, 256, 64), (1 << 20, 256, 128), (25600 - 64, 256, 64), (1 << 20, 64, 64 * 99), (128, 512, 192)]


@pytest.mark.parametrize("dtype", [0, 1, 2])
@pytest.mark.parametrize("strides", OVERLAPPING)
def test_outputs_whose_rows_share_memory_are_refused(dtype, strides):
    """Different workgroups would write the same place, in any order."""
    shared = THREE(*strides)
    assert _forward(attention(o_stride=shared), dtype) == -2
    assert _backward(attention(), gradients(dq_stride=shared), dtype) == -2
    for name in ("dk_stride", "dv_stride"):
        assert _backward(attention(), gradients(**{name: THREE(1 << 20, 96, 64)}), dtype) == -2


def test_inputs_whose_rows_share_memory_are_not():
    """Broadcast inputs: what is missing is the workspace alone."""
    b = THREE(0, 0, 64)
    p = attention(q_stride=b, k_stride=b, v_stride=b)
    assert L.lsp_attention_backward(p, gradients(do_stride=THREE(0, 0, 0)), 2, None, 0, None, check=False) == -4


@pytest.mark.parametrize("strides", [(25600, 256, 64), (1 << 20, 64, 6400), (64 * 400, 64, 6400), (256, 512, 64), (1 << 20, 1024, 128), (64, 512, 128)])
def test_outputs_of_any_order_of_axes(strides):
    """Heads before positions, positions before texts, rows of a wider matrix: what is missing is the workspace alone."""
    s = THREE(*strides)
    p = attention(o_stride=s)
    assert L.lsp_attention_backward(p, gradients(dq_stride=s), 2, None, 0, None, check=False) == -4


def test_axes_of_one_position_have_any_stride():
    one = THREE(1 << 20, 0, 64)
    p = attention(q_len=1, o_stride=one)
    assert L.lsp_attention_backward(p, gradients(dq_stride=one), 2, None, 0, None, check=False) == -4
