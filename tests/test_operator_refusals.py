"""CPU-only: what the calls of the training operators refuse, before any HIP call, and what their workspace queries say."""
import ctypes

import pytest

import paper_2406_10181_amd as L

FAKE = 0x1000            # aligned, never followed: every check here fails before any HIP call
THREE = ctypes.c_int64 * 3


def attention(**change):
    o = dict(Q=FAKE, K=FAKE, V=FAKE, O=FAKE, L=FAKE, q_lens=None, k_lens=None, q_stride=THREE(1 << 20, 256, 64), k_stride=THREE(1 << 20, 128, 64),
             v_stride=THREE(1 << 20, 128, 64), o_stride=THREE(1 << 20, 256, 64), batch=2, heads=4, kv_heads=2, q_len=100, k_len=100, head_dim=64,
             causal=1, scale=0.125, dropout=0.0, offset=0, seed=0)
    o.update(change)
    return L.lsp_attention_problem(**o)


def gradients(**change):
    o = dict(dO=FAKE, dQ=FAKE, dK=FAKE, dV=FAKE, do_stride=THREE(1 << 20, 256, 64), dq_stride=THREE(1 << 20, 256, 64), dk_stride=THREE(1 << 20, 128, 64),
             dv_stride=THREE(1 << 20, 128, 64))
    o.update(change)
    return L.lsp_attention_gradients(**o)


NAN, INF = float("nan"), float("inf")
BAD_ATTENTION = [
    (dict(Q=None), -1), (dict(K=None), -1), (dict(V=None), -1), (dict(O=None), -1), (dict(L=None), -1),
    (dict(batch=0), -2), (dict(heads=0), -2), (dict(kv_heads=0), -2), (dict(kv_heads=3), -2), (dict(q_len=0), -2), (dict(k_len=-1), -2), (dict(head_dim=0), -2),
    (dict(head_dim=12), -2), (dict(head_dim=136), -2), (dict(causal=2), -2), (dict(q_len=1 << 25), -2), (dict(batch=1 << 23), -2),
    (dict(q_stride=THREE(1 << 20, -256, 64)), -2), (dict(k_stride=THREE(1 << 20, 1 << 22, 64)), -2), (dict(v_stride=THREE(1 << 41, 128, 64)), -2),
    (dict(o_stride=THREE(1 << 20, 0, 64)), -2), (dict(o_stride=THREE(0, 256, 64)), -2), (dict(o_stride=THREE(1 << 20, 256, 8)), -2),
    (dict(q_stride=THREE(1 << 20, 256, 60)), -7), (dict(k_stride=THREE((1 << 20) + 4, 128, 64)), -7), (dict(Q=FAKE + 8), -7), (dict(L=FAKE + 4), -7), (dict(q_lens=FAKE + 2), -7),
    (dict(scale=0.0), -10), (dict(scale=-1.0), -10), (dict(scale=NAN), -10), (dict(scale=INF), -10), (dict(dropout=1.0), -10), (dict(dropout=-0.1), -10), (dict(dropout=NAN), -10),
]


@pytest.mark.parametrize("change,code", BAD_ATTENTION)
def test_attention(change, code):
    big = 1 << 30
    assert L.lsp_attention_forward(attention(**change), 2, FAKE, big, None, check=False) == code
    assert L.lsp_attention_backward(attention(**change), gradients(), 2, FAKE, big, None, check=False) == code


def test_attention_types_workspaces_and_gradients():
    p, big = attention(), 1 << 30
    assert L.lsp_attention_forward(None, 2, FAKE, big, None, check=False) == -1
    assert L.lsp_attention_forward(p, 3, FAKE, big, None, check=False) == -3
    need = L.lsp_attention_backward_workspace_bytes(p, 2)
    assert need >= 2 * 4 * 100 * 4
    back = lambda g, dtype=2, ws=FAKE, n=need: L.lsp_attention_backward(p, g, dtype, ws, n, None, check=False)
    assert back(None) == -1 and back(gradients(dO=None)) == -1 and back(gradients(dQ=None)) == -1 and back(gradients(dK=None)) == -1 and back(gradients(dV=None)) == -1
    assert back(gradients(), dtype=-1) == -3
    assert back(gradients(), ws=None) == -4 and back(gradients(), n=need - 1) == -4 and back(gradients(), ws=FAKE + 4) == -4
    assert back(gradients(dK=FAKE + 8)) == -7 and back(gradients(dv_stride=THREE(1 << 20, 132, 64))) == -7
    assert back(gradients(dk_stride=THREE(1 << 20, 0, 64))) == -2 and back(gradients(dq_stride=THREE(1 << 20, 1 << 23, 64))) == -2
    # a position's stride in fp32 is half as long
    assert L.lsp_attention_forward(attention(k_stride=THREE(1 << 30, 1 << 21, 64)), 0, FAKE, big, None, check=False) == -2


def test_attention_workspace_queries():
    q = lambda dtype=2, **c: L.lsp_attention_forward_workspace_bytes(attention(**c), dtype)
    assert q(q_len=1, k_len=8192) > 0 and q(batch=64, heads=32, kv_heads=32, q_len=1024, k_len=1024) == 0
    assert q(head_dim=12) == 0 and q(dtype=5) == 0 and L.lsp_attention_backward_workspace_bytes(attention(batch=0), 2) == 0
    few = attention(q_len=1, k_len=8192)
    need = L.lsp_attention_forward_workspace_bytes(few, 2)
    assert L.lsp_attention_forward(few, 2, None, need, None, check=False) == -4
    assert L.lsp_attention_forward(few, 2, FAKE, need - 1, None, check=False) == -4
    assert L.lsp_attention_forward(few, 2, FAKE + 8, need, None, check=False) == -4


def norm(**change):
    o = dict(x=FAKE, f=FAKE, y=2 * FAKE, h=FAKE, stats=FAKE, post_weight=FAKE, post_bias=None, gate=None, pre_weight=FAKE, pre_bias=None,
             x_stride=200, f_stride=200, y_stride=200, h_stride=200, rows=10, width=200, post=1, pre=2, eps=1e-5, residual_scale=1.0, branch_scale=1.0,
             dropout=0.0, offset=0, seed=0)
    o.update(change)
    return L.lsp_residual_norm_problem(**o)


def norm_gradients(**change):
    o = dict(dy=FAKE, dh=FAKE, dx=FAKE, df=FAKE, post_weight=FAKE, post_bias=None, gate=None, pre_weight=FAKE, pre_bias=None,
             dy_stride=200, dh_stride=200, dx_stride=200, df_stride=200)
    o.update(change)
    return L.lsp_residual_norm_gradients(**o)


BAD_NORM = [
    (dict(x=None), -1), (dict(f=None), -1), (dict(y=None), -1), (dict(h=None), -1), (dict(stats=None), -1),
    (dict(rows=0), -2), (dict(rows=(1 << 22) + 1), -2), (dict(width=0), -2), (dict(width=8193), -2), (dict(post=3), -2), (dict(pre=-1), -2),
    (dict(x_stride=199), -2), (dict(f_stride=-200), -2), (dict(y_stride=0), -2), (dict(h_stride=1 << 41), -2),
    (dict(x=FAKE + 4), -7), (dict(h=FAKE + 8), -7), (dict(stats=FAKE + 4), -7), (dict(pre_weight=FAKE + 2), -7), (dict(gate=FAKE + 8), -7),
    (dict(eps=-1.0), -10), (dict(eps=NAN), -10), (dict(residual_scale=INF), -10), (dict(branch_scale=NAN), -10), (dict(dropout=1.0), -10),
]


@pytest.mark.parametrize("change,code", BAD_NORM)
def test_residual_norm(change, code):
    assert L.lsp_residual_norm_forward(norm(**change), 2, None, check=False) == code
    assert L.lsp_residual_norm_backward(norm(**change), norm_gradients(), 2, FAKE, 1 << 30, None, check=False) == code


def test_residual_norm_types_workspaces_and_gradients():
    p = norm()
    need = L.lsp_residual_norm_backward_workspace_bytes(p, 2)
    assert need >= 5 * 200 * 4 and L.lsp_residual_norm_backward_workspace_bytes(norm(width=0), 2) == 0
    back = lambda g, p=p, dtype=2, ws=FAKE, n=need: L.lsp_residual_norm_backward(p, g, dtype, ws, n, None, check=False)
    assert L.lsp_residual_norm_forward(None, 2, None, check=False) == -1 and L.lsp_residual_norm_forward(p, 4, None, check=False) == -3
    for name in ("dy", "dh", "dx", "df"):
        assert back(norm_gradients(**{name: None})) == -1
    assert back(norm_gradients(), dtype=9) == -3
    assert back(norm_gradients(dy_stride=100)) == -2 and back(norm_gradients(), p=norm(y=FAKE)) == -2
    assert back(norm_gradients(post_weight=FAKE), p=norm(post=0)) == -2 and back(norm_gradients(pre_weight=FAKE), p=norm(pre=0)) == -2
    assert back(norm_gradients(dx=FAKE + 2)) == -7 and back(norm_gradients(gate=FAKE + 4)) == -7
    assert back(norm_gradients(), ws=None) == -4 and back(norm_gradients(), n=need - 1) == -4 and back(norm_gradients(), ws=FAKE + 8) == -4


def test_dropout():
    d = lambda x=FAKE, y=FAKE, rows=10, width=10, p=0.1, dtype=2: L.lsp_dropout(x, y, rows, width, p, 1, 0, dtype, None, check=False)
    assert d(x=None) == -1 and d(y=None) == -1
    assert d(rows=0) == -2 and d(width=0) == -2 and d(rows=1 << 40) == -2 and d(width=1 << 31) == -2
    assert d(dtype=3) == -3 and d(x=FAKE + 2) == -7 and d(y=FAKE + 8) == -7
    assert d(p=1.0) == -10 and d(p=-0.5) == -10 and d(p=NAN) == -10
    assert "range" in L.lsp_strerror(-10)


def test_binding_refuses_tensors_that_do_not_belong_together():
    import torch
    t = torch.zeros(2, 5, 4, 16)
    Lt = torch.zeros(2, 4, 5)
    L.attention_problem(t, t, t, t, Lt, scale=1.0)
    for args in ((t, t[:, :, :2], t, t, Lt), (t, t, t, t[:, :4], Lt), (t, t, t, t, Lt[:, :3]), (t, t.half(), t, t, Lt), (t.transpose(2, 3), t.transpose(2, 3), t.transpose(2, 3), t.transpose(2, 3), Lt)):
        with pytest.raises(ValueError):
            L.attention_problem(*args, scale=1.0)
    with pytest.raises(ValueError):
        L.attention_problem(t, t, t, t, Lt, scale=1.0, q_lens=torch.zeros(2))
    x, s = torch.zeros(3, 8), torch.zeros(4, 3)
    L.residual_norm_problem(x, x, x, x, s)
    for args in ((x, x[:, :4], x, x, s), (x, x.half(), x, x, s), (x, x, x, x, s[:2]), (x.t(), x.t(), x.t(), x.t(), s)):
        with pytest.raises(ValueError):
            L.residual_norm_problem(*args)
    with pytest.raises(ValueError):
        L.residual_norm_problem(x, x, x, x, s, post="rms", post_weight=torch.zeros(7))
