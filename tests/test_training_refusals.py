"""CPU-only: what rotary, cross entropy and AdamW refuse, before any HIP call, what their workspace queries say, and which tensors the binding takes for belonging together."""
import ctypes

import pytest
import torch

import paper_2406_10181_amd as L

FAKE = 0x1000            # aligned, never followed: every check here fails before any HIP call
THREE = ctypes.c_int64 * 3
BIG = 1 << 40
NAN, INF = float("nan"), float("inf")
F32, F16, BF16, F64 = torch.float32, torch.float16, torch.bfloat16, torch.float64


def rotary(**change):
    o = dict(Q=FAKE, K=2 * FAKE, V=3 * FAKE, Qr=4 * FAKE, Kr=5 * FAKE, Vr=6 * FAKE, q_weight=FAKE, k_weight=FAKE, q_bias=None, k_bias=None, frequencies=FAKE, positions=None, starts=None, lens=None,
             q_stride=THREE(1 << 20, 256, 64), k_stride=THREE(1 << 20, 128, 64), v_stride=THREE(1 << 20, 128, 64), qr_stride=THREE(1 << 20, 256, 64), kr_stride=THREE(1 << 20, 128, 64),
             vr_stride=THREE(1 << 20, 128, 64), batch=2, length=100, cache=120, heads=4, kv_heads=2, head_dim=64, rotated=64, neighbours=0, norm=1, eps=1e-5)
    o.update(change)
    return L.lsp_rotary_problem(**o)


def rotary_gradients(**change):
    o = dict(dQr=7 * FAKE, dKr=8 * FAKE, dQ=9 * FAKE, dK=10 * FAKE, q_weight=FAKE, k_weight=None, q_bias=None, k_bias=None, dqr_stride=THREE(1 << 20, 256, 64), dkr_stride=THREE(1 << 20, 128, 64),
             dq_stride=THREE(1 << 20, 256, 64), dk_stride=THREE(1 << 20, 128, 64))
    o.update(change)
    return L.lsp_rotary_gradients(**o)


BAD_ROTARY = [
    (dict(Q=None), -1), (dict(K=None), -1), (dict(Qr=None), -1), (dict(Kr=None), -1), (dict(V=None), -1), (dict(Vr=None), -1), (dict(frequencies=None), -1),
    (dict(batch=0), -2), (dict(length=0), -2), (dict(cache=0), -2), (dict(heads=0), -2), (dict(kv_heads=-1), -2), (dict(head_dim=0), -2), (dict(head_dim=60), -2), (dict(head_dim=136), -2),
    (dict(rotated=-8), -2), (dict(rotated=12), -2), (dict(rotated=72), -2), (dict(neighbours=2), -2), (dict(norm=3), -2), (dict(length=1 << 28), -2), (dict(batch=1 << 30), -2),
    (dict(heads=2 ** 31 - 1), -2), (dict(cache=1 << 30), -2),
    (dict(q_stride=THREE(1 << 20, -256, 64)), -2), (dict(k_stride=THREE(1 << 20, 1 << 22, 64)), -2), (dict(qr_stride=THREE(1 << 20, 0, 64)), -2), (dict(kr_stride=THREE(0, 128, 64)), -2),
    (dict(vr_stride=THREE(1 << 20, 128, 8)), -2), (dict(v_stride=THREE(1 << 41, 128, 64)), -2), (dict(k_stride=THREE(1 << 20, 128, 1 << 27)), -2),
    (dict(q_stride=THREE(1 << 20, 256, 60)), -7), (dict(Q=FAKE + 8), -7), (dict(Vr=FAKE + 8), -7), (dict(q_weight=FAKE + 2), -7), (dict(k_bias=FAKE + 8), -7), (dict(frequencies=FAKE + 4), -7),
    (dict(positions=FAKE + 2), -7), (dict(starts=FAKE + 1), -7), (dict(lens=FAKE + 2), -7),
    (dict(eps=-1.0), -10), (dict(eps=NAN), -10), (dict(eps=INF), -10),
    # over its input, but not row on row, or at other places
    (dict(Qr=FAKE, qr_stride=THREE(1 << 20, 512, 64)), -2), (dict(Kr=2 * FAKE, starts=FAKE), -2), (dict(Vr=3 * FAKE, starts=FAKE), -2),
]


@pytest.mark.parametrize("change,code", BAD_ROTARY)
def test_rotary(change, code):
    assert L.lsp_rotary_forward(rotary(**change), 2, None, check=False) == code
    assert L.lsp_rotary_backward(rotary(**change), rotary_gradients(), 2, FAKE, BIG, None, check=False) == code


def test_rotary_types_workspaces_and_gradients():
    p = rotary()
    need = L.lsp_rotary_backward_workspace_bytes(p, 2)
    assert need >= 2 * 64 * 4 and L.lsp_rotary_backward_workspace_bytes(rotary(norm=0), 2) == 0 and L.lsp_rotary_backward_workspace_bytes(rotary(head_dim=12), 2) == 0
    assert L.lsp_rotary_forward(None, 2, None, check=False) == -1 and L.lsp_rotary_forward(p, 3, None, check=False) == -3
    back = lambda g=None, p=p, dtype=2, ws=FAKE, n=need, **c: L.lsp_rotary_backward(p, g or rotary_gradients(**c), dtype, ws, n, None, check=False)
    for name in ("dQr", "dKr", "dQ", "dK"):
        assert back(**{name: None}) == -1 and back(**{name: FAKE * 11 + 8}) == -7
    assert L.lsp_rotary_backward(p, None, 2, FAKE, need, None, check=False) == -1
    assert back(dtype=7) == -3 and back(q_weight=FAKE + 4) == -7
    assert back(ws=None) == -4 and back(n=need - 1) == -4 and back(ws=FAKE + 8) == -4
    assert back(dq_stride=THREE(1 << 20, 0, 64)) == -2 and back(dk_stride=THREE(0, 128, 64)) == -2 and back(dqr_stride=THREE(1 << 20, 1 << 22, 64)) == -2 and back(dkr_stride=THREE(1 << 20, 132, 64)) == -7
    # what was normed is needed as it was; a norm that is none has no weights
    assert back(p=rotary(Qr=FAKE)) == -2 and back(p=rotary(Kr=2 * FAKE)) == -2 and back(p=rotary(norm=0)) == -2
    # over what it is made of, but not row on row, or from other places
    assert back(dQ=7 * FAKE, dq_stride=THREE(1 << 20, 512, 64)) == -2 and back(dQ=FAKE, dq_stride=THREE(1 << 20, 512, 64)) == -2 and back(dK=8 * FAKE, p=rotary(starts=FAKE)) == -2
    assert back(dK=2 * FAKE, dk_stride=THREE(1 << 20, 256, 64)) == -2


def loss(**change):
    o = dict(H=FAKE, W=2 * FAKE, targets=FAKE, losses=FAKE, logs=None, h_stride=64, w_stride=64, rows=100, width=64, vocab=1000, smoothing=0.0, z_loss=0.0)
    o.update(change)
    return L.lsp_cross_entropy_problem(**o)


def loss_gradients(**change):
    o = dict(dH=3 * FAKE, dW=4 * FAKE, weights=None, dh_stride=64, dw_stride=64, scale=1.0)
    o.update(change)
    return L.lsp_cross_entropy_gradients(**o)


BAD_LOSS = [
    (dict(H=None), -1), (dict(W=None), -1), (dict(targets=None), -1), (dict(losses=None), -1),
    (dict(rows=0), -2), (dict(rows=(1 << 22) + 1), -2), (dict(width=0), -2), (dict(width=60), -2), (dict(width=(1 << 16) + 8, h_stride=1 << 17, w_stride=1 << 17), -2), (dict(vocab=0), -2),
    (dict(vocab=(1 << 20) + 1), -2), (dict(h_stride=63), -2), (dict(w_stride=-64), -2), (dict(h_stride=1 << 22), -2),
    (dict(h_stride=68), -7), (dict(w_stride=66), -7), (dict(H=FAKE + 8), -7), (dict(W=FAKE + 2), -7), (dict(targets=FAKE + 8), -7), (dict(losses=FAKE + 4), -7), (dict(logs=FAKE + 4), -7),
    (dict(smoothing=1.0), -10), (dict(smoothing=-0.1), -10), (dict(smoothing=NAN), -10), (dict(z_loss=-1.0), -10), (dict(z_loss=2.0), -10), (dict(z_loss=NAN), -10),
]


@pytest.mark.parametrize("change,code", BAD_LOSS)
def test_cross_entropy(change, code):
    assert L.lsp_cross_entropy_forward(loss(**change), 2, FAKE, BIG, None, check=False) == code
    assert L.lsp_cross_entropy_backward(loss(**change), loss_gradients(), 2, FAKE, BIG, None, check=False) == code


def test_cross_entropy_types_workspaces_and_gradients():
    p = loss()
    f, b = L.lsp_cross_entropy_forward_workspace_bytes(p, 2), L.lsp_cross_entropy_backward_workspace_bytes(p, 2)
    assert 0 < f < b and L.lsp_cross_entropy_forward_workspace_bytes(loss(width=4), 2) == 0 and L.lsp_cross_entropy_backward_workspace_bytes(p, 4) == 0
    for dtype in (-1, 3):
        assert L.lsp_cross_entropy_forward(p, dtype, FAKE, BIG, None, check=False) == -3
    assert L.lsp_cross_entropy_forward(None, 2, FAKE, BIG, None, check=False) == -1
    for ws, n in ((None, f), (FAKE, f - 1), (FAKE + 8, f)):
        assert L.lsp_cross_entropy_forward(p, 2, ws, n, None, check=False) == -4
    back = lambda p=p, ws=FAKE, n=b, **c: L.lsp_cross_entropy_backward(p, loss_gradients(**c), 2, ws, n, None, check=False)
    assert L.lsp_cross_entropy_backward(p, None, 2, FAKE, b, None, check=False) == -1 and back(dH=None, dW=None) == -1
    assert back(ws=None) == -4 and back(n=b - 1) == -4 and back(ws=FAKE + 8) == -4
    assert back(dh_stride=32) == -2 and back(dw_stride=68) == -7 and back(dH=FAKE + 8) == -7 and back(dW=FAKE + 4) == -7 and back(weights=FAKE + 4) == -7
    assert back(scale=NAN) == -10 and back(scale=INF) == -10
    assert back(dH=FAKE) == -2 and back(dW=2 * FAKE) == -2 and back(dH=2 * FAKE) == -2 and back(dW=FAKE) == -2


def test_cross_entropy_workspaces_are_bounded():
    """However many rows there are: exponentials of some rows at a time."""
    at = lambda rows: L.lsp_cross_entropy_backward_workspace_bytes(loss(rows=rows, vocab=128000), 2)
    assert at(1 << 16) < (3 << 30) and at(1 << 20) - at(1 << 16) <= 4 * (1 << 20)
    forward = lambda rows: L.lsp_cross_entropy_forward_workspace_bytes(loss(rows=rows, vocab=128000), 2)
    assert forward(1 << 20) - forward(1 << 16) <= 4 * (1 << 20)


def item(**change):
    o = dict(param=FAKE, grad=FAKE, m=FAKE, v=FAKE, m_scale=FAKE, v_scale=FAKE, master=None, elements=1000, rate_factor=1.0, decay=0.0, dtype=2, grad_dtype=0)
    o.update(change)
    return L.lsp_adamw_item(**o)


def step(items, states="8bit", **change):
    o = dict(rate=1e-3, step=1)
    o.update(change)
    array = (L.lsp_adamw_item * len(items))(*items)
    return L.lsp_adamw(L.AdamwItems(array, states), check=False, **o)


@pytest.mark.parametrize("change,code", [
    (dict(param=None), -1), (dict(grad=None), -1), (dict(m=None), -1), (dict(v=None), -1), (dict(m_scale=None), -1), (dict(v_scale=None), -1), (dict(elements=0), -2), (dict(elements=(1 << 35) + 1), -2),
    (dict(elements=1 << 36), -2), (dict(dtype=3), -3), (dict(grad_dtype=-1), -3), (dict(rate_factor=NAN), -10), (dict(decay=INF), -10), (dict(param=FAKE + 8), -7), (dict(m=FAKE + 4), -7),
    (dict(master=FAKE + 4), -7), (dict(v_scale=FAKE + 2), -7)])
def test_adamw(change, code):
    assert step([item(**change)]) == code and step([item(), item(**change)]) == code


def test_adamw_numbers():
    one = [item()]
    for change, code in ((dict(step=0), -2), (dict(rate=NAN), -10), (dict(rate=INF), -10), (dict(beta1=1.0), -10), (dict(beta2=-0.1), -10), (dict(beta1=NAN), -10), (dict(eps=-1e-8), -10), (dict(eps=INF), -10),
                         (dict(grad_scale=FAKE + 2), -7)):
        assert step(one, **change) == code
    array = (L.lsp_adamw_item * 1)(item())
    call = L.lib().lsp_adamw
    assert call(None, 1, 0, 1e-3, 0.9, 0.999, 1e-8, 1, None, None) == -1 and call(array, 0, 0, 1e-3, 0.9, 0.999, 1e-8, 1, None, None) == -2
    assert call(array, (1 << 16) + 1, 0, 1e-3, 0.9, 0.999, 1e-8, 1, None, None) == -2 and call(array, 1, 2, 1e-3, 0.9, 0.999, 1e-8, 1, None, None) == -2


# ------------------------------------------------------------------ the binding
def _rotary(dtype=BF16, **change):
    q, k = torch.zeros(2, 5, 4, 16, dtype=dtype), torch.zeros(2, 5, 2, 16, dtype=dtype)
    o = dict(Q=q, K=k, Qr=q.clone(), Kr=torch.zeros(2, 9, 2, 16, dtype=dtype), V=k.clone(), Vr=torch.zeros(2, 9, 2, 16, dtype=dtype), frequencies=torch.zeros(8), norm="rms", q_weight=torch.zeros(16, dtype=dtype))
    o.update(change)
    return L.rotary_problem(o.pop("Q"), o.pop("K"), o.pop("Qr"), o.pop("Kr"), **o)


def test_rotary_tensors_that_belong_together():
    p = _rotary()
    assert (p.batch, p.length, p.cache, p.heads, p.kv_heads, p.head_dim, p.rotated) == (2, 5, 9, 4, 2, 16, 16)
    assert _rotary(frequencies=None).rotated == 0
    ok = torch.zeros(2, dtype=torch.int32)
    _rotary(starts=ok, lens=ok, positions=torch.zeros(2, 5, dtype=torch.int32), V=None, Vr=None)
    z = lambda *s, dtype=BF16: torch.zeros(*s, dtype=dtype)
    for change in (dict(Q=z(2, 5, 4, 8)), dict(Qr=z(2, 5, 3, 16)), dict(K=z(2, 4, 2, 16)), dict(Kr=z(2, 9, 3, 16)), dict(Kr=z(1, 9, 2, 16)), dict(V=None), dict(Vr=None), dict(V=z(2, 5, 1, 16)),
                   dict(Vr=z(2, 8, 2, 16)), dict(Q=z(2, 5, 4, 16, dtype=F16)), dict(V=z(2, 5, 2, 16, dtype=F32)), dict(q_weight=z(15)), dict(k_weight=z(16, dtype=F32)), dict(q_bias=z(16, dtype=F64)),
                   dict(frequencies=z(8)), dict(frequencies=z(8, dtype=F64)), dict(starts=torch.zeros(2)), dict(starts=torch.zeros(2, dtype=torch.int64)), dict(lens=torch.zeros(3, dtype=torch.int32)),
                   dict(positions=torch.zeros(2, 4, dtype=torch.int32)), dict(positions=torch.zeros(5, 2, dtype=torch.int32).t()), dict(Q=z(2, 5, 16, 4).transpose(2, 3))):
        with pytest.raises(ValueError):
            _rotary(**change)
    with pytest.raises(KeyError):
        _rotary(norm="batch")


def test_rotary_gradients_that_belong_together():
    z = lambda *s, dtype=BF16: torch.zeros(*s, dtype=dtype)
    good = dict(dQr=z(2, 5, 4, 16), dKr=z(2, 9, 2, 16), dQ=z(2, 5, 4, 16), dK=z(2, 5, 2, 16))
    make = lambda **c: L.rotary_gradients(**{**good, **c})
    back = lambda g, dtype=2: L.lsp_rotary_backward(_rotary(), g, dtype, None, 0, None, check=False)
    assert back(make(q_weight=torch.zeros(16))) == -4
    for change in (dict(dQ=z(2, 5, 3, 16)), dict(dQ=z(2, 5, 4, 16, dtype=F16)), dict(dK=z(2, 5, 2, 16, dtype=F64)), dict(q_weight=z(16)), dict(k_bias=torch.zeros(8))):
        with pytest.raises(ValueError):
            make(**change)
    for change in (dict(dKr=z(2, 5, 2, 16)), dict(dK=z(2, 9, 2, 16)), dict(dQr=z(2, 5, 2, 16), dQ=z(2, 5, 2, 16)), {k: v.float() for k, v in good.items()}):
        with pytest.raises(ValueError):
            back(make(**change))
    with pytest.raises(ValueError):
        back(make(), dtype=0)


def test_cross_entropy_tensors_that_belong_together():
    H, W, t, l = torch.zeros(6, 16, dtype=BF16), torch.zeros(30, 16, dtype=BF16), torch.zeros(6, dtype=torch.int64), torch.zeros(6)
    p = L.cross_entropy_problem(H, W, t, l, logs=l.clone())
    assert (p.rows, p.width, p.vocab) == (6, 16, 30)
    for args, more in (((H, W[:, :8], t, l), {}), ((H, W.float(), t, l), {}), ((H.double(), W.double(), t, l), {}), ((H, W, t.int(), l), {}), ((H, W, t[:5], l), {}), ((H, W, t, l[:5]), {}),
                       ((H, W, t, l.half()), {}), ((H, W, t, l), dict(logs=l[:3])), ((H, W, None, l), {}), ((H, W, t, None), {}), ((H.t().contiguous().t(), W, t, l), {}), ((H, W, t.repeat_interleave(2)[::2], l), {})):
        with pytest.raises(ValueError):
            L.cross_entropy_problem(*args, **more)
    back = lambda g, dtype=2: L.lsp_cross_entropy_backward(p, g, dtype, None, 0, None, check=False)
    assert back(L.cross_entropy_gradients(H.clone(), W.clone(), weights=l)) == -4 and back(L.cross_entropy_gradients(None, W.clone())) == -4
    for args, more in (((None, None), {}), ((H.float(), W), {}), ((H, W), dict(weights=l.half()))):
        with pytest.raises(ValueError):
            L.cross_entropy_gradients(*args, **more)
    for g in (L.cross_entropy_gradients(H[:5], W), L.cross_entropy_gradients(H, W[:29]), L.cross_entropy_gradients(H, W, weights=l[:5]), L.cross_entropy_gradients(H.float(), W.float())):
        with pytest.raises(ValueError):
            back(g)
    with pytest.raises(ValueError):
        back(L.cross_entropy_gradients(H, W), dtype=1)
    with pytest.raises(TypeError):
        L.lsp_cross_entropy_forward(_rotary(), 2, FAKE, BIG, None, check=False)
    with pytest.raises(TypeError):
        L.lsp_rotary_backward(_rotary(), L.cross_entropy_gradients(H, W), 2, FAKE, BIG, None, check=False)


def test_adamw_tensors_that_belong_together():
    t = lambda n=600, dtype=F32: torch.zeros(n, dtype=dtype)
    plain = lambda **c: {**dict(param=t(dtype=BF16), grad=t(), m=t(), v=t()), **c}
    bits = lambda **c: {**plain(m=t(dtype=torch.uint8), v=t(dtype=torch.uint8), m_scale=t(3), v_scale=t(3)), **c}
    assert L.adamw_items([plain(), plain(master=t(), decay=0.1, rate_factor=2.0)]).states == "f32"
    i = L.adamw_items([bits(), bits(param=t(dtype=F16), decay=0.5)])
    assert i.states == "8bit" and i.array[1].dtype == 1 and i.array[0].dtype == 2 and i.array[0].elements == 600 and i.array[1].decay == 0.5 and i.array[0].rate_factor == 1.0
    one, shared = t(), t(1200)
    for bad in ([], [plain(), bits()], [plain(param=t(dtype=F64))], [plain(grad=t(599))], [plain(m=t(dtype=torch.uint8))], [plain(m=t(dtype=BF16), v=t(dtype=BF16))], [bits(m_scale=t(2))],
                [bits(v_scale=None)], [bits(m_scale=t(3, dtype=F16))], [plain(m_scale=t(3))], [plain(master=t(dtype=F16))], [plain(mu=1.0)], [dict(param=t(), grad=t(), m=t())], [plain(param=t(1200)[::2])],
                [plain(m=one, v=one)], [plain(m=one), plain(v=one)], [plain(param=shared[:600], grad=shared[600:], m=shared[300:900])], [plain(param=t(0), grad=t(0), m=t(0), v=t(0))], ["x"]):
        with pytest.raises(ValueError):
            L.adamw_items(bad)
    L.adamw_items([plain(grad=one), plain(grad=one), plain(param=shared[:600], grad=one, m=shared[600:])])
    with pytest.raises(ValueError):
        L.lsp_adamw(i, rate=1e-3, step=1, grad_scale=torch.zeros(2), check=False)
    with pytest.raises(ValueError):
        L.lsp_adamw(i, rate=1e-3, step=1, grad_scale=torch.zeros(1, dtype=F64), check=False)
    with pytest.raises(ValueError):
        L.lsp_adamw(i, rate=1e-3, step=1, grad_scale=torch.zeros(1, device="meta"), check=False)
