"""Rotary positions, cross entropy and AdamW on tensors that are parts of others: rows with room between them, vectors that begin inside longer ones, repeated inputs; and sizes around a workgroup's."""
import pytest
import torch

import paper_2406_10181_amd as L
import test_gpu_adamw as adamw
import test_gpu_cross_entropy as loss
import test_gpu_rotary as rotary

pytestmark = pytest.mark.gpu
DTYPE = loss.DTYPE


def inside(t, pad):
    """A tensor of t's shape whose rows have `pad` elements of 7 behind them, and all of it."""
    whole = torch.full((t.shape[0], t.shape[1] + pad), 7.0, dtype=t.dtype, device="cuda")
    return whole[:, : t.shape[1]], whole


# the kernels' ways to store gradients: few rows with second ones, tiles of 32 to 256, dH in parts
SHAPES = [(20, 72, 700, {}), (64, 256, 1000, {}), (333, 1000, 1500, dict(left_out=0.4, smoothing=0.1)), (700, 512, 3001, {}), (1500, 520, 9001, dict(left_out=0.15)), (90, 72, 20011, {})]


@pytest.mark.parametrize("rows,width,vocab,more", SHAPES)
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_gradients_with_room_between_their_rows(dtype, rows, width, vocab, more):
    """The same bits as without, and the room is left as it was."""
    c = loss.Case(dtype, rows, width, vocab, seed=21, **more)
    c.backward()
    c.check()
    want = c.dH, c.dW
    pad = 16 // c.H.element_size()
    (c.dH, all_h), (c.dW, all_w) = inside(want[0], pad), inside(want[1], 3 * pad)
    c.backward()
    assert torch.equal(c.dH, want[0]) and torch.equal(c.dW, want[1])
    assert bool((all_h[:, width:] == 7.0).all()) and bool((all_w[:, width:] == 7.0).all())


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_room_between_rows_over_several_blocks(dtype):
    """dW is added up over blocks: in fp32 in its own rows, in 16 bits beside them."""
    c = loss.Case(dtype, 2900, 8, 200000 if dtype == "f32" else 400000, left_out=0.2, seed=22)
    c.backward()
    want = c.dH, c.dW
    pad = 32 // c.H.element_size()
    (c.dH, all_h), (c.dW, all_w) = inside(want[0], pad), inside(want[1], pad)
    c.backward()
    assert torch.equal(c.dH, want[0]) and torch.equal(c.dW, want[1])
    assert bool((all_h[:, 8:] == 7.0).all()) and bool((all_w[:, 8:] == 7.0).all())


@pytest.mark.parametrize("rows", [30, 3000])
def test_vectors_that_are_pieces_of_longer_ones(rows):
    c = loss.Case("bf16", rows, 64, 500, left_out=0.3, smoothing=0.1, seed=23)
    c.backward()
    want = {k: getattr(c, k).clone() for k in ("losses", "logs", "dH", "dW")}
    whole = {}
    for k, before in (("losses", 4), ("logs", 8), ("weights", 12), ("targets", 2)):     # (16 bytes and multiples)
        t = getattr(c, k)
        whole[k] = torch.full((before + rows + 5,), 7, dtype=t.dtype, device="cuda")
        whole[k][before:before + rows] = t
        setattr(c, k, whole[k][before:before + rows])
    c.losses.fill_(3.0), c.logs.fill_(3.0)
    c.backward()
    assert all(torch.equal(getattr(c, k), want[k]) for k in want)
    for k, before in (("losses", 4), ("logs", 8)):
        assert bool((whole[k][:before] == 7).all()) and bool((whole[k][before + rows:] == 7).all())


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_a_logit_that_is_nan_reaches_all_of_dw(dtype):
    c, want = (loss.Case(dtype, 50, 64, 300, seed=7) for _ in range(2))
    want.backward()
    c.H[20, 5] = float("nan")
    c.backward()
    rest = torch.arange(50, device="cuda") != 20
    assert torch.isnan(c.losses[20]) and torch.isnan(c.dH[20]).all() and torch.isnan(c.dW).all()
    assert torch.equal(c.losses[rest], want.losses[rest]) and torch.equal(c.dH[rest], want.dH[rest])


@pytest.mark.parametrize("states", ["f32", "8bit"])
@pytest.mark.parametrize("dtype,grad,master", [("f32", "f32", False), ("f32", "bf16", True), ("bf16", "f32", True), ("f16", "f16", False)])
def test_tensors_around_a_workgroups_size(states, dtype, grad, master):
    """A workgroup has 4096 elements, and takes whole ones another way."""
    made = [adamw.tensor(n, dtype, grad, states, master, seed=n) for n in (4095, 4096, 4097, 8191, 8192, 8193, 12289)]
    adamw.step_and_check([d for d, _ in made], dtype, states, grad_scale=0.5)
    for d, whole in made:
        for name, x in whole.items():
            assert bool((x[d[name].numel():] == 7).all()), f"{name}: written behind its end"


@pytest.mark.parametrize("norm", ["none", "rms", "layer"])
def test_gradients_over_what_was_normed(norm):
    """dQ on Q and dK on K, row on row."""
    c = rotary.Case("bf16", 2, 50, 4, 2, 96, 64, norm=norm, seed=24)
    want = c.run_backward()
    Q, K = c.Q.clone(), c.K.clone()
    c.Q, c.K = Q, K
    got = c.run_backward(dQ=Q, dK=K)
    assert got["dQ"] is Q and all(torch.equal(want[k], got[k]) for k in want)


def test_repeated_inputs():
    """One head for all, one token for all, one text for all: strides of 0 in what is read."""
    c = rotary.Case("f32", 3, 11, 4, 2, 64, 64, norm="layer", bias=True, seed=25)
    for change in (lambda t: t[:, :, :1].expand_as(t), lambda t: t[:, :1].expand_as(t), lambda t: t[:1].expand_as(t)):
        one, two = (rotary.Case("f32", 3, 11, 4, 2, 64, 64, norm="layer", bias=True, seed=25) for _ in range(2))
        for k in ("Q", "K", "V", "dQr", "dKr"):
            setattr(one, k, change(getattr(c, k)))
            setattr(two, k, change(getattr(c, k)).contiguous())
        for x in (one, two):
            L.lsp_rotary_forward(x.problem(), x.code, torch.cuda.current_stream())
        assert torch.equal(one.Qr, two.Qr) and torch.equal(one.Kr, two.Kr) and torch.equal(one.Vr, two.Vr)
        got, want = one.run_backward(), two.run_backward()
        assert all(torch.equal(got[k], want[k]) for k in want)
