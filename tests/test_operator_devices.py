"""CPU-only: tensors of one call that are on several devices, or on the host, are refused before a kernel follows their addresses."""
import pytest
import torch

import paper_2406_10181_amd as L

FAKE, ROOM = 0x1000, 1 << 40       # aligned, never followed
BF16, F32, I32 = torch.bfloat16, torch.float32, torch.int32


class OnDevice(torch.Tensor):
    """A host tensor that says of itself that it is on device 0."""
    def get_device(self):
        return 0


def on_device(t):
    return t.as_subclass(OnDevice)


def z(*shape, dtype=BF16):
    return torch.zeros(*shape, dtype=dtype)


def attention():
    return L.attention_problem, dict(Q=z(2, 5, 4, 16), K=z(2, 7, 2, 16), V=z(2, 7, 2, 16), O=z(2, 5, 4, 16), L=z(2, 4, 5, dtype=F32), q_lens=z(2, dtype=I32), k_lens=z(2, dtype=I32)), dict(scale=1.0)


def attention_gradients():
    return L.attention_gradients, dict(dO=z(2, 5, 4, 16), dQ=z(2, 5, 4, 16), dK=z(2, 7, 2, 16), dV=z(2, 7, 2, 16)), {}


def norm():
    w = {k: z(16) for k in ("post_weight", "post_bias", "gate", "pre_weight", "pre_bias")}
    return L.residual_norm_problem, dict(x=z(3, 16), f=z(3, 16), y=z(3, 16), h=z(3, 16), stats=z(4, 3, dtype=F32), **w), dict(post="layer", pre="layer")


def norm_gradients():
    w = {k: z(16, dtype=F32) for k in ("post_weight", "post_bias", "gate", "pre_weight", "pre_bias")}
    return L.residual_norm_gradients, dict(dy=z(3, 16), dh=z(3, 16), dx=z(3, 16), df=z(3, 16), **w), {}


def rotary():
    w = {k: z(16) for k in ("q_weight", "k_weight", "q_bias", "k_bias")}
    return L.rotary_problem, dict(Q=z(2, 5, 4, 16), K=z(2, 5, 2, 16), Qr=z(2, 5, 4, 16), Kr=z(2, 9, 2, 16), V=z(2, 5, 2, 16), Vr=z(2, 9, 2, 16), frequencies=z(8, dtype=F32),
                                  positions=z(2, 5, dtype=I32), starts=z(2, dtype=I32), lens=z(2, dtype=I32), **w), dict(norm="rms")


def rotary_gradients():
    return L.rotary_gradients, dict(dQr=z(2, 5, 4, 16), dKr=z(2, 9, 2, 16), dQ=z(2, 5, 4, 16), dK=z(2, 5, 2, 16), **{k: z(16, dtype=F32) for k in ("q_weight", "k_weight", "q_bias", "k_bias")}), {}


def loss():
    return L.cross_entropy_problem, dict(H=z(6, 16), W=z(30, 16), targets=z(6, dtype=torch.int64), losses=z(6, dtype=F32), logs=z(6, dtype=F32)), {}


def loss_gradients():
    return L.cross_entropy_gradients, dict(dH=z(6, 16), dW=z(30, 16), weights=z(6, dtype=F32)), {}


MAKERS = [attention, attention_gradients, norm, norm_gradients, rotary, rotary_gradients, loss, loss_gradients]


def make(maker, device=False, other=()):
    """A descriptor whose tensors are on the device, or on the host, but for those named."""
    function, tensors, more = maker()
    tensors = {k: on_device(t) if device != (k in other) else t for k, t in tensors.items()}
    descriptor = function(**tensors, **more)
    descriptor.kept = tensors                            # (it has addresses only)
    return descriptor


@pytest.mark.parametrize("maker,name", [(m, k) for m in MAKERS for k in m()[1]])
@pytest.mark.parametrize("device", [False, True])
def test_a_descriptor_has_one_device(maker, name, device):
    assert make(maker, device).device == (0 if device else -1)
    with pytest.raises(ValueError):
        make(maker, device, (name,))


BACKWARD = [(attention, attention_gradients, L.lsp_attention_backward), (norm, norm_gradients, L.lsp_residual_norm_backward), (rotary, rotary_gradients, L.lsp_rotary_backward),
            (loss, loss_gradients, L.lsp_cross_entropy_backward)]


@pytest.mark.parametrize("problem,gradients,call", BACKWARD)
def test_gradients_are_where_the_problem_is(problem, gradients, call):
    for device in (False, True):
        with pytest.raises(ValueError):
            call(make(problem, device), make(gradients, not device), 2, FAKE, ROOM, None, check=False)
    assert call(make(problem, True), make(gradients, True), 2, FAKE + 8, ROOM, None, check=False) == -4


@pytest.mark.parametrize("problem,gradients,call", BACKWARD)
def test_a_workspace_is_where_the_problem_is(problem, gradients, call):
    room = torch.empty((1 << 22) + 256, dtype=torch.uint8)
    for ws in (room, room.numpy()):
        with pytest.raises(ValueError):
            call(make(problem, True), make(gradients, True), 2, ws, 1 << 22, None, check=False)
    assert call(make(problem, True), make(gradients, True), 2, on_device(room), 0, None, check=False) == -4


def test_nothing_runs_on_the_host():
    for problem, call in ((attention, L.lsp_attention_forward), (loss, L.lsp_cross_entropy_forward)):
        with pytest.raises(ValueError):
            call(make(problem), 2, FAKE, ROOM, None, check=False)
    for problem, call in ((norm, L.lsp_residual_norm_forward), (rotary, L.lsp_rotary_forward)):
        with pytest.raises(ValueError):
            call(make(problem), 2, None, check=False)
    for problem, gradients, call in BACKWARD:
        with pytest.raises(ValueError):
            call(make(problem), make(gradients), 2, FAKE, ROOM, None, check=False)
        assert call(make(problem), make(gradients), 2, None, 0, None, check=False) == -4        # (what the library refuses, it refuses)
    items = L.adamw_items([dict(param=z(600), grad=z(600), m=z(600, dtype=F32), v=z(600, dtype=F32))])
    with pytest.raises(ValueError):
        L.lsp_adamw(items, rate=1e-3, step=1, check=False)
