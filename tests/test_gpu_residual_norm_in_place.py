"""Residual norm whose outputs lie on its inputs: the bits of separate buffers, whatever lies on what, and refusals of the rest."""
import pytest
import torch

import operator_reference as ref
from test_gpu_residual_norm import Problem
from test_operator_refusals import FAKE, norm, norm_gradients
import paper_2406_10181_amd as L

KINDS = [("none", "none"), ("rms", "none"), ("none", "layer"), ("layer", "rms")]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("post,pre", KINDS)
@pytest.mark.parametrize("width", [5, 100, 515, 1029, 2050, 2999, 4101])
@pytest.mark.parametrize("y,h", [("f", "h"), ("y", "x"), ("y", "f"), ("x", "f"), ("f", "x")])
def test_forward(dtype, post, pre, width, y, h):
    want = Problem(dtype, 300, width, post, pre, dropout=0.2, backward=False).run()
    p = Problem(dtype, 300, width, post, pre, dropout=0.2, backward=False)
    p.y, p.h = getattr(p, y), getattr(p, h)
    got = p.run()
    assert torch.equal(got["y"], want["y"]) and torch.equal(got["h"], want["h"])


@pytest.mark.gpu
@pytest.mark.parametrize("width", [100, 2999])
def test_all_in_one_buffer(width):
    """x, f and y the same, as a norm alone has them; y and h the same: h stays."""
    p = Problem("bf16", 40, width, "none", "rms", b=0.0, backward=False)
    want = p.run()
    x = p.x.clone()
    p.f = p.y = p.x
    got = p.run()
    assert torch.equal(got["h"], want["h"]) and torch.equal(got["y"], x)
    q = Problem("bf16", 40, width, "none", "rms", b=0.0, backward=False)
    q.y = q.h
    assert torch.equal(q.run()["h"], want["h"])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("post,pre", KINDS)
@pytest.mark.parametrize("width", [5, 100, 515, 1029, 2050, 2999, 4101])
@pytest.mark.parametrize("dx,df", [("dy", "dh"), ("dh", "dy"), ("x", "f"), ("f", "x"), ("dx", "f")])
def test_backward(dtype, post, pre, width, dx, df):
    p = Problem(dtype, 600, width, post, pre, dropout=0.2)
    want = p.run()
    grads = {k: None if t is None else t.clone() for k, t in p.grads.items()}
    p.backward = False
    p.run()                                                         # (y, h and the statistics stay: x and f are about to go)
    p.backward = True
    p.dx, p.df = getattr(p, dx), getattr(p, df)
    got = p.run()
    assert torch.equal(got["dx"], want["dx"]) and torch.equal(got["df"], want["df"])
    assert all(t is None or torch.equal(t, grads[k]) for k, t in p.grads.items())


@pytest.mark.gpu
@pytest.mark.parametrize("width", [100, 515, 1029, 2999, 4101])
def test_what_overflows_stays_in_its_column(width):
    """A gradient that fp16 cannot hold is stored over the branch's input as an infinity, beside columns that another thread of the row reads."""
    for at in (width - 2, width - 9, 0):
        results = []
        for in_place in (False, True):
            p = Problem("f16", 50, width, "none", "rms", vectors=("gate",), b=1.0)
            p.dy[:, at] = 60000.0
            p.v["gate"][at] = 4.0
            if in_place:
                p.df = p.f
            results.append(p.run())
        want, got = results
        assert torch.isinf(want["df"][:, at]).all() and torch.isfinite(want["dx"]).all()
        for name in want:
            assert torch.equal(want[name], got[name]), (at, name)


STEP = dict(x=FAKE, f=3 * FAKE, y=5 * FAKE, h=7 * FAKE)


def test_refusals():
    """CPU: one buffer with two row strides, and gradients of a problem whose inputs are gone."""
    forward = lambda **c: L.lsp_residual_norm_forward(norm(**{**STEP, **c}), 2, None, check=False)
    for out in ("y", "h"):
        for on in ("x", "f"):
            assert forward(**{out: STEP[on], out + "_stride": 208}) == -2
            assert forward(**{out: STEP[on], on + "_stride": 208}) == -2
    assert forward(y=STEP["h"], y_stride=208) == -2
    grads = dict(dy=9 * FAKE, dh=11 * FAKE, dx=13 * FAKE, df=15 * FAKE)
    for out in ("y", "h"):
        for on in ("x", "f"):
            assert L.lsp_residual_norm_backward(norm(**{**STEP, out: STEP[on]}), norm_gradients(**grads), 2, FAKE, 1 << 30, None, check=False) == -2
    back = lambda g={}, **c: L.lsp_residual_norm_backward(norm(**{**STEP, **c}), norm_gradients(**{**grads, **g}), 2, None, 0, None, check=False)
    assert back() == -4                                             # (what is missing is the workspace alone)
    for out in ("dx", "df"):
        for on in ("dy", "dh"):
            assert back({out: grads[on]}) == -4 and back({out: grads[on], out + "_stride": 208}) == -2
        for on in ("x", "f"):
            assert back({out: STEP[on]}) == -4 and back({out: STEP[on], out + "_stride": 208}) == -2
    assert back(dict(dx=grads["df"])) == -4 and back(dict(dx=grads["df"], dx_stride=208)) == -2
    one = dict(rows=1)
    assert back(dict(dx=grads["dy"], dx_stride=208), **one) == -4
