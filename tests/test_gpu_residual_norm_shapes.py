"""Residual norm where the kernels' shapes change: the ends of rows, wide rows with every sum, rows of no norm in place, rows by the thousand."""
import pytest
import torch

import operator_reference as ref
from test_gpu_residual_norm import Problem

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,width", [(9, 4104), (300, 4099), (513, 5001), (5, 8185), (270, 7552)])
def test_wide_rows_with_all_vectors(dtype, rows, width):
    """Two units a thread: weights and the biases' sums are not in registers."""
    Problem(dtype, rows, width, "layer", "layer", dropout=0.25).check()
    Problem(dtype, rows, width, "none", "layer").check()
    Problem(dtype, rows, width, "rms", "rms", vectors=("gate", "pre_weight"), dropout=0.1).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("width", [2, 8, 10, 511, 513, 519, 1023, 1025, 1543, 2047, 2051, 3079, 4095])
def test_ends_of_rows(dtype, width):
    """The last columns of a row, a thread's own or shared with its neighbour's, in every shape of a workgroup."""
    Problem(dtype, 1030, width, "rms", "layer", dropout=0.1).check()
    Problem(dtype, 3, width, "layer", "none").check()


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("post,pre", [("none", "none"), ("none", "rms"), ("rms", "none"), ("layer", "layer")])
@pytest.mark.parametrize("width", [5, 100, 515, 1029, 2050, 4093, 4101])
def test_in_place_at_odd_widths(dtype, post, pre, width):
    """y over x and dx over dy give the bits of separate buffers, also where no sum makes the threads of a row wait for one another."""
    p = Problem(dtype, 600, width, post, pre, dropout=0.2)
    want = p.run()
    grads = {k: None if t is None else t.clone() for k, t in p.grads.items()}
    p.dx = p.dy
    got = p.run()
    assert torch.equal(got["dx"], want["dx"]) and torch.equal(got["df"], want["df"])
    assert all(t is None or torch.equal(t, grads[k]) for k, t in p.grads.items())
    p.backward, p.y = False, p.x
    got = p.run()
    assert torch.equal(got["y"], want["y"]) and torch.equal(got["h"], want["h"])


@pytest.mark.parametrize("rows,width", [(20000, 40), (9000, 130), (5000, 520), (4097, 1032)])
def test_many_rows(rows, width):
    """Hundreds of rows a workgroup, and their parts added up."""
    Problem("bf16", rows, width, "none", "layer", dropout=0.1).check()
    Problem("f32", rows, width, "rms", "rms").check()


@pytest.mark.parametrize("width", [5, 100, 515, 1029, 4101])
def test_what_is_dropped_may_be_infinite_at_the_ends_of_rows(width):
    """Also where a thread reads columns that are its neighbour's."""
    want = Problem("f16", 40, width, "none", "layer", dropout=0.4).run()
    p = Problem("f16", 40, width, "none", "layer", dropout=0.4)
    p.f[torch.from_numpy(ref.keep_matrix(40, width, 3, 1, 0.4) == 0).cuda()] = float("-inf")
    got = p.run()
    for name in want:
        assert torch.equal(want[name], got[name]), name
