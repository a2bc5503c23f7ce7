"""Rotary positions as far as they go, against angles in exact arithmetic: sines and cosines of any position and frequency have the digits of near ones.

A head of pairs (1, 0) turns into cosines and sines, in fp32 with no norm.  What is left of a quarter of a turn is at most 1/8, rounded to fp32: 2^-28 of a turn, 0.4 EPS of the angle; the sine and the cosine of
it are within 2 units of their last place, 4 EPS relative.  The products with 1 and 0 are exact."""
import math
from fractions import Fraction

import numpy as np
import pytest
import torch

import paper_2406_10181_amd as L
from operator_reference import EPS

pytestmark = pytest.mark.gpu
TWO_PI = 2 * Fraction("3.14159265358979323846264338327950288419716939937510582097494459230781640628620899862803482534211706798214808651328230664709384460955058223172535940812848111745")
FAR = 2 ** 31 - 1
POSITIONS = [0, 1, -1, 7, 1000, 4097, 131071, -131071, 999983, 2 ** 24 + 1, 2 ** 27 - 1, 10 ** 9 + 7, FAR, FAR - 1, -FAR - 1, -FAR, 1 - 10 ** 9]


def cosines_and_sines(positions, frequencies):
    """[tokens][pairs][2] in float64; the whole turns are taken off in exact arithmetic."""
    out = np.zeros((len(positions), len(frequencies), 2))
    for i, p in enumerate(positions):
        for j, f in enumerate(frequencies):
            turns = p * Fraction(float(f)) / TWO_PI
            angle = float((turns - round(turns)) * TWO_PI)
            out[i, j] = math.cos(angle), math.sin(angle)
    return out


@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("base", [1.0, 0.7, 2.0 ** 20, 2.0 ** 40])
def test_angles(base, neighbours):
    n, pairs = len(POSITIONS), 48
    frequencies = (torch.tensor(base, dtype=torch.float64) * 10000.0 ** (-torch.arange(pairs, dtype=torch.float64) / pairs)).float()
    Q = torch.zeros(1, n, 1, 2 * pairs, device="cuda")
    (Q[..., ::2] if neighbours else Q[..., :pairs]).fill_(1.0)
    Qr, Kr = torch.empty_like(Q), torch.empty_like(Q)
    p = L.rotary_problem(Q, Q, Qr, Kr, frequencies=frequencies.cuda(), neighbours=neighbours, positions=torch.tensor([POSITIONS], dtype=torch.int32, device="cuda"))
    L.lsp_rotary_forward(p, 0, torch.cuda.current_stream())
    want = cosines_and_sines(POSITIONS, frequencies.tolist())
    got = Qr[0, :, 0].double().cpu().numpy()
    got = got.reshape(n, pairs, 2) if neighbours else np.stack([got[:, :pairs], got[:, pairs:]], axis=-1)
    off = np.abs(got - want) / (EPS * (0.4 + 4 * np.abs(want)))
    assert off.max() <= 1.0, (off.max(), np.unravel_index(off.argmax(), off.shape))
    assert torch.equal(Qr, Kr)


def test_starts_past_32_bits():
    """A position is starts + i in 64 bits: behind the last place of a cache keys go nowhere, queries turn on."""
    n, pairs = 5, 16
    frequencies = torch.tensor([1.0 / (k + 1) for k in range(pairs)])
    Q = torch.zeros(2, n, 1, 2 * pairs, device="cuda")
    Q[..., :pairs] = 1.0
    Qr, Kr = torch.empty_like(Q), torch.full_like(Q, 7.0)
    p = L.rotary_problem(Q, Q, Qr, Kr, frequencies=frequencies.cuda(), starts=torch.tensor([FAR - 1, -FAR - 1], dtype=torch.int32, device="cuda"))
    L.lsp_rotary_forward(p, 0, torch.cuda.current_stream())
    for b, start in enumerate((FAR - 1, -FAR - 1)):
        want = cosines_and_sines([start + i for i in range(n)], frequencies.tolist())
        got = Qr[b, :, 0].double().cpu().numpy()
        off = np.abs(np.stack([got[:, :pairs], got[:, pairs:]], axis=-1) - want) / (EPS * (0.4 + 4 * np.abs(want)))
        assert off.max() <= 1.0, off.max()
    assert bool((Kr == 7.0).all())


def test_a_gradient_turns_back_by_the_same_angle():
    n, pairs = len(POSITIONS), 16
    frequencies = torch.tensor([0.9 ** k for k in range(pairs)])
    d = torch.zeros(1, n, 1, 2 * pairs, device="cuda")
    d[..., :pairs] = 1.0
    dQ, dK = torch.empty_like(d), torch.empty_like(d)
    p = L.rotary_problem(d, d, torch.empty_like(d), torch.empty_like(d), frequencies=frequencies.cuda(), positions=torch.tensor([POSITIONS], dtype=torch.int32, device="cuda"))
    L.lsp_rotary_backward(p, L.rotary_gradients(d, d, dQ, dK), 0, None, 0, torch.cuda.current_stream())
    want = cosines_and_sines(POSITIONS, frequencies.tolist()) * np.array([1.0, -1.0])
    got = dQ[0, :, 0].double().cpu().numpy()
    off = np.abs(np.stack([got[:, :pairs], got[:, pairs:]], axis=-1) - want) / (EPS * (0.4 + 4 * np.abs(want)))
    assert off.max() <= 1.0, off.max()
