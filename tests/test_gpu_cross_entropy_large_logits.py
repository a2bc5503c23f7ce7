"""Cross entropy of logits of 1e2 to 3e7, each exactly a number in fp32, against the definition in 64 bits: what the kernels may be off does not grow with the logits.

A logit is one product that all words share and one that tells them apart, and zeros; so z, its differences and a row's maximum have no error.  With t the maximum, s the sum of exp(z - t) and
d = z - t (|d| <= 32), all in fp32: exp(d) is off by EPS (4 |d| + 16), relative (the product with log2(e), the constant, the sum with 15 in 16 bits, which is up to 5.6 EPS near the top, the
exponential); s by that and V / 16 + 64 roundings of its additions; p = exp(d) / s by the sum of both and four more.  A target's p - 1 is expm1(hit - t - log s), off by p times what the exponent is
off, the exponential's own EPS times |p - 1|, and four roundings."""
import numpy as np
import pytest
import torch

import paper_2406_10181_amd as L
from operator_reference import EPS, TINY, U

pytestmark = pytest.mark.gpu
DTYPE = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
# (H's and W's share of what all words have, the step between words); every sum of them is a multiple of fp32's last place there
LARGE = {"1e2": (1.0, 96.0, 0.125), "1e4": (1.0, 9984.0, 0.125), "-1e4": (-1.0, 9984.0, 0.125), "1e6": (16.0, 57344.0, 0.25), "3e7": (512.0, 57344.0, 2.0), "-3e7": (-512.0, 57344.0, 2.0)}


@pytest.mark.parametrize("one_word", [False, True])
@pytest.mark.parametrize("size", LARGE)
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,vocab", [(20, 300), (130, 9001), (300, 2500)])
def test_gradients_do_not_depend_on_how_large_logits_are(dtype, rows, vocab, size, one_word):
    h0, w0, step = LARGE[size]
    g = np.random.default_rng(rows)
    H, W = np.zeros((rows, 16)), np.zeros((vocab, 16))
    H[:, 0], H[:, 1], W[:, 0] = h0, 1.0, w0
    W[:, 1] = step * g.integers(-int(16 / step), 1, vocab)                   # differences of at most 16
    if one_word:                                                             # one has all of the probability, at both ends of the vocabulary's tiles
        W[:, 1], W[vocab - 1, 1] = -16.0, 16.0
        H[:, 1] = np.where(np.arange(rows) % 2, 1.0, -1.0)                   # (and of odd rows the others share it)
    targets = g.integers(0, vocab, rows)
    targets[::3] = vocab - 1
    weights = (0.5 + g.random(rows)).astype(np.float32)
    z = H @ W.T
    t = z.max(1, keepdims=True)
    d = z - t
    assert np.array_equal(z, z.astype(np.float32)) and d.min() >= -32.0
    s = np.exp(d).sum(1, keepdims=True)
    p = np.exp(d) / s
    at, u, one = np.arange(rows), U[dtype], np.zeros_like(z)
    one[at, targets] = 1.0
    es = EPS * (vocab / 16 + 64) + (EPS * (4 * np.abs(d) + 16) * p).sum(1, keepdims=True)           # of s, relative
    ep = p * (EPS * (4 * np.abs(d) + 20) + es)
    less = np.where(one > 0, np.expm1(d - np.log(s)), p)                     # dz before the weights
    # a target's: the exponent is hit - t - log s
    e_target = p * (es + 4 * EPS * (np.log(s) + np.abs(d))) + 4 * EPS * np.abs(less)
    dz = less * weights[:, None]
    edz = np.where(one > 0, e_target, ep + u * p) * weights[:, None] + (u + 4 * EPS) * np.abs(dz)
    if dtype != "f32":
        edz += 2.0 ** -39 * weights[:, None]                                 # below the smallest exponential of a piece
    if dtype == "f16":
        edz += 2.0 ** -37 * 2 * weights.max()                                # and the smallest gradient
    loss, logs = (np.log(s) - d[at, targets][:, None])[:, 0], (t + np.log(s))[:, 0]
    want = {"losses": (loss, es[:, 0] + 4 * EPS * (np.abs(loss) + np.log(s[:, 0]) + np.abs(d[at, targets]))), "logs": (logs, es[:, 0] + 4 * EPS * (np.abs(logs) + np.log(s[:, 0])))}
    for k, value, off in (("dH", dz @ W, edz @ np.abs(W) + EPS * (vocab + 4) * (np.abs(dz) @ np.abs(W))), ("dW", dz.T @ H, edz.T @ np.abs(H) + EPS * (rows + 4) * (np.abs(dz).T @ np.abs(H)))):
        want[k] = (value, off * (1 + u) + u * np.abs(value) + TINY[dtype])

    code, new = L.DTYPE_CODE[dtype], lambda x: torch.from_numpy(x).to(DTYPE[dtype]).cuda()
    tensors = dict(H=new(H), W=new(W), targets=torch.from_numpy(targets).cuda(), weights=torch.from_numpy(weights).cuda(), losses=torch.empty(rows, device="cuda"), logs=torch.empty(rows, device="cuda"))
    assert np.array_equal(tensors["W"].double().cpu().numpy(), W) and np.array_equal(tensors["H"].double().cpu().numpy(), H)
    tensors.update(dH=torch.empty_like(tensors["H"]), dW=torch.empty_like(tensors["W"]))
    problem = L.cross_entropy_problem(*(tensors[k] for k in ("H", "W", "targets", "losses")), logs=tensors["logs"])
    n = L.lsp_cross_entropy_backward_workspace_bytes(problem, code)
    L.lsp_cross_entropy_backward(problem, L.cross_entropy_gradients(tensors["dH"], tensors["dW"], weights=tensors["weights"]), code, torch.empty(n, dtype=torch.uint8, device="cuda"), n,
                                 torch.cuda.current_stream())
    for k, (value, bound) in want.items():
        off = np.abs(tensors[k].double().cpu().numpy() - value)
        assert np.all(off <= bound), f"{k}: {np.nanmax(off / bound):.2f} times its bound"
