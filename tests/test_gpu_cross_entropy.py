"""lsp_cross_entropy_forward and lsp_cross_entropy_backward against the definition in 64 bits, through the C ABI."""
import numpy as np
import pytest
import torch

import paper_2406_10181_amd as L
import training_reference as ref

pytestmark = pytest.mark.gpu
DTYPE = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def f64(t):
    return t.double().cpu().numpy()


def room(n):
    return torch.full((n + 256,), 255, dtype=torch.uint8, device="cuda")     # (what lies there is not used: NaN as a float)


class Case:
    def __init__(self, dtype, rows, width, vocab, smoothing=0.0, z_loss=0.0, left_out=0.0, weights=True, scale=1.0, seed=0, reach=1.0, pad=0):
        g = torch.Generator().manual_seed(seed)
        t = DTYPE[dtype]
        self.__dict__.update(dtype=dtype, code=L.DTYPE_CODE[dtype], smoothing=smoothing, z_loss=z_loss, scale=scale)
        W = torch.randn(vocab, width, generator=g) / width ** 0.5
        self.targets = torch.randint(0, vocab, (rows,), generator=g)
        H = (reach * (torch.randn(rows, width, generator=g) + 4 * torch.rand(rows, 1, generator=g) * W[self.targets])).to(t)
        self.targets[torch.rand(rows, generator=g) < left_out] = -100
        self.H, self.W = torch.zeros(rows, width + pad, dtype=t)[:, :width], torch.zeros(vocab, width + pad, dtype=t)[:, :width]
        self.H.copy_(H), self.W.copy_(W.to(t))
        self.weights = (0.5 + torch.rand(rows, generator=g)) / rows if weights else None
        for k in ("H", "W", "targets", "weights"):                           # (strides as they are)
            x = getattr(self, k)
            if x is not None:
                y = torch.empty_strided(x.shape, x.stride(), dtype=x.dtype, device="cuda")
                y.copy_(x)
                setattr(self, k, y)
        new = lambda x: torch.full_like(x, 7.0)
        self.losses, self.logs = (torch.full((rows,), 7.0, device="cuda") for _ in range(2))
        self.dH, self.dW = new(self.H), new(self.W)

    def problem(self):
        return L.cross_entropy_problem(self.H, self.W, self.targets, self.losses, logs=self.logs, smoothing=self.smoothing, z_loss=self.z_loss)

    def forward(self):
        p = self.problem()
        n = L.lsp_cross_entropy_forward_workspace_bytes(p, self.code)
        L.lsp_cross_entropy_forward(p, self.code, room(n), n, torch.cuda.current_stream())

    def backward(self, dH=True, dW=True):
        p = self.problem()
        n = L.lsp_cross_entropy_backward_workspace_bytes(p, self.code)
        ws = room(n)
        L.lsp_cross_entropy_backward(p, L.cross_entropy_gradients(self.dH if dH else None, self.dW if dW else None, weights=self.weights, scale=self.scale), self.code, ws, n,
                                     torch.cuda.current_stream())
        assert bool((ws[n:] == 255).all()), "written behind the workspace"

    def check(self, names=("losses", "logs", "dH", "dW")):
        want = ref.cross_entropy(f64(self.H), f64(self.W), self.targets.cpu().numpy(), smoothing=self.smoothing, z_loss=self.z_loss, weights=None if self.weights is None else f64(self.weights),
                                 scale=self.scale, dtype=self.dtype)
        for k in names:
            value, bound = want[k]
            got = f64(getattr(self, k))
            off = np.abs(got - value)
            assert np.all(off <= bound), f"{k}: {np.nanmax(off / np.maximum(bound, 1e-300)):.2f} times its bound ({np.isnan(got).sum()} NaN)"


SHAPES = [
    # dtype, rows, width, vocab, more
    ("f32", 64, 256, 1000, dict()),
    ("f32", 1, 8, 1, dict()),
    ("bf16", 1, 8, 7, dict(smoothing=0.1)),
    ("f16", 1, 64, 300, dict(z_loss=1e-2)),
    ("bf16", 17, 40, 513, dict(smoothing=0.2, z_loss=1e-3, left_out=0.3)),
    ("f16", 257, 72, 255, dict(left_out=0.5)),
    ("f32", 130, 24, 2049, dict(smoothing=0.1, z_loss=1e-4, left_out=0.2, pad=8)),
    ("bf16", 300, 264, 4099, dict(pad=64)),
    ("f16", 333, 1000, 1500, dict(smoothing=0.1, left_out=0.4, weights=False, scale=1 / 333)),
    ("bf16", 700, 512, 3001, dict(weights=False)),
    ("f32", 515, 136, 700, dict(weights=False, scale=-3.0)),
    ("bf16", 2100, 64, 300, dict(left_out=0.1)),
]


@pytest.mark.parametrize("dtype,rows,width,vocab,more", SHAPES)
def test_losses_and_gradients(dtype, rows, width, vocab, more):
    c = Case(dtype, rows, width, vocab, **more)
    c.forward()
    c.check(("losses", "logs"))
    before = c.losses.clone(), c.logs.clone()
    c.losses.fill_(7.0), c.logs.fill_(7.0)
    c.backward()
    c.check()
    assert torch.equal(before[0], c.losses) and torch.equal(before[1], c.logs)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_the_tiles_of_large_problems(dtype):
    """Products of 256 x 256 tiles and of 128 x 128, ragged on every side."""
    c = Case(dtype, 1500, 520, 9001, left_out=0.15)
    c.backward()
    c.check()
    c = Case(dtype, 520, 2056, 4100)
    c.backward()
    c.check()


@pytest.mark.parametrize("rows,width,vocab,left_out", [(2900, 1032, 12100, 0.2)])
def test_more_tiles_than_compute_units(rows, width, vocab, left_out):
    """Over 256 tiles of 256 x 256, several of every panel ragged."""
    c = Case("bf16", rows, width, vocab, left_out=left_out, seed=12)
    c.backward()
    c.check()


@pytest.mark.parametrize("smoothing,z_loss", [(0.0, 0.0), (0.1, 1e-2)])
def test_gradients_by_differences(smoothing, z_loss):
    """Along directions of H and of W: (f(x + h e) - f(x - h e)) / 2h against the gradient, f = sum of weights * losses of the forward call in fp32."""
    c = Case("f32", 40, 24, 90, smoothing=smoothing, z_loss=z_loss, seed=13)
    h = 2.0 ** -7
    for k in ("H", "W"):
        x = getattr(c, k)
        x.copy_((x * 1024).round() / 1024)                                   # (steps of 2^-7 are exact)
    c.backward()
    g = f64(c.weights)
    for k in ("H", "W"):
        x, got = getattr(c, k), f64(getattr(c, "d" + k))
        for e in (torch.randint(0, 2, x.shape, generator=torch.Generator().manual_seed(14)).float().cuda() * 2 - 1, torch.sign(getattr(c, "d" + k))):
            along = f64(e) @ f64(c.W).T if k == "H" else f64(c.H) @ f64(e).T # z's derivative
            kept, f, off = x.clone(), [], 0.0
            for sign in (1, -1):
                x.copy_(kept + sign * h * e)
                c.forward()
                f.append(float((f64(c.losses) * g).sum()))
                _, bound = ref.cross_entropy(f64(c.H), f64(c.W), c.targets.cpu().numpy(), smoothing=smoothing, z_loss=z_loss)["losses"]
                off += float((bound * np.abs(g)).sum()) / (2 * h)
            x.copy_(kept)
            # What the third derivative leaves: h^2 / 6 of it.  L's is the third central moment of z' under the probabilities, at most R^3 / (6 sqrt 3) for z' within a range R; its second is
            # at most R^2 / 4 and its first A = max |z'|, so that of z_loss L^2 is at most 2 z_loss (3 A R^2 / 4 + (|L| + 2 h A) R^3 / (6 sqrt 3)).
            R, A = np.ptp(along, axis=1), np.abs(along).max(1)
            third = R ** 3 / (6 * 3 ** 0.5)
            third = third + 2 * z_loss * (0.75 * A * R ** 2 + (np.abs(f64(c.logs)) + 2 * h * A) * third)
            right = float((got * f64(e)).sum())
            # (and the gradient's own bound)
            want = ref.cross_entropy(f64(c.H), f64(c.W), c.targets.cpu().numpy(), smoothing=smoothing, z_loss=z_loss, weights=g)["d" + k][1]
            allowed = off + h * h / 6 * float((np.abs(g) * third).sum()) + float((want * np.abs(f64(e))).sum())
            assert abs((f[0] - f[1]) / (2 * h) - right) <= allowed, (k, f, right, allowed)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("rows", [20, 400])
def test_no_rounding_is_seen_beside_the_last_one(dtype, rows):
    """Of equal weights, beside results that are rounded once.  dH: the targets' dz has no rounding, and other probabilities, a few hundredths of it, are off by u each: some percent.  dW of up to
    32 rows too; of more the targets' dz is just below a power of two, where a rounding is off by u / 2 at most, as results are on average by about u / sqrt(6): (1 + (1 / 4 / 3) / (1 / 6)) ** 0.5 = 1.22."""
    c = Case(dtype, rows, 512, 3000, weights=False, scale=1 / rows, seed=15)
    c.backward()
    want = ref.cross_entropy(f64(c.H), f64(c.W), c.targets.cpu().numpy(), scale=1 / rows, dtype=dtype)
    for k, times in (("dH", 1.1), ("dW", 1.1 if rows <= 32 else 1.3)):
        value = torch.from_numpy(want[k][0])
        once = (value.to(DTYPE[dtype]).double() - value).norm()
        assert (torch.from_numpy(f64(getattr(c, k))) - value).norm() <= times * once, k


def test_rows_that_do_not_count_are_not_read():
    c = Case("bf16", 90, 64, 500, seed=2)
    c.targets[::3] = torch.tensor([-1, 500, -2 ** 63, 2 ** 62, 2 ** 32], device="cuda").repeat(6)
    out = c.targets.ge(500) | c.targets.lt(0)
    kept = c.H.clone()
    c.H[out] = float("nan")
    c.weights[out] = float("nan")
    c.backward()
    assert not c.losses[out].any() and not c.logs[out].any() and not c.dH[out].any()
    c.H, c.weights = kept, torch.where(out, 0.0, c.weights)
    c.check()


def test_no_row_counts():
    c = Case("f16", 40, 64, 500, left_out=1.1)
    c.backward()
    assert not c.losses.any() and not c.dH.any() and not c.dW.any()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_wide_logits(dtype):
    """Logits of some hundreds: most probabilities underflow, some rows have one word with all of it."""
    c = Case(dtype, 100, 64, 800, reach=40.0, seed=4)
    c.backward()
    c.check()


def test_one_gradient_alone():
    c = Case("bf16", 200, 128, 900, seed=5)
    c.backward()
    both = c.dH.clone(), c.dW.clone()
    c.dH.fill_(7.0), c.dW.fill_(7.0)
    c.backward(dW=False)
    assert torch.equal(c.dH, both[0]) and bool((c.dW == 7.0).all())
    c.dH.fill_(7.0)
    c.backward(dH=False)
    assert torch.equal(c.dW, both[1]) and bool((c.dH == 7.0).all())


def test_the_same_bits_from_run_to_run():
    c = Case("f16", 600, 256, 5000, left_out=0.2, seed=6)
    c.backward()
    first = [x.clone() for x in (c.losses, c.dH, c.dW)]
    for _ in range(3):
        c.dH.fill_(7.0), c.dW.fill_(7.0)
        c.backward()
        assert all(torch.equal(a, b) for a, b in zip(first, (c.losses, c.dH, c.dW)))


def test_a_word_that_is_nan_stays_in_its_row_and_in_dw():
    c = Case("bf16", 50, 64, 300, seed=7)
    want = Case("bf16", 50, 64, 300, seed=7)
    want.backward()
    c.H[20, 5] = float("nan")
    c.backward()
    rest = torch.arange(50, device="cuda") != 20
    assert torch.isnan(c.losses[20]) and torch.isnan(c.dH[20]).all()
    assert torch.equal(c.losses[rest], want.losses[rest]) and torch.equal(c.dH[rest], want.dH[rest])


def test_a_captured_call_repeats_with_other_rows():
    """The rows that count are found on the device: a replay finds those that count then."""
    c = Case("bf16", 300, 128, 1000, seed=8)
    p = c.problem()
    n = L.lsp_cross_entropy_backward_workspace_bytes(p, c.code)
    ws = room(n)
    g = L.cross_entropy_gradients(c.dH, c.dW, weights=c.weights)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        L.lsp_cross_entropy_backward(p, g, c.code, ws, n, torch.cuda.current_stream())
    for k in range(4):
        gen = torch.Generator().manual_seed(k)
        targets = torch.randint(0, 1000, (300,), generator=gen)
        targets[torch.rand(300, generator=gen) < 0.3 * k] = -100
        c.targets.copy_(targets)
        c.H.copy_(torch.randn(c.H.shape, generator=gen))
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        c.check()


@pytest.mark.parametrize("rows", [1, 24, 32, 33])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_few_rows_and_weights_that_change_between_replays(dtype, rows):
    """Rows with second ones behind them; which count, and the largest weight, is found by each replay; weights of rows that do not count are not used, and one of infinity stays in its row and in dW."""
    c = Case(dtype, rows, 64, 700, seed=16)
    p = c.problem()
    n = L.lsp_cross_entropy_backward_workspace_bytes(p, c.code)
    ws = room(n)
    g = L.cross_entropy_gradients(c.dH, c.dW, weights=c.weights)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        L.lsp_cross_entropy_backward(p, g, c.code, ws, n, torch.cuda.current_stream())
    for k in range(5):
        gen = torch.Generator().manual_seed(k)
        targets = torch.randint(0, 700, (rows,), generator=gen)
        targets[torch.rand(rows, generator=gen) < 0.25 * k] = -1             # (the last time no row counts)
        weights = torch.rand(rows, generator=gen) * 10.0 ** (k - 2)
        c.targets.copy_(targets), c.weights.copy_(weights), c.H.copy_(torch.randn(c.H.shape, generator=gen))
        left_out = c.targets < 0
        c.weights[left_out] = 0.0                                            # (for the oracle)
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        c.check()
        kept = c.dH.clone(), c.dW.clone()
        c.weights[left_out] = float("nan")
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(kept[0], c.dH) and torch.equal(kept[1], c.dW)
        c.weights[left_out] = 0.0
    c.targets.fill_(5)
    c.weights.fill_(1.0)
    graph.replay()
    torch.cuda.synchronize()
    kept = c.dH.clone()
    c.weights[0] = float("inf")
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(kept[1:], c.dH[1:]) and not torch.isfinite(c.dH[0]).any()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_blocks_of_rows(dtype):
    """More rows than one block of exponentials holds: dW is a sum over blocks."""
    vocab = 200000 if dtype == "f32" else 400000                            # 1 GiB is 1280 rows of these
    c = Case(dtype, 2900, 8, vocab, left_out=0.2, seed=9)
    c.backward()
    H, W, t, g = c.H.double(), c.W.double(), c.targets, c.weights.double()
    rows = ((t >= 0) & (t < vocab)).nonzero().squeeze(1)
    dH, dW, losses = torch.zeros_like(H), torch.zeros_like(W), torch.zeros(2900, dtype=torch.float64, device="cuda")
    for some in rows.split(256):
        z = H[some].mm(W.t().contiguous())
        lse = torch.logsumexp(z, 1)
        losses[some] = lse - z[torch.arange(len(some)), t[some]]
        d = torch.exp(z - lse[:, None])
        d[torch.arange(len(some)), t[some]] -= 1.0
        d *= g[some, None]
        dH[some] = d.mm(W)
        dW += d.t().contiguous().mm(H[some])
    # norms of the errors: fp32 sums of this many terms of random signs; 16 bits: two roundings of every probability (one of them of all), then the result's
    u = ref.U[dtype]
    for got, want in ((c.losses, losses), (c.dH, dH), (c.dW, dW)):
        rel = float((got.double() - want).norm() / want.norm())
        assert rel <= (2e-5 if dtype == "f32" or got is c.losses else 3 * u), rel


@pytest.mark.parametrize("scale", [1e-30, 1e-12, 1.0, 2e4, 1e30])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_scales_of_the_loss(dtype, scale):
    """Of a scaled loss, or a mean over many tokens: gradients of z keep their digits, whatever fp16's range."""
    c = Case(dtype, 70, 64, 300, weights=False, scale=scale, seed=11)
    c.backward()
    want = ref.cross_entropy(f64(c.H), f64(c.W), c.targets.cpu().numpy(), scale=scale, dtype=dtype)
    for k in ("dH", "dW"):
        value, bound = want[k]
        largest = 65504.0 if dtype == "f16" else 3.38e38
        inside = np.abs(value) + bound < largest
        off = np.abs(f64(getattr(c, k)) - value)
        assert np.all(off[inside] <= bound[inside]), (k, np.max(off[inside] / bound[inside]))
        assert np.all(np.isinf(f64(getattr(c, k))[np.abs(value) - bound > largest * 1.001]))
