"""Norms, gated residual and dropout between two blocks, and the backward pass, against the formulas in 64 bits."""
import numpy as np
import pytest
import torch

import operator_reference as ref
import paper_2406_10181_amd as L

pytestmark = pytest.mark.gpu
_TORCH = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_CODE = {"f32": 0, "f16": 1, "bf16": 2}
VECTORS = ("post_weight", "post_bias", "gate", "pre_weight", "pre_bias")
# sums over a row go through 16 terms a thread at most, six steps in a wave and eight waves; a few operations more on each value
C = 64 * ref.EPS


class Problem:
    def __init__(self, dtype, rows, width, post, pre, vectors=VECTORS, dropout=0.0, seed=3, offset=1, backward=True, mean=0.0, a=1.0, b=0.7, eps=1e-5):
        g = torch.Generator().manual_seed(rows * 10007 + width)
        t = _TORCH[dtype]
        self.dtype, self.rows, self.width, self.backward = dtype, rows, width, backward
        self.x, self.f = (torch.randn(rows, width, generator=g) * 2 + mean).to(t).cuda(), (torch.randn(rows, width, generator=g) + mean).to(t).cuda()
        self.v = {k: (torch.randn(width, generator=g) * 0.3 + (1.0 if "weight" in k or k == "gate" else 0.0)).to(t).cuda()
                  if k in vectors and (post != "none" or not k.startswith("post")) and (pre != "none" or not k.startswith("pre")) else None for k in VECTORS}
        self.dy, self.dh = torch.randn(rows, width, generator=g).to(t).cuda(), torch.randn(rows, width, generator=g).to(t).cuda()
        self.options = dict(post=post, pre=pre, eps=eps, residual_scale=a, branch_scale=b, dropout=dropout, seed=seed, offset=offset)
        self.y, self.h, self.dx, self.df = (torch.full_like(self.x, float("nan")) for _ in range(4))
        self.stats = torch.full((4, rows), float("nan"), device="cuda")
        self.grads = {k: None if t is None else torch.full((width,), float("nan"), device="cuda") for k, t in self.v.items()}

    def enqueue(self, stream):
        p = L.residual_norm_problem(self.x, self.f, self.y, self.h, self.stats, **self.v, **self.options)
        L.lsp_residual_norm_forward(p, _CODE[self.dtype], stream)
        if self.backward:
            n = L.lsp_residual_norm_backward_workspace_bytes(p, _CODE[self.dtype])
            if not hasattr(self, "ws"):
                self.ws = torch.full((n // 4 + 64,), 7.0, device="cuda")
            g = L.residual_norm_gradients(self.dy, self.dh, self.dx, self.df, **self.grads)
            L.lsp_residual_norm_backward(p, g, _CODE[self.dtype], self.ws, n, stream)
            self.ws_floats = n // 4

    def run(self):
        self.enqueue(torch.cuda.current_stream())
        torch.cuda.synchronize()
        return self.results()

    def results(self):
        out = {"y": self.y, "h": self.h}
        if self.backward:
            out.update(dx=self.dx, df=self.df, **{k: t for k, t in self.grads.items() if t is not None})
        return {k: t.clone() for k, t in out.items()}

    def check(self):
        got = self.run()
        o = self.options
        n = lambda t: None if t is None else t.double().cpu().numpy()
        keep = ref.keep_matrix(self.rows, self.width, o["seed"], o["offset"], o["dropout"]) if o["dropout"] else 1.0
        v = {k: n(t) for k, t in self.v.items()}
        x, f, dy, dh = n(self.x), n(self.f), n(self.dy), n(self.dh)
        a, b = o["residual_scale"], float(np.float32(o["branch_scale"]))
        w = ref.residual_norm(x, f, post=o["post"], pre=o["pre"], eps=float(np.float32(o["eps"])), a=a, b=b, w_post=v["post_weight"], b_post=v["post_bias"], gate=v["gate"],
                              w_pre=v["pre_weight"], b_pre=v["pre_bias"], keep=keep, dy=dy, dh=dh)
        one = np.ones(self.width)
        wp, wq, gate = (one if v[k] is None else np.abs(v[k]) for k in ("post_weight", "pre_weight", "gate"))
        bp, bq = (0 * one if v[k] is None else np.abs(v[k]) for k in ("post_bias", "pre_bias"))
        b = abs(b)                                                  # (sizes from here on)
        most = lambda t: np.abs(t).max(1, keepdims=True)
        u, tiny = ref.U[self.dtype], ref.TINY[self.dtype]
        # what goes into each value, in size; C of that is fp32's share, u of the value the rounding's
        f_hat = (np.abs(f) + most(f)) / w["f_dev"]
        branch = b * gate * keep * (f_hat * wp + bp)
        y_in = a * np.abs(x) + branch
        y_hat = 2 * (y_in + most(y_in)) / w["y_dev"]
        tol = {"y": C * y_in, "h": C * (y_hat * wq + bq)}
        if self.backward:
            e = np.abs(dh) * wq
            t_in = np.abs(dy) + (e + most(e) + y_hat * (e * y_hat).mean(1, keepdims=True)) / w["y_dev"] if o["pre"] != "none" else np.abs(dy) + e
            du = b * t_in * gate * keep
            e2 = du * wp
            tol["dx"] = C * a * t_in
            tol["df"] = C * ((e2 + most(e2) + f_hat * (e2 * f_hat).mean(1, keepdims=True)) / w["f_dev"] if o["post"] != "none" else du)
            rows = 1 + self.rows / 512                              # terms of a sum over rows that one thread adds, in units of 64
            s = C * rows
            tol.update(pre_weight=s * (np.abs(dh) * y_hat).sum(0), pre_bias=s * np.abs(dh).sum(0), gate=s * (b * t_in * keep * (f_hat * wp + bp)).sum(0),
                       post_weight=s * (du * f_hat).sum(0), post_bias=s * du.sum(0))
        for name, t in got.items():
            r = ref.EPS if name in VECTORS else u
            bound = tol[name] * (1 + r) + r * np.abs(w[name]) + (0 if name in VECTORS else tiny)
            off = np.abs(n(t) - w[name])
            assert np.isfinite(n(t)).all() and (off <= bound).all(), (name, float((off / bound).max()))
        if self.backward:
            assert (self.ws[self.ws_floats:] == 7.0).all()
        return got


KINDS = [("none", "none"), ("none", "rms"), ("none", "layer"), ("rms", "none"), ("rms", "rms"), ("layer", "layer"), ("layer", "rms")]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("post,pre", KINDS)
@pytest.mark.parametrize("dropout", [0.0, 0.2])
def test_kinds(dtype, post, pre, dropout):
    Problem(dtype, 37, 200, post, pre, dropout=dropout).check()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,width", [(1, 1), (2, 7), (1, 8), (3, 9), (5, 511), (5, 512), (6, 513), (9, 1024), (7, 1025), (4, 2048), (5, 2049), (3, 2999), (3, 4096),
                                        (5, 4097), (2, 8191), (3, 8192), (1500, 33), (700, 1100), (530, 4100)])
def test_sizes(dtype, rows, width):
    Problem(dtype, rows, width, "layer", "rms", dropout=0.1).check()
    Problem(dtype, rows, width, "rms", "layer").check()


@pytest.mark.parametrize("vectors", [(), ("post_weight",), ("gate", "pre_bias"), ("post_bias", "pre_weight")])
def test_vectors_that_are_left_out(vectors):
    Problem("bf16", 20, 300, "layer", "layer", vectors=vectors, dropout=0.1).check()
    Problem("f32", 20, 300, "rms", "rms", vectors=vectors).check()


@pytest.mark.parametrize("post,pre", [("layer", "layer"), ("rms", "rms")])
def test_a_large_mean_costs_no_digits_of_the_deviation(post, pre):
    Problem("f32", 16, 1000, post, pre, mean=300.0).check()


def test_scales():
    Problem("f32", 16, 130, "rms", "layer", a=0.5, b=-2.0, eps=0.1).check()
    Problem("bf16", 16, 130, "none", "rms", a=0.0, b=1.0).check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strides_and_in_place(dtype):
    """Rows inside wider ones, at addresses off the 16-byte steps; y over x, dx over dy."""
    plain = Problem(dtype, 21, 333, "layer", "rms", dropout=0.1)
    want = plain.run()
    p = Problem(dtype, 21, 333, "layer", "rms", dropout=0.1)

    def inside(t, fill=True):
        wide = torch.full((21, 333 + 70), 7.0, dtype=t.dtype, device="cuda")
        view = wide[:, :333]
        if fill:
            view.copy_(t)
        return view, wide

    guards = []
    for name in ("x", "f", "dy", "dh"):
        setattr(p, name, inside(getattr(p, name))[0])
    for name in ("y", "h", "df"):
        view, wide = inside(getattr(p, name), False)
        setattr(p, name, view)
        guards.append(wide)
    p.dx = p.dy
    got = p.run()
    for name in want:
        assert torch.equal(want[name], got[name]), name
    assert all((w[:, 333:] == 7.0).all() for w in guards)
    q = Problem(dtype, 21, 333, "layer", "rms", dropout=0.1, backward=False)
    q.y = q.x
    got = q.run()
    assert torch.equal(got["y"], want["y"]) and torch.equal(got["h"], want["h"])


def test_without_a_next_norm():
    """h left out: y alone, and its gradient alone."""
    p = Problem("bf16", 11, 100, "rms", "none", dropout=0.3)
    p.dh.zero_()
    want = p.run()
    q = Problem("bf16", 11, 100, "rms", "none", dropout=0.3)
    q.h = q.dh = None
    q.enqueue(torch.cuda.current_stream())
    torch.cuda.synchronize()
    for name in ("y", "dx", "df", "post_weight", "gate"):
        t = q.grads[name] if name in q.grads else getattr(q, name)
        assert torch.equal(t, want[name]), name


def test_what_is_dropped_may_be_infinite():
    p = Problem("f32", 9, 64, "none", "layer", dropout=0.4)
    want = p.run()
    q = Problem("f32", 9, 64, "none", "layer", dropout=0.4)
    q.f[torch.from_numpy(ref.keep_matrix(9, 64, 3, 1, 0.4) == 0).cuda()] = float("inf")
    got = q.run()
    for name in want:
        assert torch.equal(want[name], got[name]), name


def test_same_bits_again_on_any_stream_and_in_graphs():
    p = Problem("bf16", 999, 1200, "rms", "layer", dropout=0.1)
    first = p.run()
    stream = torch.cuda.Stream()
    for t in p.results():
        (p.grads[t] if t in p.grads else getattr(p, t)).fill_(float("nan"))
    torch.cuda.synchronize()
    p.enqueue(stream)
    stream.synchronize()
    for name, t in p.results().items():
        assert torch.equal(first[name], t), name
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p.enqueue(torch.cuda.current_stream())
    for _ in range(3):
        for t in first:
            (p.grads[t] if t in p.grads else getattr(p, t)).fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        for name, t in p.results().items():
            assert torch.equal(first[name], t), name


def test_gradients_against_differences():
    """The change of <y, dy> + <h, dh> along a direction, by central differences of the forward pass in fp32: steps of 2^-5 leave a third
    derivative of about 2^-10 / 6 and fp32's noise far below; a hundredth of the gradient's norm is the bound."""
    args = ("f32", 12, 96, "layer", "rms")
    p = Problem(*args, dropout=0.2)
    got = p.run()
    step = 2.0 ** -5
    for name in ("x", "f") + VECTORS:
        base = p.v[name] if name in p.v else getattr(p, name)
        u = torch.randn(base.shape, generator=torch.Generator().manual_seed(5)).cuda()
        u /= u.norm()
        sides = []
        for sign in (1.0, -1.0):
            q = Problem(*args, dropout=0.2, backward=False)
            (q.v[name] if name in q.v else getattr(q, name)).add_(sign * step * u)
            r = q.run()
            sides.append(float((r["y"].double() * p.dy.double()).sum() + (r["h"].double() * p.dh.double()).sum()))
        g = got["d" + name if name in ("x", "f") else name].double()
        assert abs((sides[0] - sides[1]) / (2 * step) - float((g * u).sum())) <= 0.01 * float(g.norm()), name
