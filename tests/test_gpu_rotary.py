"""lsp_rotary_forward and lsp_rotary_backward against the definition in 64 bits, through the C ABI."""
import numpy as np
import pytest
import torch

import paper_2406_10181_amd as L
import training_reference as ref

pytestmark = pytest.mark.gpu
DTYPE = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def f64(t):
    return t.double().cpu().numpy()


def check(got, want, what):
    value, bound = want
    off = np.abs(f64(got) - value)
    assert np.all(off <= bound), f"{what}: {np.max(off / bound):.2f} times its bound, at {np.unravel_index(np.argmax(off / bound), off.shape)}"


class Case:
    def __init__(self, dtype, batch, length, heads, kv_heads, dim, rotated, norm="rms", neighbours=False, bias=False, cache=0, positions=None, starts=None, lens=None, weights=True, seed=0):
        g = torch.Generator().manual_seed(seed)
        t = DTYPE[dtype]
        normal = lambda *s: torch.randn(*s, generator=g)
        self.__dict__.update(dtype=dtype, batch=batch, length=length, cache=cache or length, norm=norm, neighbours=neighbours, code=L.DTYPE_CODE[dtype], eps=1e-5)
        joint = (normal(batch, length, heads + 2 * kv_heads, dim) * 2 + 0.3).to(t).cuda()
        self.Q, self.K, self.V = joint.split([heads, kv_heads, kv_heads], dim=2)
        self.Qr = torch.full((batch, length, heads, dim), 7.0, dtype=t, device="cuda")
        self.Kr, self.Vr = (torch.full((batch, self.cache, kv_heads, dim), 7.0, dtype=t, device="cuda") for _ in range(2))
        self.frequencies = (100.0 ** (-torch.arange(rotated // 2) / max(1, rotated // 2))).float().cuda()
        self.positions, self.starts, self.lens = (None if x is None else torch.tensor(x, dtype=torch.int32) for x in (positions, starts, lens))
        self.vectors = {k: None for k in ("q_weight", "k_weight", "q_bias", "k_bias")}
        if weights:
            self.vectors = {k: (1 + 0.2 * normal(dim) if k.endswith("weight") else 0.3 * normal(dim)).to(t).cuda() if k.endswith("weight") or bias else None for k in self.vectors}
        self.dQr, self.dKr = normal(*self.Qr.shape).to(t).cuda(), normal(*self.Kr.shape).to(t).cuda()

    def numbers(self):
        cuda = lambda x: None if x is None else x.cuda()
        return dict(frequencies=self.frequencies if len(self.frequencies) else None, neighbours=self.neighbours, positions=cuda(self.positions), starts=cuda(self.starts), lens=cuda(self.lens),
                    norm=self.norm, eps=self.eps, **self.vectors)

    def problem(self, values=True, **change):
        more = dict(V=self.V, Vr=self.Vr) if values else {}
        self.kept = dict(self.numbers(), **more)
        return L.rotary_problem(*(change.get(k, getattr(self, k)) for k in ("Q", "K", "Qr", "Kr")), **self.kept)

    def want(self, which, d=None, there=None):
        counts, position, place = ref.tokens(self.batch, self.length, *(None if x is None else x.numpy() for x in (self.positions, self.starts, self.lens)))
        angle = position[..., None].astype(float) * f64(self.frequencies)
        vector = lambda k: None if self.vectors[k] is None else f64(self.vectors[k])
        return ref.rotary(f64(getattr(self, which.upper())), angle, neighbours=self.neighbours, norm=self.norm, eps=self.eps, weight=vector(which + "_weight"), bias=vector(which + "_bias"),
                          dtype=self.dtype, d=d, there=there), counts, place

    def check_forward(self, Qr, Kr, Vr=None):
        (want, counts, place), (want_k, _, _) = self.want("q"), self.want("k")
        got = f64(Qr)
        assert np.all(got[~counts] == 7.0), "rows that do not count"
        off = np.abs(got - want["y"][0])[counts] / want["y"][1][counts]
        assert not off.size or off.max() <= 1.0, f"Qr: {off.max():.2f}"
        left = np.ones((self.batch, self.cache), bool)
        for b, i in zip(*np.nonzero(counts)):
            at = place[b, i]
            if 0 <= at < self.cache:
                left[b, at] = False
                off = np.abs(f64(Kr[b, at]) - want_k["y"][0][b, i]) / want_k["y"][1][b, i]
                assert off.max() <= 1.0, f"Kr at {b}, {i}: {off.max():.2f}"
                assert Vr is None or torch.equal(Vr[b, at], self.V[b, i])
        assert np.all(f64(Kr)[left] == 7.0) and (Vr is None or np.all(f64(Vr)[left] == 7.0)), "places that nothing goes to"

    def run_backward(self, values=False, **change):
        p = self.problem(values)
        out = {k: torch.full(getattr(self, k[1:]).shape, 7.0, dtype=DTYPE[self.dtype], device="cuda") for k in ("dQ", "dK")}
        out.update(change)
        names = [k for k, v in self.vectors.items() if v is not None and self.norm != "none"]
        sums = {k: torch.full_like(self.vectors[k], 7.0, dtype=torch.float32) for k in names}
        g = L.rotary_gradients(change.get("dQr", self.dQr), change.get("dKr", self.dKr), out["dQ"], out["dK"], **sums)
        n = L.lsp_rotary_backward_workspace_bytes(p, self.code)
        ws = torch.full((max(n, 16),), 255, dtype=torch.uint8, device="cuda")
        L.lsp_rotary_backward(p, g, self.code, ws, n, torch.cuda.current_stream())
        return dict(out, **sums)

    def check_backward(self, got):
        counts, _, place = ref.tokens(self.batch, self.length, *(None if x is None else x.numpy() for x in (self.positions, self.starts, self.lens)))
        for which in "qk":
            there = counts if which == "q" else counts & (place >= 0) & (place < self.cache)
            d = f64(self.dQr) if which == "q" else np.zeros(self.K.shape)
            if which == "k":
                for b, i in zip(*np.nonzero(there)):
                    d[b, i] = f64(self.dKr[b, place[b, i]])
            d[~there] = 0.0
            want, _, _ = self.want(which, d, there)
            dx = f64(got["d" + which.upper()])
            assert np.all(dx[~there] == 0.0), "gradients of rows that do not count"
            off = (np.abs(dx - want["dx"][0]) / want["dx"][1])[there]
            assert not off.size or off.max() <= 1.0, f"d{which.upper()}: {off.max():.2f}"
            for name in ("weight", "bias"):
                if f"{which}_{name}" in got:
                    check(got[f"{which}_{name}"], want[name], f"{which}_{name}")


SHAPES = [
    # dtype, batch, length, heads, kv_heads, dim, rotated, more
    ("bf16", 2, 37, 4, 2, 128, 128, dict(norm="rms")),
    ("f16", 2, 37, 4, 2, 128, 128, dict(norm="rms", neighbours=True)),
    ("f32", 2, 37, 4, 2, 128, 128, dict(norm="layer", bias=True)),
    ("f32", 1, 5, 3, 3, 8, 8, dict(norm="rms")),
    ("bf16", 1, 5, 3, 1, 24, 16, dict(norm="layer", bias=True, neighbours=True)),
    ("f16", 3, 9, 4, 4, 32, 8, dict(norm="rms", bias=True)),
    ("bf16", 2, 301, 8, 2, 80, 32, dict(norm="layer", bias=True, neighbours=True)),
    ("f32", 2, 65, 5, 5, 96, 96, dict(norm="none")),
    ("bf16", 2, 65, 12, 4, 64, 64, dict(norm="none", neighbours=True)),
    ("f16", 1, 1, 1, 1, 64, 0, dict(norm="rms")),
    ("bf16", 1, 1, 33, 3, 128, 64, dict(norm="rms", weights=False)),
    ("bf16", 1, 3000, 2, 1, 40, 40, dict(norm="layer")),
    ("f32", 1, 20000, 1, 1, 16, 16, dict(norm="rms", bias=True)),
]


@pytest.mark.parametrize("dtype,batch,length,heads,kv_heads,dim,rotated,more", SHAPES)
def test_forward_and_backward(dtype, batch, length, heads, kv_heads, dim, rotated, more):
    c = Case(dtype, batch, length, heads, kv_heads, dim, rotated, **more)
    L.lsp_rotary_forward(c.problem(), c.code, torch.cuda.current_stream())
    c.check_forward(c.Qr, c.Kr, c.Vr)
    c.check_backward(c.run_backward())


@pytest.mark.parametrize("norm", ["none", "rms", "layer"])
@pytest.mark.parametrize("lens", [[5, 0, 11], [1, 12, -3], [0, 0, 0]])
def test_rows_that_do_not_count_are_neither_read_nor_written(norm, lens):
    c = Case("bf16", 3, 11, 4, 2, 64, 32, norm=norm, lens=lens, bias=True, seed=3)
    for b, n in enumerate(lens):
        for t in (c.Q, c.K, c.V, c.dQr, c.dKr):
            t[b, max(0, min(n, 11)):] = float("nan")
    L.lsp_rotary_forward(c.problem(), c.code, torch.cuda.current_stream())
    for t in (c.Q, c.K, c.V, c.dQr, c.dKr):                                  # (the reference multiplies them by zeros)
        back = torch.nan_to_num(t.float(), nan=0.0)
        if t is c.dQr or t is c.dKr:
            t.copy_(t)
        setattr(c, {id(c.Q): "Q0", id(c.K): "K0", id(c.V): "V0", id(c.dQr): "dQr0", id(c.dKr): "dKr0"}[id(t)], back)
    got = c.run_backward()
    c.Q, c.K, c.V, c.dQr, c.dKr = c.Q0, c.K0, c.V0.to(c.V.dtype), c.dQr0, c.dKr0
    c.check_forward(c.Qr, c.Kr, c.Vr)
    c.check_backward(got)


@pytest.mark.parametrize("starts", [[0, 20, 7], [30, 31, 29], [-2, 40, 2 ** 31 - 1]])
def test_keys_and_values_go_to_their_places(starts):
    """Places before the cache and behind it are not written, and their keys have no gradient."""
    c = Case("f16", 3, 4, 4, 2, 64, 64, cache=32, starts=starts, lens=[4, 3, 4], seed=5)
    L.lsp_rotary_forward(c.problem(), c.code, torch.cuda.current_stream())
    c.check_forward(c.Qr, c.Kr, c.Vr)
    c.check_backward(c.run_backward())


def test_positions_are_other_than_places():
    far = [[0, 1000003, 5, 2 ** 31 - 1], [7, 7, -9, -2 ** 31]]
    c = Case("f32", 2, 4, 2, 1, 32, 32, cache=9, positions=far, starts=[5, 1], seed=6)
    L.lsp_rotary_forward(c.problem(), c.code, torch.cuda.current_stream())
    c.check_forward(c.Qr, c.Kr, c.Vr)
    c.check_backward(c.run_backward())


def test_in_place():
    """Turning in place, and gradients where those of the results are, gives the same bits."""
    c = Case("bf16", 2, 50, 4, 2, 128, 128, norm="rms", seed=7)
    stream = torch.cuda.current_stream()
    L.lsp_rotary_forward(c.problem(), c.code, stream)
    want = c.run_backward()
    dQ, dK = c.dQr.clone(), c.dKr.clone()
    got = c.run_backward(dQr=dQ, dKr=dK, dQ=dQ, dK=dK)
    assert all(torch.equal(want[k], got[k]) for k in want)
    Q, K = c.Q.clone(), c.K.clone()
    L.lsp_rotary_forward(c.problem(values=False, Q=Q, Qr=Q, K=K, Kr=K), c.code, stream)
    assert torch.equal(Q, c.Qr) and torch.equal(K, c.Kr)


def test_gradients_by_differences():
    """Along a direction, in fp32 with a step that the curvature allows: (f(x + h e) - f(x - h e)) / 2h against the gradient."""
    c = Case("f32", 2, 13, 3, 3, 16, 16, norm="layer", bias=True, neighbours=True, seed=8)
    got = c.run_backward()
    loss = lambda: float((f64(c.Qr) * f64(c.dQr)).sum() + (f64(c.Kr) * f64(c.dKr)).sum())
    stream = torch.cuda.current_stream()
    for which in ("Q", "K"):
        x, e = getattr(c, which), torch.randn(c.Q.shape, generator=torch.Generator().manual_seed(9)).cuda()
        kept, h, f = x.clone(), 1e-2, []
        for sign in (1, -1):
            x.copy_(kept + sign * h * e)
            L.lsp_rotary_forward(c.problem(), c.code, stream)
            f.append(loss())
        x.copy_(kept)
        there = float((f64(got["d" + which]) * f64(e)).sum())
        # results are off by up to (D + 32) EPS of about 10 magnitudes each, summed with 1248 gradients as random signs; the third derivative's part is h^2 / 6 of some hundreds
        assert abs((f[0] - f[1]) / (2 * h) - there) <= 0.02 * max(1.0, abs(there)) + 0.05, (which, f, there)


def test_a_captured_call_repeats():
    c = Case("bf16", 2, 100, 8, 8, 128, 128, norm="rms", seed=10)
    stream = torch.cuda.Stream()
    p = c.problem()
    dQ, dK = torch.empty_like(c.dQr), torch.empty_like(c.dKr)
    w = torch.empty(128, device="cuda")
    g = L.rotary_gradients(c.dQr, c.dKr, dQ, dK, q_weight=w)
    n = L.lsp_rotary_backward_workspace_bytes(p, c.code)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        L.lsp_rotary_forward(p, c.code, torch.cuda.current_stream())
        L.lsp_rotary_backward(p, g, c.code, ws, n, torch.cuda.current_stream())
    for seed in range(3):
        c.Q.copy_(torch.randn(c.Q.shape, generator=torch.Generator().manual_seed(seed)))
        c.Qr.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        c.check_forward(c.Qr, c.Kr, c.Vr)
        c.vectors, kept = dict(c.vectors, k_weight=c.vectors["k_weight"]), c.vectors
        c.check_backward(dict(dQ=dQ, dK=dK, q_weight=w))
        c.vectors = kept


def test_the_cache_is_what_attention_reads():
    """Single tokens: the call that turns the keys fills the cache, and attention over it is attention over all keys turned at once."""
    c = Case("f32", 2, 6, 4, 2, 64, 64, norm="rms", seed=11)
    stream = torch.cuda.current_stream()
    L.lsp_rotary_forward(c.problem(), c.code, stream)
    O, logs = torch.empty_like(c.Qr), torch.empty(2, 4, 6, device="cuda")
    p = L.attention_problem(c.Qr, c.Kr, c.V, O, logs, scale=0.125, causal=True)
    n = L.lsp_attention_forward_workspace_bytes(p, 0)
    L.lsp_attention_forward(p, 0, torch.empty(max(n, 16), dtype=torch.uint8, device="cuda"), n, stream)
    K, V = (torch.zeros(2, 10, 2, 64, device="cuda") for _ in range(2))
    for i in range(6):
        q, o, one = torch.empty(2, 1, 4, 64, device="cuda"), torch.empty(2, 1, 4, 64, device="cuda"), torch.empty(2, 4, 1, device="cuda")
        starts = torch.full((2,), i, dtype=torch.int32, device="cuda")
        step = L.rotary_problem(c.Q[:, i:i + 1], c.K[:, i:i + 1], q, K, V=c.V[:, i:i + 1], Vr=V, frequencies=c.frequencies, starts=starts, norm="rms", q_weight=c.vectors["q_weight"],
                                k_weight=c.vectors["k_weight"])
        L.lsp_rotary_forward(step, 0, stream)
        lens = starts + 1
        p = L.attention_problem(q, K, V, o, one, k_lens=lens, scale=0.125, causal=True)
        n = L.lsp_attention_forward_workspace_bytes(p, 0)
        L.lsp_attention_forward(p, 0, torch.empty(max(n, 16), dtype=torch.uint8, device="cuda"), n, stream)
        # the same keys bit by bit; attention sums them in another order: 64 products and 6 keys in fp32, of values of about 10
        assert torch.equal(q[:, 0], c.Qr[:, i]) and torch.equal(K[:, i], c.Kr[:, i])
        assert float((o[:, 0] - O[:, i]).abs().max()) <= 2.0 ** -24 * 200 * 10
