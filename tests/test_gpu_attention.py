"""Attention and its backward pass against the definition in 64 bits (operator_reference.py, with bounds derived from the kernels' roundings)."""
import math

import numpy as np
import pytest
import torch

import operator_reference as ref
import paper_2406_10181_amd as L

pytestmark = pytest.mark.gpu
_TORCH = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_CODE = {"f32": 0, "f16": 1, "bf16": 2}


def _normal(seed, dtype, *shape):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(*shape, generator=g).to(_TORCH[dtype])


def _lens(x):
    return None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")


class Call:
    """Tensors of one problem on the GPU, filled with NaN where something is written."""

    def __init__(self, dtype, Q, K, V, dO=None, **options):
        self.dtype, self.code, self.options = dtype, _CODE[dtype], options
        self.Q, self.K, self.V, self.dO = (None if t is None else t.cuda() for t in (Q, K, V, dO))
        self.make_outputs()

    def make_outputs(self):
        B, Sq, H, D = self.Q.shape
        nan = float("nan")
        self.O = torch.full((B, Sq, H, D), nan, dtype=self.Q.dtype, device="cuda")
        self.L = torch.full((B, H, Sq), nan, device="cuda")
        if self.dO is not None:
            self.dQ = torch.full_like(self.O, nan)
            self.dK = torch.full(self.K.shape, nan, dtype=self.Q.dtype, device="cuda")
            self.dV = torch.full(self.K.shape, nan, dtype=self.Q.dtype, device="cuda")

    def enqueue(self, stream=None):
        o = dict(self.options)
        o["q_lens"], o["k_lens"] = self.q_lens, self.k_lens
        p = L.attention_problem(self.Q, self.K, self.V, self.O, self.L, **o)
        n = L.lsp_attention_forward_workspace_bytes(p, self.code)
        self.ws = torch.full((max(n, 16) // 4,), float("nan"), device="cuda") if not hasattr(self, "ws") else self.ws
        L.lsp_attention_forward(p, self.code, self.ws, n, stream)
        if self.dO is not None:
            n = L.lsp_attention_backward_workspace_bytes(p, self.code)
            self.bws = torch.full((n // 4,), float("nan"), device="cuda") if not hasattr(self, "bws") else self.bws
            L.lsp_attention_backward(p, L.attention_gradients(self.dO, self.dQ, self.dK, self.dV), self.code, self.bws, n, stream)

    def run(self):
        self.q_lens, self.k_lens = _lens(self.options.get("q_lens")), _lens(self.options.get("k_lens"))
        self.enqueue(torch.cuda.current_stream())
        torch.cuda.synchronize()
        return self.results()

    def results(self):
        names = ("O", "L", "dQ", "dK", "dV") if self.dO is not None else ("O", "L")
        return {n: getattr(self, n).clone() for n in names}


def _check(got, want, what):
    for name, (value, bound) in want.items():
        g = got[name].double().cpu().numpy()
        fine = np.isfinite(value)
        assert np.array_equal(g[~fine], value[~fine]), f"{what}: {name} where nothing is seen"
        assert np.isfinite(g[fine]).all(), f"{what}: {name} is not finite"
        off = np.abs(g[fine] - value[fine])
        worst = float(np.max(off / np.maximum(bound[fine], 1e-300), initial=0.0))
        assert worst <= 1.0, f"{what}: {name} is {worst:.2f} times its bound off"


def _problem(dtype, B, H, Hk, Sq, Sk, D, seed=1, backward=True):
    Q, K, V = _normal(seed, dtype, B, Sq, H, D), _normal(seed + 1, dtype, B, Sk, Hk, D), _normal(seed + 2, dtype, B, Sk, Hk, D)
    return Q, K, V, _normal(seed + 3, dtype, B, Sq, H, D) if backward else None


def _against_reference(dtype, B, H, Hk, Sq, Sk, D, backward=True, seed=1, **options):
    Q, K, V, dO = _problem(dtype, B, H, Hk, Sq, Sk, D, seed, backward)
    options.setdefault("scale", 1.0 / math.sqrt(D))
    got = Call(dtype, Q, K, V, dO, **options).run()
    f = [None if t is None else t.double().numpy() for t in (Q, K, V, dO)]
    _check(got, ref.attention(*f[:3], dO=f[3], dtype=dtype, **{**dict(causal=False), **options}), (dtype, B, H, Hk, Sq, Sk, D, options))
    return got


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("Sq,Sk", [(1, 1), (1, 2), (2, 1), (31, 33), (64, 64), (65, 127), (128, 129), (200, 31), (31, 200), (257, 300)])
@pytest.mark.parametrize("causal", [False, True])
def test_lengths(dtype, Sq, Sk, causal):
    """Lengths round the tiles' sizes; causal with more queries than keys leaves the first ones without any."""
    _against_reference(dtype, 2, 2, 1, Sq, Sk, 64, causal=causal)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("D", [8, 16, 24, 32, 40, 64, 72, 80, 96, 104, 128])
def test_head_dims(dtype, D):
    _against_reference(dtype, 1, 2, 2, 150, 150, D, causal=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,Hk", [(1, 1), (4, 1), (6, 2), (6, 3), (8, 8)])
def test_shared_heads(dtype, H, Hk):
    _against_reference(dtype, 3, H, Hk, 100, 100, 32, causal=True)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("q_lens,k_lens", [([150, 1, 0, 77, 64], [150, 1, 0, 77, 64]), ([150, 150, 3, 70, 128], [0, 9, 150, 65, 1]),
                                           (None, [150, 0, 64, 1, 149]), ([0, 150, 65, 2, 64], None), ([1000, -5, 20, 20, 20], [1000, 20, -5, 150, 20])])
def test_ragged_batches(dtype, causal, q_lens, k_lens):
    """Lengths of zero and one, rows that see nothing, lengths outside the range (taken as the nearer end)."""
    _against_reference(dtype, 5, 2, 1, 150, 150, 32, causal=causal, q_lens=q_lens, k_lens=k_lens)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("Sq,Sk,H,Hk", [(1, 1500, 8, 2), (1, 700, 3, 3), (3, 1111, 8, 1), (5, 2000, 40, 1), (17, 3000, 2, 2), (1, 8, 8, 2), (40, 513, 4, 2)])
def test_few_queries(dtype, Sq, Sk, H, Hk):
    """The keys are split among workgroups, and the query heads of a key head share tiles where they fit."""
    _against_reference(dtype, 2, H, Hk, Sq, Sk, 64, backward=Sk < 1000, causal=True)
    _against_reference(dtype, 2, H, Hk, Sq, Sk, 128, backward=False, causal=True, q_lens=[Sq, max(1, Sq - 1)], k_lens=[Sk // 2 + 1, 3])


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("p", [0.1, 0.5, 0.999])
@pytest.mark.parametrize("Sq,Sk,D", [(70, 70, 32), (130, 200, 64), (1, 300, 128)])
def test_dropout(dtype, p, Sq, Sk, D):
    _against_reference(dtype, 2, 4, 2, Sq, Sk, D, causal=True, dropout=p, seed=7)
    _against_reference(dtype, 1, 2, 1, Sq, Sk, D, dropout=p, offset=3)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_scores_of_any_size(dtype):
    """Scores of several hundred (one key takes everything, the running maximum moves often) and of nearly nothing."""
    Q, K, V, dO = _problem(dtype, 1, 2, 2, 200, 200, 64)
    for factor in (40.0, 1e-3):
        q = (Q.float() * factor).to(Q.dtype)
        got = Call(dtype, q, K, V, dO, scale=0.125, causal=True).run()
        f = [t.double().numpy() for t in (q, K, V, dO)]
        _check(got, ref.attention(*f[:3], dO=f[3], dtype=dtype, scale=0.125, causal=True), (dtype, factor))


def test_rising_scores_move_the_maximum():
    """Every key scores more than the one before, by more than the running maximum may lag."""
    Q, K, V, dO = _problem("bf16", 1, 1, 1, 64, 300, 32)
    Q, K = torch.zeros_like(Q), torch.zeros_like(K)
    Q[..., 0] = 1.0
    K[0, :, 0, 0] = torch.arange(300).to(K.dtype)
    got = Call("bf16", Q, K, V, dO, scale=1.0).run()
    f = [t.double().numpy() for t in (Q, K, V, dO)]
    _check(got, ref.attention(*f[:3], dO=f[3], dtype="bf16", scale=1.0, causal=False), "rising")


@pytest.mark.parametrize("size", [1e-6, 1e4])
def test_fp16_gradients_of_any_size(size):
    """Gradients far below and near the top of fp16's range: the gradients of the scores are scaled on the way."""
    Q, K, V, dO = _problem("f16", 2, 2, 1, 300, 300, 64)
    dO = (dO.float().clamp(-4, 4) * size).half()
    got = Call("f16", Q, K, V, dO, scale=0.125).run()
    f = [t.double().numpy() for t in (Q, K, V, dO)]
    want = ref.attention(*f[:3], dO=f[3], dtype="f16", scale=0.125, causal=False)
    if size > 1:
        assert np.abs(want["dV"][0]).max() < 65504
    _check(got, want, size)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_rows_that_do_not_count_are_not_read(dtype):
    """NaN and infinities behind the lengths change nothing, and what belongs to these rows is zero."""
    Q, K, V, dO = _problem(dtype, 3, 4, 2, 150, 150, 80)
    q_lens, k_lens = [150, 70, 0], [33, 101, 150]
    clean = Call(dtype, Q, K, V, dO, scale=0.1, q_lens=q_lens, k_lens=k_lens, causal=True, dropout=0.2, seed=5).run()
    for t, lens, bad in ((Q, q_lens, float("nan")), (dO, q_lens, float("inf")), (K, k_lens, float("-inf")), (V, k_lens, float("nan"))):
        for b, n in enumerate(lens):
            t[b, n:] = bad
    dirty = Call(dtype, Q, K, V, dO, scale=0.1, q_lens=q_lens, k_lens=k_lens, causal=True, dropout=0.2, seed=5).run()
    for name in clean:
        assert torch.equal(clean[name], dirty[name]), name
    for b in range(3):
        assert not dirty["O"][b, q_lens[b]:].any() and not dirty["dQ"][b, q_lens[b]:].any()
        assert not dirty["dK"][b, k_lens[b]:].any() and not dirty["dV"][b, k_lens[b]:].any()
        assert (dirty["L"][b, :, q_lens[b]:] == -math.inf).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strides(dtype):
    """Views into a joint projection, heads before positions, inputs broadcast over batches and positions: the results of contiguous tensors."""
    B, S, H, Hk, D = 2, 130, 4, 2, 64
    joint = _normal(1, dtype, B, S, H + 2 * Hk, D).cuda()
    views = joint.split([H, Hk, Hk], dim=2)
    dO = _normal(2, dtype, B, S, H, D).cuda()
    options = dict(scale=0.125, causal=True)
    plain = Call(dtype, *[v.contiguous() for v in views], dO, **options).run()

    def same(call, what):
        got = call.run()
        for name in plain:
            assert torch.equal(plain[name], got[name]), (what, name)

    same(Call(dtype, *views, dO, **options), "joint projection")
    same(Call(dtype, *[v.transpose(1, 2).contiguous().transpose(1, 2) for v in views], dO.transpose(1, 2).contiguous().transpose(1, 2), **options), "heads first")
    call = Call(dtype, *views, dO, **options)
    outs = torch.full((B, H + 2 * Hk, S, D), float("nan"), dtype=joint.dtype, device="cuda").split([H, Hk, Hk], dim=1)
    call.dQ, call.dK, call.dV = (t.transpose(1, 2) for t in outs)
    call.O = torch.full((S, B, H, D), float("nan"), dtype=joint.dtype, device="cuda").transpose(0, 1)
    same(call, "outputs of other orders")
    # broadcast inputs: one text's keys for all, one gradient for all positions
    K1, V1, d1 = views[1][:1].contiguous(), views[2][:1].contiguous(), dO[:, :1].contiguous()
    wide = Call(dtype, views[0], K1.expand(B, S, Hk, D), V1.expand(B, S, Hk, D), d1.expand(B, S, H, D), **options).run()
    full = Call(dtype, views[0], K1.repeat(B, 1, 1, 1), V1.repeat(B, 1, 1, 1), d1.repeat(1, S, 1, 1), **options).run()
    for name in wide:
        assert torch.equal(wide[name], full[name]), name


def test_offsets_past_32_bits():
    """A cache of more than 4 GiB: positions nearly 8 MiB apart, in front of and behind 2^31 and 2^32 bytes."""
    S, D, step = 600, 64, (8 << 20) // 2 - 8
    store = torch.empty(S * step, dtype=torch.bfloat16, device="cuda")
    K, V = (torch.as_strided(store, (1, S, 1, D), (S * step, step, D, 1), o) for o in (0, 64))
    Q, Kc, Vc, dO = _problem("bf16", 1, 2, 1, 70, S, D)
    K.copy_(Kc.cuda())
    V.copy_(Vc.cuda())
    got = Call("bf16", Q, K, V, dO, scale=0.125, causal=True).run()
    want = Call("bf16", Q, Kc, Vc, dO, scale=0.125, causal=True).run()
    for name in want:
        assert torch.equal(want[name], got[name]), name


@pytest.mark.parametrize("dtype,dropout", [("bf16", 0.0), ("f16", 0.2), ("f32", 0.0)])
def test_same_bits_again_on_any_stream_and_in_graphs(dtype, dropout):
    call = Call(dtype, *_problem(dtype, 2, 4, 1, 333, 333, 64), scale=0.125, causal=True, dropout=dropout)
    first = call.run()
    for _ in range(3):
        again = call.run()
        for name in first:
            assert torch.equal(first[name], again[name]), name
    stream = torch.cuda.Stream()
    call.make_outputs()
    torch.cuda.synchronize()
    call.enqueue(stream)
    stream.synchronize()
    for name, t in call.results().items():
        assert torch.equal(first[name], t), name
    graph = torch.cuda.CUDAGraph()
    call.make_outputs()
    with torch.cuda.graph(graph):
        call.enqueue(torch.cuda.current_stream())
    for k in range(3):
        for name in first:
            getattr(call, name).fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        for name, t in call.results().items():
            assert torch.equal(first[name], t), (k, name)


@pytest.mark.parametrize("dropout", [0.0, 0.3])
def test_gradients_against_differences(dropout):
    """The change of <O, dO> along a direction, by central differences of the forward pass.  With steps of 2^-5 the third derivative leaves
    about 2^-10 / 6 of what the gradients' norms allow, and fp32 (2^-24 of sums of 10^4 terms over the step) less: a hundredth of that norm is the bound."""
    Q, K, V, dO = _problem("f32", 1, 4, 2, 48, 48, 32)
    options = dict(scale=0.17, causal=True, dropout=dropout, seed=11)
    got = Call("f32", Q, K, V, dO, **options).run()
    step = 2.0 ** -5
    for k, name in enumerate(("dQ", "dK", "dV")):
        u = _normal(50 + k, "f32", *(Q, K, V)[k].shape)
        u /= u.norm()
        sides = []
        for sign in (1.0, -1.0):
            moved = [Q, K, V]
            moved[k] = moved[k] + sign * step * u
            sides.append(float((Call("f32", *moved, **options).run()["O"].double().cpu() * dO.double()).sum()))
        by_difference = (sides[0] - sides[1]) / (2 * step)
        g = got[name].double().cpu()
        assert abs(by_difference - float((g * u).sum())) <= 0.01 * float(g.norm()), name


def test_workspace_is_all_that_is_touched():
    """Guards behind the workspaces, and behind L, stay."""
    call = Call("bf16", *_problem("bf16", 1, 4, 2, 3, 2000, 64), scale=0.125)
    p = L.attention_problem(call.Q, call.K, call.V, call.O, call.L, scale=0.125)
    sizes = L.lsp_attention_forward_workspace_bytes(p, 2), L.lsp_attention_backward_workspace_bytes(p, 2)
    assert sizes[0] > 0
    call.ws, call.bws = (torch.full((n // 4 + 64,), 7.0, device="cuda") for n in sizes)
    room = torch.full((call.L.numel() + 64,), 7.0, device="cuda")
    call.L = room[: call.L.numel()].view(call.L.shape)
    call.run()
    for n, t in ((sizes[0] // 4, call.ws), (sizes[1] // 4, call.bws), (call.L.numel(), room)):
        assert (t[n:] == 7.0).all()
