"""lsp_adamw against the definition in 64 bits, through the C ABI."""
import numpy as np
import pytest
import torch

import paper_2406_10181_amd as L
import training_reference as ref
from operator_reference import EPS, TINY, U

pytestmark = pytest.mark.gpu
DTYPE = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
RATES = dict(rate=3e-3, beta1=0.9, beta2=0.98, eps=1e-8)


def f64(t):
    return t.double().cpu().numpy()


def tensor(n, dtype, grad, states, master, seed, decay=0.1, rate_factor=1.0, guard=64):
    """A dict for adamw_items whose tensors are pieces of longer ones; the rest is 7 and has to stay so."""
    g = torch.Generator().manual_seed(seed)
    whole = {}

    def piece(name, values, t):
        x = torch.full((len(values) + guard,), 7, dtype=t, device="cuda")
        x[: len(values)] = values.to(t).cuda() if t != torch.uint8 else values.cuda()
        whole[name] = x
        return x[: len(values)]

    p, blocks = torch.randn(n, generator=g) * 0.05, (n + 255) // 256
    d = dict(param=piece("param", p, DTYPE[dtype]), grad=piece("grad", torch.randn(n, generator=g) * torch.exp(2 * torch.randn(n, generator=g)) * 0.01, DTYPE[grad]), decay=decay, rate_factor=rate_factor)
    if states == "f32":
        d["m"], d["v"] = piece("m", torch.randn(n, generator=g) * 1e-3, torch.float32), piece("v", torch.rand(n, generator=g) * 1e-5, torch.float32)
    else:
        code = torch.randint(0, 256, (n,), generator=g).to(torch.uint8)
        code[(code & 0x7F) == 0x7F] = 0                                      # e4m3's NaN
        d["m"], d["v"] = piece("m", code, torch.uint8), piece("v", torch.randint(0, 256, (n,), generator=g).to(torch.uint8), torch.uint8)
        d["m_scale"], d["v_scale"] = piece("m_scale", torch.rand(blocks, generator=g) * 1e-5, torch.float32), piece("v_scale", torch.rand(blocks, generator=g) * 1e-5, torch.float32)
    d["master"] = piece("master", p, torch.float32) if master else None
    return d, whole


def state_of(d, k):
    if "m_scale" not in d:
        return f64(d[k])
    n = d[k].numel()
    return (ref.m_values if k == "m" else ref.v_values)(d[k].cpu().numpy()) * ref.of_blocks(f64(d[k + "_scale"]), n)


def want_of(d, step, grad_scale=1.0, **rates):
    p = f64(d["param"] if d["master"] is None else d["master"])
    r = dict(RATES, **rates)
    r["rate"] *= d["rate_factor"]
    return ref.adamw(p, f64(d["grad"]), state_of(d, "m"), state_of(d, "v"), decay=d["decay"], step=step, grad_scale=grad_scale, **r)


def check(d, dtype, states, want, before):
    p, m, v, by = want
    n = len(p)
    ep = EPS * (2 * np.abs(p) + 24 * by) + 1e-37                             # some two dozen roundings on the way of an update, two of the sum
    if d["master"] is not None:
        off = np.abs(f64(d["master"]) - p)
        assert np.all(off <= ep), f"master {np.max(off / ep)}"
        assert torch.equal(d["param"], d["master"].to(DTYPE[dtype]))
    else:
        bound = ep * (1 + U[dtype]) + U[dtype] * np.abs(p) + TINY[dtype]
        off = np.abs(f64(d["param"]) - p)
        assert np.all(off <= bound), f"param {np.max(off / bound)}"
    size_m = np.abs(before["m"]) + np.abs(m) + np.abs(before["g"])
    for k, x, e in (("m", m, EPS * 4 * size_m + 1e-44), ("v", v, EPS * 6 * v + 1e-44)):
        if states == "f32":
            off = np.abs(f64(d[k]) - x)
            assert np.all(off <= e), f"{k} {np.max(off / e)}"
            continue
        largest = 448.0 if k == "m" else 1.875
        pad = np.zeros(-n % 256)
        top = np.concatenate([np.abs(x), pad]).reshape(-1, 256).max(1)
        etop = np.concatenate([e, pad]).reshape(-1, 256).max(1)
        scale = f64(d[k + "_scale"])
        assert np.all(np.abs(scale - top / largest) <= (2 * EPS * top + etop) / largest + 1e-44), k
        # a code stands for a value within half a step of what it was made of: steps are 2^-3 of the power of two below it, and not smaller than the smallest
        got = (ref.m_values if k == "m" else ref.v_values)(d[k].cpu().numpy())
        s = ref.of_blocks(top / largest, n)
        y = np.where(s > 0, x / np.where(s > 0, s, 1.0), 0.0)
        exponent = np.floor(np.log2(np.maximum(np.abs(y), 1e-300)))
        if k == "m":
            half = 2.0 ** (np.maximum(exponent, -6) - 4)
            assert np.all(np.abs(got - y) <= half * (1 + 1e-9) + 8 * EPS * np.abs(y) + np.where(s > 0, e / np.where(s > 0, s, 1.0), 0.0)), k
        else:
            half = 2.0 ** (np.maximum(exponent, -31) - 4)
            least = 2.0 ** -31 * 1.125
            fine = np.abs(got - y) <= half * (1 + 1e-9) + 12 * EPS * y
            assert np.all(fine | ((y <= least) & (got == least))), k
            assert np.all((got > 0) == (v > 0)), "a v that is not 0 never becomes 0"


def step_and_check(ds, dtype, states, step=3, grad_scale=None):
    scale = 1.0 if grad_scale is None else grad_scale
    want = [want_of(d, step, scale) for d in ds]
    before = [dict(m=state_of(d, "m"), g=f64(d["grad"]) * scale) for d in ds]
    at = None if grad_scale is None else torch.tensor([grad_scale], device="cuda")
    L.lsp_adamw(L.adamw_items(ds), step=step, grad_scale=at, stream=torch.cuda.current_stream(), **RATES)
    for d, w, b in zip(ds, want, before):
        check(d, dtype, states, w, b)


@pytest.mark.parametrize("states", ["f32", "8bit"])
@pytest.mark.parametrize("dtype,grad,master", [("f32", "f32", False), ("bf16", "bf16", False), ("bf16", "f32", True), ("f16", "f16", True), ("f16", "bf16", False), ("bf16", "f32", False)])
def test_sizes(states, dtype, grad, master):
    made = [tensor(n, dtype, grad, states, master, seed=n) for n in (1, 7, 255, 256, 257, 2047, 2048, 2049, 5000)]
    step_and_check([d for d, _ in made], dtype, states, grad_scale=0.5)
    for d, whole in made:
        for name, x in whole.items():
            assert bool((x[d[name].numel():] == 7).all()), f"{name}: written behind its end"


@pytest.mark.parametrize("states", ["f32", "8bit"])
def test_many_tensors_with_rates_of_their_own(states):
    """More than one launch holds."""
    made = [tensor(100 + 37 * k, "bf16", "f32", states, k % 3 == 0, seed=k, decay=0.01 * (k % 4), rate_factor=0.5 + k % 2) for k in range(71)]
    step_and_check([d for d, _ in made], "bf16", states, step=1)


def test_types_side_by_side():
    made = [(tensor(300 + k, dt, gr, "8bit", ma, seed=k)[0], dt) for k, (dt, gr, ma) in enumerate([("f32", "bf16", False), ("f16", "f32", True), ("bf16", "bf16", False)])]
    want = [want_of(d, 5) for d, _ in made]
    before = [dict(m=state_of(d, "m"), g=f64(d["grad"])) for d, _ in made]
    L.lsp_adamw(L.adamw_items([d for d, _ in made]), step=5, stream=torch.cuda.current_stream(), **RATES)
    for (d, dt), w, b in zip(made, want, before):
        check(d, dt, "8bit", w, b)


def test_training_begins_at_zeros():
    """States of all zeros, codes and scales; then some steps of them."""
    d, _ = tensor(1000, "f32", "f32", "8bit", False, seed=1)
    for k in ("m", "v", "m_scale", "v_scale"):
        d[k].zero_()
    for step in range(1, 6):
        step_and_check([d], "f32", "8bit", step=step)
        d["grad"].copy_(torch.randn(1000, generator=torch.Generator().manual_seed(step)))
    assert not (d["v"] == 0).any()


def test_gradients_of_zero_and_blocks_of_nothing():
    d, _ = tensor(700, "f32", "f32", "8bit", False, seed=2)
    for k in ("m", "v", "m_scale", "v_scale", "grad"):
        d[k].zero_()
    d["grad"][300] = 1e-3
    step_and_check([d], "f32", "8bit", step=1)
    assert int((d["v"] != 0).sum()) == 1 and float(d["v_scale"][0]) == 0.0


def test_tiny_blocks():
    """Largest values below 2^-90: their scales' inverses are infinite, the codes are as good as others'."""
    d, _ = tensor(600, "f32", "f32", "8bit", False, seed=3)
    d["m"].zero_(), d["v"].zero_()
    d["grad"].mul_(1e-16)
    step_and_check([d], "f32", "8bit", step=1)


@pytest.mark.parametrize("states", ["f32", "8bit"])
@pytest.mark.parametrize("eps", [0.0, 1e-46, 1e-8])
def test_elements_without_gradients_only_decay(states, eps):
    """m and v of 0: no update, also with an eps that is 0 in fp32."""
    d, _ = tensor(900, "f32", "f32", states, False, seed=8)
    for k in ("m", "v", "m_scale", "v_scale", "grad"):
        if k in d:
            d[k].zero_()
    d["grad"][::3] = 1e-2
    before = d["param"].clone()
    L.lsp_adamw(L.adamw_items([d]), step=1, stream=torch.cuda.current_stream(), **dict(RATES, eps=eps))
    without = torch.arange(900, device="cuda") % 3 != 0
    want = f64(before) * (1 - RATES["rate"] * d["decay"])
    assert np.all(np.abs(f64(d["param"]) - want)[without.cpu().numpy()] <= 3 * EPS * np.abs(want[without.cpu().numpy()]))
    moved = f64(d["param"] - before)[::3]
    assert np.all(np.abs(moved + RATES["rate"]) < 0.01 * RATES["rate"] + RATES["rate"] * d["decay"] * np.abs(f64(before)[::3]))


@pytest.mark.parametrize("bad", [float("inf"), float("nan"), -float("inf")])
def test_a_scale_that_is_not_finite_leaves_everything(bad):
    d, whole = tensor(3000, "bf16", "f32", "8bit", True, seed=4)
    kept = {k: x.clone() for k, x in whole.items()}
    L.lsp_adamw(L.adamw_items([d]), step=2, grad_scale=torch.tensor([bad], device="cuda"), stream=torch.cuda.current_stream(), **RATES)
    assert all(torch.equal(kept[k].view(torch.uint8), x.view(torch.uint8)) for k, x in whole.items())


def test_a_gradient_that_is_not_finite_spoils_its_element_and_block_only():
    d, _ = tensor(1024, "f32", "f32", "8bit", False, seed=5)
    d["grad"][300] = float("nan")
    L.lsp_adamw(L.adamw_items([d]), step=2, stream=torch.cuda.current_stream(), **RATES)
    assert torch.isnan(d["param"]).nonzero().flatten().tolist() == [300]


def test_a_captured_call_repeats():
    d, _ = tensor(5000, "bf16", "f32", "f32", True, seed=6)
    items = L.adamw_items([d])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        L.lsp_adamw(items, step=7, stream=torch.cuda.current_stream(), **RATES)
    for k in range(3):
        d["grad"].copy_(torch.randn(5000, generator=torch.Generator().manual_seed(k)))
        want, before = want_of(d, 7), dict(m=state_of(d, "m"), g=f64(d["grad"]))
        graph.replay()
        torch.cuda.synchronize()
        check(d, "bf16", "f32", want, before)
