"""Rotary positions, cross entropy and AdamW where offsets pass 32 bits, on streams side by side, and in graphs that share a workspace."""
import pytest
import torch

import paper_2406_10181_amd as L
import training_reference as ref

pytestmark = pytest.mark.gpu
U = ref.U["bf16"]


def randn(*shape, seed=0, dtype=torch.bfloat16):
    return torch.randn(*shape, generator=torch.Generator("cuda").manual_seed(seed), device="cuda", dtype=dtype)


def test_places_far_into_a_cache():
    """4.5 GB of keys: what goes to their ends is what goes to a small cache, and nothing else is written."""
    batch, length, cache, heads, dim = 2, 7, 1_100_000, 8, 128
    K, Q = randn(batch, length, heads, dim), randn(batch, length, heads, dim, seed=1)
    starts = torch.tensor([3, cache - 5], dtype=torch.int32, device="cuda")                 # (two places of the last text are behind its cache)
    positions = starts[:, None] + torch.arange(length, dtype=torch.int32, device="cuda")
    frequencies = 100.0 ** (-torch.arange(dim // 2, device="cuda", dtype=torch.float32) / 64)
    far, near = (torch.full((batch, n, heads, dim), 7.0, dtype=torch.bfloat16, device="cuda") for n in (cache, length))
    values = torch.full_like(far, 7.0)
    stream = torch.cuda.current_stream()
    common = dict(frequencies=frequencies, norm="rms")
    p = L.rotary_problem(Q, K, torch.empty_like(Q), far, V=Q, Vr=values, starts=starts, **common)
    L.lsp_rotary_forward(p, 2, stream)
    L.lsp_rotary_forward(L.rotary_problem(Q, K, torch.empty_like(Q), near, positions=positions, **common), 2, stream)
    there = 0
    for b in range(batch):
        n = min(length, cache - int(starts[b]))
        at = slice(int(starts[b]), int(starts[b]) + n)
        assert torch.equal(far[b, at], near[b, :n]) and torch.equal(values[b, at], Q[b, :n])
        there += n
    for x in (far, values):
        assert int((x.view(-1, heads * dim) != 7.0).any(1).sum()) == there
    del values, x                                                                           # and back: the same gradients from far places
    d = randn(batch, length, heads, dim, seed=2)
    for b in range(batch):
        n = min(length, cache - int(starts[b]))
        far[b, int(starts[b]):int(starts[b]) + n] = d[b, :n]
    d[1, 5:] = 0.0
    out = [torch.empty_like(K) for _ in range(4)]
    p = L.rotary_problem(Q, K, torch.empty_like(Q), torch.empty_like(far), starts=starts, **common)
    L.lsp_rotary_backward(p, L.rotary_gradients(d, far, out[0], out[1]), 2, None, 0, stream)
    p = L.rotary_problem(Q, K, torch.empty_like(Q), near, positions=positions, **common)
    L.lsp_rotary_backward(p, L.rotary_gradients(d, d, out[2], out[3]), 2, None, 0, stream)
    assert torch.equal(out[0], out[2]) and torch.equal(out[1], out[3])


def test_the_largest_vocabulary():
    """2^20 words of width 2056: 4.3 GB of W and of its gradient."""
    rows, width, vocab = 40, 2056, 1 << 20
    W, H = randn(vocab, width) / width ** 0.5, randn(rows, width, seed=1)
    targets = torch.randint(0, vocab, (rows,), generator=torch.Generator().manual_seed(2)).cuda()
    targets[0], targets[1] = vocab - 1, vocab
    losses, dH, dW = torch.empty(rows, device="cuda"), torch.empty_like(H), torch.empty_like(W)
    p = L.cross_entropy_problem(H, W, targets, losses)
    n = L.lsp_cross_entropy_backward_workspace_bytes(p, 2)
    L.lsp_cross_entropy_backward(p, L.cross_entropy_gradients(dH, dW), 2, torch.empty(n, dtype=torch.uint8, device="cuda"), n, torch.cuda.current_stream())
    wide, h = W.double(), H.double()
    z = h.mm(wide.t())
    lse = torch.logsumexp(z, 1)
    at = torch.arange(rows, device="cuda")
    t = targets.clamp(max=vocab - 1)
    want = lse - z[at, t]
    dz = torch.exp(z - lse[:, None])
    dz[at, t] -= 1.0
    want[1], dz[1] = 0.0, 0.0
    of_h, of_w = dz.mm(wide), dz.t().mm(h)
    # norms: losses of some 14 from sums of 2056 products; 16 bits: two roundings of a probability (none of a target's), one of the result
    rel = lambda got, right: float((got.double() - right).norm() / right.norm())
    assert rel(losses, want) <= 2e-5 and rel(dH, of_h) <= 3 * U
    for part in (slice(0, 1000), slice(vocab // 2 - 500, vocab // 2 + 500), slice(vocab - 1000, vocab), slice(0, vocab)):
        assert rel(dW[part], of_w[part]) <= 3 * U, part


@pytest.mark.parametrize("states,n", [("8bit", (1 << 31) + 777), ("f32", (1 << 30) + 777)])
def test_tensors_past_32_bits(states, n):
    """Parts of a tensor of 4.3 GB and more become what they become as tensors of their own."""
    if states == "8bit":
        t = dict(m=torch.randint(0, 100, (n,), dtype=torch.uint8, device="cuda"), v=torch.randint(0, 256, (n,), dtype=torch.uint8, device="cuda"),
                 m_scale=torch.rand((n + 255) // 256, device="cuda") * 1e-5, v_scale=torch.rand((n + 255) // 256, device="cuda") * 1e-5)
    else:
        t = dict(m=torch.randn(n, device="cuda") * 1e-3, v=torch.rand(n, device="cuda") * 1e-5)
    t.update(param=randn(n), grad=randn(n, seed=1))
    parts = []
    for begin, end in ((0, 5120), ((1 << 29) - 512, (1 << 29) + 512), (n - 777 - 2048, n)):
        of = lambda k, begin=begin, end=end: slice(begin // 256, (end + 255) // 256) if k.endswith("scale") else slice(begin, end)
        parts.append((of, {k: x[of(k)].clone() for k, x in t.items()}))
    rates = dict(rate=3e-3, step=3, stream=torch.cuda.current_stream())
    L.lsp_adamw(L.adamw_items([t]), **rates)
    for of, part in parts:
        before = part["param"].clone()
        L.lsp_adamw(L.adamw_items([part]), **rates)
        assert not torch.equal(before, part["param"])
        for k, x in t.items():
            assert torch.equal(x[of(k)], part[k]), k


def test_tensors_left_on_the_host_are_refused():
    H, W, t, losses = randn(6, 16), randn(30, 16), torch.zeros(6, dtype=torch.int64, device="cuda"), torch.zeros(6, device="cuda")
    for args, more in (((H, W.cpu(), t, losses), {}), ((H, W, t.cpu(), losses), {}), ((H, W, t, losses.cpu()), {}), ((H, W, t, losses), dict(logs=losses.cpu())), ((H.cpu(), W, t, losses), {})):
        with pytest.raises(ValueError):
            L.cross_entropy_problem(*args, **more)
    for args, more in (((H, W.cpu()), {}), ((H, W), dict(weights=losses.cpu()))):
        with pytest.raises(ValueError):
            L.cross_entropy_gradients(*args, **more)
    item = lambda **c: {**dict(param=randn(600), grad=randn(600), m=torch.zeros(600, device="cuda"), v=torch.zeros(600, device="cuda")), **c}
    for k in ("grad", "m", "v"):
        with pytest.raises(ValueError):
            L.adamw_items([item(), item(**{k: item()[k].cpu()})])
    with pytest.raises(ValueError):
        L.lsp_adamw(L.adamw_items([item()]), rate=1e-3, step=1, grad_scale=torch.ones(1), stream=torch.cuda.current_stream())


def calls_of(seed):
    """A call of each operator, on tensors of its own: (run(stream), results)."""
    Q, K = randn(2, 300, 8, 64, seed=seed), randn(2, 300, 8, 64, seed=seed + 1)
    Qr, Kr, dQ, dK, w = torch.empty_like(Q), torch.empty_like(K), torch.empty_like(Q), torch.empty_like(K), torch.empty(64, device="cuda")
    frequencies = torch.rand(32, device="cuda")
    p = L.rotary_problem(Q, K, Qr, Kr, frequencies=frequencies, norm="rms")
    g = L.rotary_gradients(K, Q, dQ, dK, q_weight=w)
    H, W, t = randn(700, 264, seed=seed), randn(3000, 264, seed=seed + 1) / 16, torch.randint(-1000, 3000, (700,), device="cuda")
    losses, dH, dW = torch.empty(700, device="cuda"), torch.empty_like(H), torch.empty_like(W)
    c, cg = L.cross_entropy_problem(H, W, t, losses), L.cross_entropy_gradients(dH, dW)
    sizes = L.lsp_rotary_backward_workspace_bytes(p, 2), L.lsp_cross_entropy_backward_workspace_bytes(c, 2)
    item = dict(param=W.clone(), grad=dW, m=torch.zeros(W.shape, device="cuda"), v=torch.zeros(W.shape, device="cuda"))
    items = L.adamw_items([item])

    def run(stream, workspace):
        L.lsp_rotary_forward(p, 2, stream)
        L.lsp_rotary_backward(p, g, 2, workspace, sizes[0], stream)
        L.lsp_cross_entropy_backward(c, cg, 2, workspace, sizes[1], stream)
        L.lsp_adamw(items, rate=1e-3, step=1, stream=stream)
    kept = (Q, K, frequencies, H, W, t, p, g, c, cg, items)           # (descriptors hold addresses only)
    return run, (Qr, Kr, dQ, dK, w, losses, dH, dW), item, max(sizes), kept


def begin_again(results, item, param):
    for x in results:
        x.fill_(7.0)
    item["param"].copy_(param), item["m"].zero_(), item["v"].zero_()


def test_two_streams_at_once():
    """Each with a workspace of its own; what comes of it is what comes of one after the other."""
    both = [calls_of(10), calls_of(20)]
    params = [c[2]["param"].clone() for c in both]
    spaces = [torch.empty(c[3], dtype=torch.uint8, device="cuda") for c in both]
    want = []
    for (run, results, item, _, _), space in zip(both, spaces):
        run(torch.cuda.current_stream(), space)
        want.append([x.clone() for x in (*results, *item.values())])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        for (_, results, item, _, _), param in zip(both, params):
            begin_again(results, item, param)
        torch.cuda.synchronize()
        for (run, *_), space, stream in zip(both, spaces, streams):
            run(stream, space)
        torch.cuda.synchronize()
        for (_, results, item, _, _), right in zip(both, want):
            assert all(torch.equal(x, y) for x, y in zip((*results, *item.values()), right))


def test_two_graphs_that_share_a_workspace():
    """Nothing of a call is kept in its workspace; replays with eager work between."""
    both = [calls_of(30), calls_of(40)]
    params = [c[2]["param"].clone() for c in both]
    space = torch.empty(max(c[3] for c in both), dtype=torch.uint8, device="cuda")
    want = []
    for run, results, item, _, _ in both:
        run(torch.cuda.current_stream(), space)
        want.append([x.clone() for x in (*results, *item.values())])
    torch.cuda.synchronize()
    graphs = []
    for run, *_ in both:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            run(torch.cuda.current_stream(), space)
        graphs.append(graph)
    for k in range(4):
        for (_, results, item, _, _), param in zip(both, params):
            begin_again(results, item, param)
        space.fill_(255)
        for graph in graphs if k % 2 else reversed(graphs):
            graph.replay()
        torch.cuda.synchronize()
        for (_, results, item, _, _), right in zip(both, want):
            assert all(torch.equal(x, y) for x, y in zip((*results, *item.values()), right))
