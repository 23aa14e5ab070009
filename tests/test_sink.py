"""Attention with sinks, forward and backward, against the formulas in 64 bits, and what its entry points refuse.

Tolerances are what the roundings can add up to, element by element (u: half a step of the inputs' type, relative; z: half the smallest step of
binary16, absolute, for probabilities that small):
  output  u |O| (its own rounding) + sum_j (u P + z) |V|
  dV      u |dV| + sum_i (u P + z) |dO|
  dS      e = u |dS| + z + P u sum_c |dO O| (delta is formed from the rounded output);  dQ: u |dQ| + scale sum_j e |K|;  dK: u |dK| + scale sum_i e |Q|
and for sums, exponentials and the log-sum-exp in 32 bits f = 2e-5 relative to the sums of magnitudes (scores here stay below 60, whose
exponents are rounded by 60 log2(e) 2^-24 = 5e-6; sums of some thousand values in any order add a few 1e-6).
"""
import math

import pytest

torch = pytest.importorskip("torch")
import torch.utils.checkpoint  # noqa: E402

import paper_2506_06095_amd as smha  # noqa: E402

F = 2e-5


def rounding(dtype):
    return torch.finfo(dtype).eps / 2, 2.0 ** -25 if dtype == torch.float16 else 0.0


def visible(Sq, Sk, off, n, window, n_sink):
    """bool [Sq, Sk] for one sequence, entry by entry from the definition."""
    p = torch.arange(Sq)[:, None] + off
    j = torch.arange(Sk)[None, :]
    seen = (j <= p) & (p >= 0) & (p < n)
    return seen & ((p - j < window) | (j < n_sink)) if window else seen


def reference(q, k, v, g, window, n_sink, offsets, lengths, scale):
    """{name: (value, bound)} of out, lse, dq, dk, dv, in 64 bits on the CPU."""
    (B, H, Sq, d), (Hkv, Sk) = q.shape, k.shape[1:3]
    u, z = rounding(q.dtype)
    scale = scale if scale > 0 else d ** -0.5
    q, k, v, g = (t.detach().cpu().double() for t in (q, k, v, g))
    names = ("out", "dq", "dk", "dv")
    val = {n: torch.zeros_like(q if n in ("out", "dq") else k) for n in names}
    tol = {n: torch.zeros_like(val[n]) for n in names}
    lse = torch.full((B, H, Sq), -math.inf, dtype=torch.float64)
    for b in range(B):
        n = Sk if lengths is None else min(max(lengths[b], 0), Sk)
        off = Sk - Sq if offsets is None else offsets[b]
        seen = visible(Sq, Sk, off, n, window, n_sink)
        some = seen.any(1)
        if not some.any():
            continue
        # what is not seen may hold anything: it is taken out before it meets anything
        used = seen.any(0)
        for h in range(H):
            c = h * Hkv // H
            Q, G = (torch.where(some[:, None], t[b, h], 0.0) for t in (q, g))
            K, V = (torch.where(used[:, None], t[b, c], 0.0) for t in (k, v))
            s = (Q @ K.T * scale).masked_fill(~seen, -math.inf)
            l = torch.logsumexp(s, 1)
            P = torch.where(seen, torch.exp(s - torch.where(some, l, 0.0)[:, None]), 0.0)
            lse[b, h] = l
            O = P @ V
            dP, delta = G @ V.T, (G * O).sum(1, keepdim=True)
            dS = P * (dP - delta)
            eP = torch.where(seen, (u + F) * P + z, 0.0)
            mag = G.abs() @ V.abs().T + (G.abs() * O.abs()).sum(1, keepdim=True)
            eS = torch.where(seen, u * dS.abs() + z + P * u * (G * O).abs().sum(1, keepdim=True) + F * P * mag, 0.0)
            val["out"][b, h], val["dq"][b, h] = O, scale * dS @ K
            tol["out"][b, h], tol["dq"][b, h] = eP @ V.abs(), scale * eS @ K.abs()
            val["dk"][b, c] += scale * dS.T @ Q
            val["dv"][b, c] += P.T @ G
            tol["dk"][b, c] += scale * eS.T @ Q.abs()
            tol["dv"][b, c] += eP.T @ G.abs()
    full = {n: (val[n], tol[n] * (1 + u) + u * val[n].abs() + (z if z else 0.0)) for n in names}
    full["lse"] = (lse, F * (1 + lse.abs()))
    return full


def tensors(B, H, Hkv, Sq, Sk, d, dtype, layout="bhsd", seed=1):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def new(heads, rows):
        shape = (B, rows, heads, d) if layout == "bshd" else (B, heads, rows, d)
        t = torch.randn(shape, generator=gen, device="cuda").to(dtype)
        return t.transpose(1, 2) if layout == "bshd" else t

    return new(H, Sq), new(Hkv, Sk), new(Hkv, Sk), new(H, Sq)


def int32(values):
    return None if values is None else torch.tensor(values, dtype=torch.int32, device="cuda")


def check(got, want, what):
    value, bound = want
    got = got.detach().cpu().double()
    assert got.shape == value.shape
    same = (got == value) | (torch.isfinite(got) & ((got - value).abs() <= bound))
    assert bool(same.all()), f"{what}: {int((~same).sum())} of {same.numel()} off, worst {float(((got - value).abs() - bound)[~same].max())} over its bound"


CASES = [
    # B, H, Hkv, Sq, Sk, d, window, n_sink, offsets, lengths, layout
    (1, 1, 1, 1, 1, 64, 0, 0, None, None, "bhsd"),
    (1, 2, 1, 1, 300, 128, 100, 4, None, None, "bhsd"),               # a single token
    (2, 4, 2, 128, 128, 64, 16, 4, None, None, "bhsd"),
    (1, 2, 1, 200, 200, 80, 64, 8, None, None, "bshd"),
    (2, 3, 3, 333, 333, 128, 100, 130, None, [333, 17], "bhsd"),      # sinks past a tile and past the window
    (3, 4, 1, 65, 300, 96, 70, 3, [235, 100, -20], [300, 120, 30], "bhsd"),
    (1, 2, 2, 257, 129, 64, 0, 0, None, None, "bhsd"),                # more queries than keys: the first do not exist
    (3, 2, 1, 150, 150, 32, 33, 1, None, [0, 1, 150], "bshd"),        # an empty sequence
    (1, 2, 2, 190, 190, 8, 1, 0, None, None, "bhsd"),                 # every query sees itself alone
    (1, 2, 2, 190, 190, 128, 1, 1, None, None, "bhsd"),
    (1, 2, 1, 130, 130, 64, 500, 400, None, None, "bhsd"),            # window and sinks past the sequence
    (1, 8, 1, 1100, 1100, 128, 300, 2, None, None, "bhsd"),           # key tiles whose queries are cut into parts
    (1, 8, 1, 1500, 1500, 64, 0, 0, None, [1400], "bshd"),
    (2, 2, 2, 100, 1000, 128, 64, 64, [900, 0], [1000, 100], "bhsd"),  # keys that no query sees
    (2, 2, 1, 40, 500, 64, 50, 20, [500, -40], [500, 500], "bhsd"),   # all queries outside
    # more than 8192 queries, whose dS is multiplied rounded
    (9, 8, 2, 240, 240, 64, 50, 4, None, [240, 1, 0, 100, 129, 64, 239, 33, 200], "bshd"),
    (9, 8, 8, 240, 240, 32, 0, 0, None, None, "bhsd"),
    (9, 8, 1, 240, 250, 80, 16, 1, [10, 0, -100, 10, 10, 200, 5, 10, 10], [250, 240, 250, 250, 130, 250, 128, 10, 250], "bhsd"),
    (9, 8, 4, 240, 240, 128, 100, 130, None, None, "bshd"),
    (1, 16, 1, 1100, 1100, 128, 300, 2, None, None, "bhsd"),          # and key tiles cut into parts
]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "x".join(str(x) for x in c[:8]))
def test_forward_and_backward_are_the_formulas(case, dtype):
    B, H, Hkv, Sq, Sk, d, window, n_sink, offsets, lengths, layout = case
    q, k, v, g = tensors(B, H, Hkv, Sq, Sk, d, dtype, layout)
    want = reference(q, k, v, g, window, n_sink, offsets, lengths, 0.0)
    for t in (q, k, v):
        t.requires_grad_()
    out = smha.sink_attention(q, k, v, window, n_sink, offsets=int32(offsets), lengths=int32(lengths))
    grads = torch.autograd.grad(out, (q, k, v), g)
    for name, got in zip(("out", "dq", "dk", "dv"), (out, *grads)):
        check(got, want[name], name)
    with torch.no_grad():
        alone = torch.empty_like(out)
        lse = torch.empty(B, H, Sq, device="cuda")
        smha.smha_sink_forward(q, k, v, alone, lse, window, n_sink, int32(offsets), int32(lengths))
        assert torch.equal(alone, out)
        assert torch.equal(smha.sink_attention(q, k, v, window, n_sink, offsets=int32(offsets), lengths=int32(lengths)), out)
    check(lse, want["lse"], "lse")


@pytest.mark.gpu
def test_the_way_through_python_is_the_native_one(monkeypatch):
    """The calls that the native path leaves to Python: the same bits, gradients among them."""
    from paper_2506_06095_amd import sink
    q, k, v, g = tensors(2, 4, 2, 150, 150, 64, torch.bfloat16, "bshd")
    n = int32([150, 70])

    def run():
        x = [t.detach().requires_grad_() for t in (q, k, v)]
        out = smha.sink_attention(*x, 40, 3, lengths=n)
        with torch.no_grad():
            assert torch.equal(smha.sink_attention(*x, 40, 3, lengths=n), out)
        return (out, *torch.autograd.grad(out, x, g))

    native = run()
    assert type(native[0].grad_fn).__name__ != "_SinkAttentionBackward"
    monkeypatch.setattr(sink, "_call", lambda *args: None)
    general = run()
    assert type(general[0].grad_fn).__name__ == "_SinkAttentionBackward"
    assert all(torch.equal(a, b) for a, b in zip(native, general))


@pytest.mark.gpu
@pytest.mark.parametrize("native", [True, False])
def test_gradients_for_some_inputs_and_no_second_derivative(monkeypatch, native):
    from paper_2506_06095_amd import sink
    if not native:
        monkeypatch.setattr(sink, "_call", lambda *args: None)
    q, k, v, g = tensors(1, 2, 2, 64, 64, 64, torch.float16)
    x = [t.detach().requires_grad_() for t in (q, k, v)]
    want = torch.autograd.grad(smha.sink_attention(*x, 16, 1), x, g)
    only_k = k.detach().requires_grad_()
    (dk,) = torch.autograd.grad(smha.sink_attention(q, only_k, v, 16, 1), (only_k,), g)
    assert torch.equal(dk, want[1])
    dq, dk, dv = torch.autograd.grad(smha.sink_attention(*x, 16, 1), x, g, create_graph=True)
    assert torch.equal(dq, want[0]) and torch.equal(dv, want[2])
    with pytest.raises(RuntimeError, match="twice" if native else "does not require grad"):
        dq.float().sum().backward()


@pytest.mark.gpu
@pytest.mark.parametrize("native", [True, False])
def test_the_graph_of_a_call(monkeypatch, native):
    """What autograd's own operators do: one backward pass unless it is kept, hooks of saved tensors, recomputation, nothing left behind, no forward mode."""
    from paper_2506_06095_amd import sink
    if not native:
        monkeypatch.setattr(sink, "_call", lambda *args: None)
    q, k, v, g = tensors(1, 2, 2, 64, 64, 64, torch.float16)
    n = int32([50])
    x = [t.detach().requires_grad_() for t in (q, k, v)]

    def call():
        return smha.sink_attention(*x, 16, 1, lengths=n)

    out = call()
    first = torch.autograd.grad(out, x, g, retain_graph=True)
    assert all(torch.equal(a, b) for a, b in zip(first, torch.autograd.grad(out, x, g)))
    with pytest.raises(RuntimeError, match="second time"):
        torch.autograd.grad(out, x, g)
    seen = []
    with torch.autograd.graph.saved_tensors_hooks(lambda t: (seen.append(t.shape), t.cpu())[1], lambda t: t.cuda()):
        out = call()
    assert len(seen) >= 5
    assert all(torch.equal(a, b) for a, b in zip(first, torch.autograd.grad(out, x, g)))
    again = torch.utils.checkpoint.checkpoint(lambda *y: smha.sink_attention(*y, 16, 1, lengths=n) * 1, *x, use_reentrant=False)
    assert all(torch.equal(a, b) for a, b in zip(first, torch.autograd.grad(again, x, g)))
    (dk,) = torch.autograd.grad(call(), (x[1],), g)
    assert torch.equal(dk, first[1])
    out = call()
    out.backward(g)
    out = call()
    out.backward(g)
    assert all(torch.equal(t.grad, d + d) for t, d in zip(x, first))
    del out, again
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    for _ in range(3):
        call()  # (a graph that nothing goes back through)
        torch.autograd.grad(call(), x, g)
    assert torch.cuda.memory_allocated() == before
    with torch.autograd.forward_ad.dual_level(), pytest.raises((RuntimeError, NotImplementedError)):
        smha.sink_attention(torch.autograd.forward_ad.make_dual(x[0], g), k, v, 16, 1)


@pytest.mark.gpu
def test_inputs_changed_before_the_backward_pass_are_noticed():
    q, k, v, g = tensors(1, 2, 2, 64, 64, 64, torch.float16)
    q.requires_grad_()
    n = int32([50])
    out = smha.sink_attention(q, k, v, 16, 1, lengths=n)
    n += 1
    with pytest.raises(RuntimeError, match="inplace"):
        out.backward(g)


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
def test_what_does_not_exist_may_hold_anything(d):
    """NaN and infinities in keys past the length, in keys that no query sees and in queries that do not exist change nothing."""
    q, k, v, g = tensors(2, 4, 2, 200, 400, d, torch.float16)
    offsets, lengths, window, n_sink = [180, -30], [370, 150], 40, 5
    args = dict(window=window, n_sink=n_sink, offsets=int32(offsets), lengths=int32(lengths))

    def run(q, k, v, g):
        q, k, v = (t.detach().requires_grad_() for t in (q, k, v))
        out = smha.sink_attention(q, k, v, **args)
        return (out, *torch.autograd.grad(out, (q, k, v), g))

    clean = run(q, k, v, g)
    q2, k2, v2, g2 = (t.clone() for t in (q, k, v, g))
    for b in range(2):
        seen = visible(200, 400, offsets[b], lengths[b], window, n_sink)
        for t in (q2, g2):
            t[b, :, ~seen.any(1)] = math.nan
        for t in (k2, v2):
            t[b, :, ~seen.any(0)] = math.inf
    for name, a, c in zip(("out", "dq", "dk", "dv"), run(q2, k2, v2, g2), clean):
        assert torch.equal(a, c), name


@pytest.mark.gpu
def test_gradients_are_those_of_differences():
    """Along random directions, against central differences of the formula in 64 bits (step 1e-4: their error is of the order 1e-8)."""
    q, k, v, g = tensors(1, 4, 2, 96, 96, 64, torch.bfloat16)
    window, n_sink = 20, 3
    bounds = reference(q, k, v, g, window, n_sink, None, None, 0.0)
    x = [t.detach().requires_grad_() for t in (q, k, v)]
    grads = torch.autograd.grad(smha.sink_attention(*x, window, n_sink), x, g)
    seen = visible(96, 96, 0, 96, window, n_sink)

    def value(q, k, v):
        k, v = (t.repeat_interleave(2, dim=1) for t in (k, v))
        s = (q @ k.mT / 8).masked_fill(~seen, -math.inf)
        return float((torch.softmax(s, -1) @ v * g.cpu().double()).sum())

    base = [t.detach().cpu().double() for t in (q, k, v)]
    gen = torch.Generator().manual_seed(5)
    for i, name in enumerate(("dq", "dk", "dv")):
        way = torch.randn(base[i].shape, generator=gen, dtype=torch.float64)
        plus, minus = ([t + sign * 1e-4 * way if j == i else t for j, t in enumerate(base)] for sign in (1, -1))
        slope = (value(*plus) - value(*minus)) / 2e-4
        got = float((grads[i].cpu().double() * way).sum())
        assert abs(got - slope) <= float((bounds[name][1] * way.abs()).sum()) + 1e-6 * abs(slope), name


@pytest.mark.gpu
def test_broadcast_inputs_and_gradients():
    """Keys and values expanded over the batch, and the expanded gradient of a sum: as with copies of them."""
    q, k, v, _ = tensors(3, 4, 2, 70, 70, 64, torch.float16)
    one_k, one_v = k[:1].clone().requires_grad_(), v[:1].clone().requires_grad_()
    smha.sink_attention(q, one_k.expand(3, -1, -1, -1), one_v.expand(3, -1, -1, -1), 20, 2).sum().backward()
    all_k, all_v = (t[:1].repeat(3, 1, 1, 1).requires_grad_() for t in (k, v))
    smha.sink_attention(q, all_k, all_v, 20, 2).sum().backward()
    assert torch.equal(one_k.grad, all_k.grad.sum(0, keepdim=True)) and torch.equal(one_v.grad, all_v.grad.sum(0, keepdim=True))


@pytest.mark.gpu
def test_results_do_not_depend_on_the_run():
    """Sums that are cut into parts are added in a fixed order: the same bits every time."""
    q, k, v, g = tensors(1, 8, 1, 1100, 1100, 128, torch.bfloat16)
    assert smha.smha_sink_workspace(1, 8, 1, 1100, 1100, 128, 300, 2) > 1100 * 8 * 8 * 2  # (parts of sums among it)
    for t in (q, k, v):
        t.requires_grad_()
    runs = [torch.autograd.grad(smha.sink_attention(q, k, v, 300, 2), (q, k, v), g) for _ in range(3)]
    for again in runs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(again, runs[0]))


@pytest.mark.gpu
def test_other_streams_and_a_captured_step():
    """Forward and backward on a stream of its own, and captured into a graph that is replayed with other inputs, lengths and offsets."""
    shape = (2, 4, 2, 150, 150, 64, torch.float16)
    q, k, v, g = tensors(*shape)
    n = int32([150, 90])

    def step():
        out, lse = torch.empty_like(q), torch.empty(2, 4, 150, device="cuda")
        grads = [torch.empty_like(t) for t in (q, k, v)]
        smha.smha_sink_forward(q, k, v, out, lse, 30, 4, None, n)
        smha.smha_sink_backward(q, k, v, out, lse, g, *grads, 30, 4, None, n)
        return (out, *grads)

    want = [t.clone() for t in step()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = step()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for seed, lengths in ((1, [150, 90]), (2, [1, 150]), (3, [0, 77])):
        for t, fresh in zip((q, k, v, g), tensors(*shape, seed=seed)):
            t.copy_(fresh)
        n.copy_(int32(lengths))
        eager = [t.clone() for t in step()]
        torch.cuda.synchronize()
        for t in captured:
            t.fill_(math.nan)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(captured, eager)), seed


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
def test_few_queries_have_finer_gradients(dtype):
    """The same sequences alone and among copies that make more than 8192 queries of them.  Alone, dQ and dK are off by their own rounding (1, in its
    units) and that of P in delta (0.1 of its square); among many by dS's rounding too (1 more): errors as sqrt(1.1) to sqrt(2.1), 0.72."""
    q, k, v, g = tensors(2, 12, 12, 100, 100, 64, dtype)
    want = reference(q, k, v, g, 16, 1, None, None, 0.0)

    def error(copies):
        x = [t.repeat(copies, 1, 1, 1).requires_grad_() for t in (q, k, v)]
        dq, dk, _ = torch.autograd.grad(smha.sink_attention(*x, 16, 1), x, g.repeat(copies, 1, 1, 1))
        return [float((got[:2].cpu().double() - want[name][0]).norm()) for got, name in ((dq, "dq"), (dk, "dk"))]

    assert 2 * 12 * 100 <= 8192 < 7 * 2 * 12 * 100
    for few, many in zip(error(1), error(7)):
        assert few <= 0.85 * many, (few, many)


@pytest.mark.gpu
def test_a_query_that_is_not_a_number_gives_none():
    q, k, v, g = tensors(1, 4, 2, 200, 200, 64, torch.bfloat16)
    want = reference(q, k, v, g, 50, 3, None, None, 0.0)
    q[0, 1, 77] = math.nan
    out, lse = torch.empty_like(q), torch.empty(1, 4, 200, device="cuda")
    smha.smha_sink_forward(q, k, v, out, lse, 50, 3)
    assert bool(out[0, 1, 77].isnan().all()) and bool(lse[0, 1, 77].isnan())
    out[0, 1, 77], lse[0, 1, 77] = want["out"][0][0, 1, 77].cuda(), want["lse"][0][0, 1, 77].cuda()
    check(out, want["out"], "out")
    check(lse, want["lse"], "lse")


@pytest.mark.gpu
@pytest.mark.parametrize("scale", [1e-38, 1e-20, 30.0])
def test_scales(scale):
    """Scores that are all alike, and scores of thousands.  A score, a sum of 64 products in 32 bits, is exact to 64 half steps of the products'
    magnitudes; its product with log2(e), the difference to the largest and the log-sum-exp take a few more."""
    q, k, v, _ = tensors(1, 2, 2, 90, 90, 64, torch.float16)
    out, lse = torch.empty_like(q), torch.empty(1, 2, 90, device="cuda")
    smha.smha_sink_forward(q, k, v, out, lse, 40, 2, scale=scale)
    seen = visible(90, 90, 0, 90, 40, 2)
    Q, K, V = (t.cpu().double() for t in (q, k, v))
    s = (Q @ K.mT * scale).masked_fill(~seen, -math.inf)
    P = torch.softmax(s, -1)
    e = 70 * 2.0 ** -24 * (Q.abs() @ K.abs().mT * scale).masked_fill(~seen, 0).amax(-1, keepdim=True) + F
    u = 2.0 ** -11
    assert bool(((out.cpu().double() - P @ V).abs() <= (u + 2 * e) * (P @ V.abs()) * (1 + u) + u * (P @ V).abs() + 2.0 ** -24 * V.abs().sum(-2, keepdim=True)).all())
    assert bool(((lse.cpu().double() - torch.logsumexp(s, -1)).abs() <= 2 * e[..., 0] + 2.0 ** -24 * torch.logsumexp(s, -1).abs()).all())


@pytest.mark.gpu
def test_a_large_batch_is_its_parts():
    """More key heads than the order of workgroups takes in turn at once (280 of 10 tiles each): as in ten calls.  dK and dV may be summed in other
    parts there: they differ by a rounding each, and by the sums' own, under 1e-5 of at most 1200 products of a few units."""
    B, each = 70, 7
    q, k, v, g = tensors(B, 4, 4, 1200, 1200, 64, torch.bfloat16)
    n = int32([1200 - 13 * (i % 50) for i in range(B)])
    assert each * 4 * 1200 > 8192  # (dS is rounded in both)

    def step(at):
        x = [t[at].detach().requires_grad_() for t in (q, k, v)]
        out = smha.sink_attention(*x, 100, 2, lengths=n[at].contiguous())
        return (out, *torch.autograd.grad(out, x, g[at]))

    whole = step(slice(None))
    for i in range(0, B, each):
        at = slice(i, i + each)
        for name, a, b in zip(("out", "dq", "dk", "dv"), whole, step(at)):
            if name in ("out", "dq"):
                assert torch.equal(a[at], b), (name, i)
            else:
                assert bool(((a[at].float() - b.float()).abs() <= 2 * 2.0 ** -8 * b.float().abs() + 1e-2).all()), (name, i)


@pytest.mark.gpu
def test_two_passes_at_once():
    """On two streams, whose kernels and workspaces may overlap in time."""
    inputs = [tensors(2, 8, 2, 700, 700, 128, torch.bfloat16, seed=seed) for seed in (1, 2)]

    def one(q, k, v, g):
        x = [t.detach().requires_grad_() for t in (q, k, v)]
        out = smha.sink_attention(*x, 200, 4)
        return (out, *torch.autograd.grad(out, x, g))

    want = [one(*t) for t in inputs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in inputs]
    for _ in range(3):
        got = []
        for stream, t in zip(streams, inputs):
            with torch.cuda.stream(stream):
                got.append(one(*t))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for x, y in zip(got, want) for a, b in zip(x, y))


@pytest.mark.gpu
def test_a_captured_step_of_autograd():
    shape = (2, 4, 2, 300, 300, 64, torch.bfloat16)
    q, k, v, g = tensors(*shape)
    x = [t.requires_grad_() for t in (q, k, v)]
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        out = smha.sink_attention(*x, 60, 4)
        captured = (out, *torch.autograd.grad(out, x, g))
    for seed in (1, 2, 3):
        fresh = tensors(*shape, seed=seed)
        with torch.no_grad():
            for t, new in zip((q, k, v, g), fresh):
                t.copy_(new)
        y = [t.requires_grad_() for t in fresh[:3]]
        eager = smha.sink_attention(*y, 60, 4)
        eager = (eager, *torch.autograd.grad(eager, y, fresh[3]))
        with torch.no_grad():
            for t in captured:
                t.fill_(math.nan)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(captured, eager)), seed


def test_refusals():
    """On the CPU: what the C ABI says to arguments that do not fit, before it looks for a GPU."""
    import ctypes as C
    from paper_2506_06095_amd.binding import _load
    lib = _load()
    ptr = C.c_void_p(4096)

    def forward(q=ptr, o=ptr, B=1, H=4, Hkv=2, Sq=8, Sk=8, d=64, dtype=0, strides=None, window=4, n_sink=0, out=None):
        s, out = ((C.c_int64 * 3)(*x) if x else None for x in (strides, out))
        return lib.smha_sink_forward(q, ptr, ptr, o, None, None, B, H, Hkv, Sq, Sk, d, dtype, s, None, None, out, None, None, window, n_sink, 0.0, None)

    invalid, unsupported, shape = 1, 2, 3
    assert forward(q=None) == invalid and forward(B=0) == invalid and forward(Sk=0) == invalid
    assert forward(window=-1) == invalid and forward(n_sink=-1) == invalid
    assert forward(H=5) == shape
    assert forward(d=136) == unsupported and forward(d=12) == unsupported and forward(dtype=2) == unsupported
    assert forward(q=C.c_void_p(4100)) == unsupported
    assert forward(strides=(2048, 512, 60)) == unsupported and forward(strides=(2048, 512, 56)) == unsupported and forward(strides=(-8, 512, 64)) == unsupported
    assert forward(Sk=1 << 25) == unsupported
    assert forward(B=2, out=(0, 512, 64)) == unsupported and forward(out=(2048, 0, 64)) == unsupported  # heads written in one place
    assert forward(B=1 << 12, H=1 << 12) == unsupported  # more workgroups than a launch has
    need = C.c_size_t(0)
    assert lib.smha_sink_workspace(1, 4, 2, 8, 8, 64, 4, 0, None) == invalid and lib.smha_sink_workspace(1, 4, 2, 8, 8, 64, 4, 0, C.byref(need)) == 0
    assert need.value == 2 * 4 * 128 * 4

    def backward(workspace, size, **written):
        strides = [(C.c_int64 * 3)(*written[n]) if n in written else None for n in ("q", "k", "v", "o", "do", "dq", "dk", "dv")]
        return lib.smha_sink_backward(*[ptr] * 10, 1, 4, 2, 8, 8, 64, 0, *strides, None, None, 4, 0, 0.0, workspace, size, None)

    assert backward(None, need.value) == invalid and backward(ptr, need.value - 1) == invalid
    for name in ("dq", "dk", "dv"):
        assert backward(ptr, need.value, **{name: (1024, 0, 64)}) == unsupported, name


def test_refusals_of_the_binding():
    q = torch.zeros(1, 4, 8, 64, dtype=torch.float16)
    k = torch.zeros(1, 2, 8, 64, dtype=torch.float16)
    with pytest.raises(ValueError, match="one GPU"):
        smha.sink_attention(q, k, k, 4)
    with pytest.raises(ValueError, match="multiple"):
        smha.sink_attention(q, k.repeat(1, 2, 1, 1)[:, :3], k.repeat(1, 2, 1, 1)[:, :3], 4)
    with pytest.raises(ValueError, match="float16 or bfloat16"):
        smha.sink_attention(q.float(), k.float(), k.float(), 4)
    with pytest.raises(ValueError, match="must be"):
        smha.sink_attention(q, k, k[:, :, :4], 4)


@pytest.mark.gpu
def test_refusals_of_the_binding_on_the_gpu():
    q, k, v, _ = tensors(1, 4, 2, 8, 8, 64, torch.float16)
    with pytest.raises(ValueError, match="lengths"):
        smha.sink_attention(q, k, v, 4, lengths=torch.tensor([8], device="cuda"))
    with pytest.raises(ValueError, match="offsets"):
        smha.sink_attention(q, k, v, 4, offsets=torch.zeros(2, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError, match="window"):
        smha.sink_attention(q, k, v, -1)
    with pytest.raises(smha.SmhaError):
        wide = torch.zeros(1, 4, 8, 136, dtype=torch.float16, device="cuda")
        smha.sink_attention(wide, wide, wide, 4)
    with pytest.raises(smha.SmhaError):
        smha.sink_attention(wide.requires_grad_(), wide, wide, 4)
