"""Attention on a cache (window and sinks, shared prefix, accounts of attention received) against the formulas in 64 bits, eviction
against a plain selection, exactly; both together as a serving loop runs them; and refusals.

Tolerance of an output: u |O| (its rounding) + sum_j (u P + z) |V| (the probabilities' rounding to the inputs' type) + F sum_j P |V| with u half a
step of the type, z half the smallest step of binary16 and F = 2e-5 for sums and exponentials in 32 bits (scores stay below 60, whose
exponents are rounded by 60 log2(e) 2^-24 = 5e-6).  Weights: F of what was added, and the rounding of the sum.
"""
import math

import pytest

torch = pytest.importorskip("torch")

import paper_2506_06095_amd as smha  # noqa: E402

F = 2e-5


def reference(q, k, v, lengths, window=0, n_sink=0, prefix=None, scale=0.0):
    """(out, its bound, attention received [B,Hkv,Sk]) in 64 bits on the CPU."""
    (B, H, T, d), (Hkv, Sk) = q.shape, k.shape[1:3]
    u, z = torch.finfo(q.dtype).eps / 2, 2.0 ** -25 if q.dtype == torch.float16 else 0.0
    scale = scale if scale > 0 else d ** -0.5
    q, k, v = (t.cpu().double() for t in (q, k, v))
    out, tol, got = torch.zeros_like(q), torch.zeros_like(q), torch.zeros(B, Hkv, Sk, dtype=torch.float64)
    for b in range(B):
        n = min(max(lengths[b], 0), Sk)
        pos = torch.arange(T)[:, None] + n - T
        j = torch.arange(n)[None, :]
        seen = (j <= pos) & (pos >= 0)
        if window:
            seen &= (pos - j < window) | (j < n_sink)
        used = seen.any(0)
        for h in range(H):
            c = h * Hkv // H
            K, V = (torch.where(used[:, None], t[b, c, :n], 0.0) for t in (k, v))
            see = seen
            if prefix is not None:
                K, V = (torch.cat([p[c].cpu().double(), t]) for p, t in zip(prefix, (K, V)))
                see = torch.cat([(pos >= 0).expand(T, prefix[0].shape[1]), seen], 1)
            s = (q[b, h] @ K.T * scale).masked_fill(~see, -math.inf)
            P = torch.where(see, torch.exp(s - torch.logsumexp(s, 1).nan_to_num(neginf=0.0)[:, None]), 0.0)
            out[b, h] = P @ V
            tol[b, h] = torch.where(see, (u + F) * P + z, 0.0) @ V.abs()
            got[b, c, :n] += P[:, P.shape[1] - n:].sum(0)
    return out, tol * (1 + u) + u * out.abs() + z, got


def make(B, H, Hkv, T, Sk, d, dtype=torch.float16, layout="bhsd", P=0, seed=1):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def new(heads, rows):
        shape = (B, rows, heads, d) if layout == "bshd" else (B, heads, rows, d)
        t = torch.randn(shape, generator=gen, device="cuda").to(dtype)
        return t.transpose(1, 2) if layout == "bshd" else t

    prefix = tuple(torch.randn(Hkv, P, d, generator=gen, device="cuda").to(dtype) for _ in range(2)) if P else None
    return new(H, T), new(Hkv, Sk), new(Hkv, Sk), prefix


def int32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def check(got, want, bound, what):
    got = got.detach().cpu().double()
    ok = torch.isfinite(got) & ((got - want).abs() <= bound)
    assert got.shape == want.shape and bool(ok.all()), f"{what}: {int((~ok).sum())} of {ok.numel()} off, worst {float(((got - want).abs() - bound).max())}"


CASES = [
    # B, H, Hkv, T, Sk, d, window, n_sink, P, lengths, layout
    (1, 1, 1, 1, 1, 64, 0, 0, 0, [1], "bhsd"),
    (1, 8, 2, 1, 256, 64, 64, 4, 0, [256], "bhsd"),
    (3, 4, 4, 1, 100, 128, 0, 0, 0, [0, 1, 100], "bshd"),               # an empty sequence, one key
    (2, 6, 2, 3, 333, 80, 50, 7, 0, [333, 2], "bhsd"),                  # fewer keys than tokens
    (2, 16, 2, 5, 700, 128, 100, 40, 0, [699, 130], "bshd"),            # 40 rows on a key head
    (2, 16, 1, 4, 97, 32, 0, 0, 0, [97, 33], "bhsd"),                   # 64 rows
    (1, 16, 2, 40, 120, 64, 60, 3, 0, [119], "bhsd"),                   # 320 rows
    (1, 4, 1, 1, 20000, 128, 0, 0, 0, [19999], "bhsd"),                 # many segments
    (2, 4, 2, 1, 9000, 64, 4096, 130, 0, [9000, 8999], "bhsd"),
    (70, 2, 1, 1, 64, 8, 0, 0, 0, [(7 * i) % 65 for i in range(70)], "bhsd"),   # more sequences than lanes
    (150, 4, 2, 2, 300, 64, 33, 2, 0, [(31 * i) % 301 for i in range(150)], "bhsd"),
    (4, 12, 12, 1, 96, 64, 0, 0, 333, [96, 20, 1, 50], "bhsd"),
    (3, 8, 2, 2, 40, 128, 0, 0, 1, [40, 1, 0], "bshd"),                 # sequences whose first token does not exist
    (40, 8, 2, 1, 70, 128, 0, 0, 5000, [(9 * i) % 71 for i in range(40)], "bhsd"),  # 160 rows on a prefix head
    (17, 8, 1, 1, 30, 64, 0, 0, 100, list(range(1, 18)), "bhsd"),
    (17, 8, 1, 1, 30, 64, 0, 0, 1000, list(range(1, 18)), "bhsd"),      # 136 rows: a tile of 128 and one of 8
    (70, 2, 1, 1, 2000, 64, 0, 0, 0, [(29 * i) % 2001 for i in range(70)], "bhsd"),
    (70, 4, 4, 1, 1400, 128, 0, 0, 0, [(1400 - 21 * i) for i in range(67)] + [0, 1, 2], "bshd"),   # 280 groups of up to 44 tiles, whole
    (20, 8, 2, 3, 50, 128, 0, 0, 64, [(3 * i) % 7 for i in range(20)], "bshd"),   # of which many do not exist
    (5, 12, 1, 1, 40, 96, 0, 0, 65, [40, 1, 2, 3, 40], "bhsd"),         # 60 rows, a key past two tiles of 32
    (1, 2, 2, 1, 5, 96, 0, 0, 31, [5], "bhsd"),
    (2, 2, 1, 1, 50, 64, 1, 0, 0, [50, 49], "bhsd"),                    # a window of one key
]


@pytest.mark.gpu
@pytest.mark.parametrize("weigh", [False, True], ids=["", "weights"])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "x".join(str(x) for x in c[:9]))
def test_attention_is_the_formula(case, dtype, weigh):
    B, H, Hkv, T, Sk, d, window, n_sink, P, lengths, layout = case
    q, k, v, prefix = make(B, H, Hkv, T, Sk, d, dtype, layout, P)
    want, bound, received = reference(q, k, v, lengths, window, n_sink, prefix)
    before = torch.rand(B, Hkv, Sk, device="cuda")
    weights = before.clone() if weigh else None
    out = smha.cache_attention(q, k, v, int32(lengths), window=window, n_sink=n_sink, prefix=prefix, weights=weights)
    check(out, want, bound, "output")
    if weigh:
        sum_ = before.cpu().double() + received
        check(weights, sum_, F * received + 2.0 ** -24 * sum_, "weights")
        untouched = received == 0
        assert torch.equal(weights.cpu()[untouched], before.cpu()[untouched])
    again = torch.full_like(out, math.nan)
    weights = before.clone() if weigh else None
    assert smha.cache_attention(q, k, v, int32(lengths), window=window, n_sink=n_sink, prefix=prefix, weights=weights, out=again) is again
    assert torch.equal(again, out)


@pytest.mark.gpu
def test_what_is_not_seen_may_hold_anything():
    q, k, v, _ = make(2, 8, 2, 2, 600, 128)
    lengths, window, n_sink = [555, 1], 100, 5
    want = smha.cache_attention(q, k, v, int32(lengths), window=window, n_sink=n_sink)
    want_weighed = smha.cache_attention(q, k, v, int32(lengths), window=window, n_sink=n_sink, weights=torch.zeros(2, 2, 600, device="cuda"))
    for t in (k, v):
        t[0, :, 555:] = math.nan
        t[0, :, 5:455 - 1] = math.inf
        t[1, :, 1:] = math.nan
    weights = torch.zeros(2, 2, 600, device="cuda")
    assert torch.equal(smha.cache_attention(q, k, v, int32(lengths), window=window, n_sink=n_sink), want)
    assert torch.equal(smha.cache_attention(q, k, v, int32(lengths), window=window, n_sink=n_sink, weights=weights), want_weighed)
    # (sequence 1's first token does not exist: its 8 queries are one token's)
    assert abs(float(weights[0].sum()) - 16) < 1e-3 and abs(float(weights[1].sum()) - 8) < 1e-3
    assert bool((weights[0, :, 5:454] == 0).all()) and bool((weights[:, :, 555:] == 0).all())


@pytest.mark.gpu
@pytest.mark.parametrize("Sk, P", [(64, 0), (64, 70), (3000, 0), (50, 5000)])   # direct, direct with a prefix, cut, wide
def test_a_token_that_is_not_a_number_gives_none(Sk, P):
    q, k, v, prefix = make(12, 8, 1, 1, Sk, 64, P=P)
    n = int32([Sk] * 12)
    want, bound, _ = reference(q, k, v, n.tolist(), 0, 0, prefix)
    q[3, 5] = math.nan
    weights = torch.zeros(12, 1, Sk, device="cuda")
    out = smha.cache_attention(q, k, v, n, prefix=prefix)
    weighed = smha.cache_attention(q, k, v, n, prefix=prefix, weights=weights)
    assert bool(weights[3].isnan().all()) and not weights[:3].isnan().any() and not weights[4:].isnan().any()
    for got in (out, weighed):
        assert bool(got[3, 5].isnan().all())
        got[3, 5] = want[3, 5].to(got)
        check(got, want, bound, "others")


@pytest.mark.gpu
def test_autograd_notices_a_cache_that_was_written():
    """What was saved of keys that an eviction moved, or of an account, is not used for gradients."""
    q, k, v, _ = make(2, 4, 2, 1, 40, 64)
    w, pos, n = torch.rand(2, 2, 40, device="cuda"), torch.arange(40, dtype=torch.int32, device="cuda").expand(2, 2, 40).contiguous(), int32([40, 30])
    for write in (lambda: smha.cache_evict(k, v, w, pos, n, 20), lambda: smha.cache_evict(k, v, w, pos, n, 20, out=(w, pos, n))):
        x = q.detach().requires_grad_()
        out = smha.sink_attention(x, k, v, 10, 2)
        write()
        with pytest.raises(RuntimeError, match="inplace"):
            out.float().sum().backward()
    x = torch.ones(2, 2, 40, device="cuda", requires_grad=True)
    product = (x * w).sum()
    smha.cache_attention(q, k, v, n, weights=w)
    with pytest.raises(RuntimeError, match="inplace"):
        product.backward()
    with torch.inference_mode():
        a, b, c, _ = make(1, 4, 2, 1, 40, 64)
        smha.cache_attention(a, b, c, int32([40]), weights=torch.zeros(1, 2, 40, device="cuda"))
        smha.cache_evict(b, c, torch.zeros(1, 2, 40, device="cuda"), torch.zeros(1, 2, 40, dtype=torch.int32, device="cuda"), int32([40]), 20)


@pytest.mark.gpu
def test_two_calls_at_once():
    """On two streams, whose kernels and workspaces may overlap in time."""
    calls = [make(6, 16, 4, 1, 3000, 128, dtype=torch.bfloat16, seed=seed, P=0) for seed in (1, 2)]
    n = int32([3000, 10, 2999, 1500, 0, 700])

    def one(q, k, v, _):
        w = torch.zeros(6, 4, 3000, device="cuda")
        return smha.cache_attention(q, k, v, n, weights=w), w

    want = [one(*c) for c in calls]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in calls]
    for _ in range(3):
        got = []
        for stream, c in zip(streams, calls):
            with torch.cuda.stream(stream):
                got.append(one(*c))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for x, y in zip(got, want) for a, b in zip(x, y))


@pytest.mark.gpu
def test_one_token_is_the_last_query_of_a_whole_pass():
    """Token by token on a growing cache as sink_attention on the whole sequence (both within their bounds of the same formula)."""
    S, window, n_sink = 150, 40, 3
    q, k, v, _ = make(2, 4, 2, S, S, 64, torch.bfloat16)
    whole = smha.sink_attention(q, k, v, window, n_sink)
    for n in (1, 2, 40, 41, 44, 100, 150):
        token = q[:, :, n - 1:n]
        want, bound, _ = reference(token, k, v, [n, n], window, n_sink)
        got = smha.cache_attention(token, k, v, int32([n, n]), window=window, n_sink=n_sink)
        check(got, want, bound, f"token {n}")
        check(whole[:, :, n - 1:n], want, bound, f"query {n}")


@pytest.mark.gpu
def test_strides_streams_and_a_captured_call():
    """Caches that are slices of larger ones, a stream of its own, and a captured call that follows the lengths."""
    q, k, v, prefix = make(3, 8, 2, 1, 300, 64, P=100)
    big_k, big_v = (torch.full((3, 2, 400, 72), math.nan, dtype=torch.float16, device="cuda") for _ in range(2))
    big_k[:, :, 50:350, :64], big_v[:, :, 50:350, :64] = k, v
    pk, pv = (torch.stack([t, t], 2)[:, :, 0] for t in prefix)
    wide = torch.zeros(3, 2, 320, device="cuda")
    n = int32([300, 7, 128])
    plain_w = torch.zeros(3, 2, 300, device="cuda")
    want = smha.cache_attention(q, k, v, n, prefix=prefix, weights=plain_w)
    got = smha.cache_attention(q, big_k[:, :, 50:350, :64], big_v[:, :, 50:350, :64], n, prefix=(pk, pv), weights=wide[:, :, 10:310])
    assert torch.equal(got, want) and torch.equal(wide[:, :, 10:310], plain_w) and not wide[:, :, :10].any() and not wide[:, :, 310:].any()
    plain = smha.cache_attention(q, k, v, n, prefix=prefix)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = smha.cache_attention(q, k, v, n, prefix=prefix, stream=side)
    side.synchronize()
    assert torch.equal(got, plain)
    graph = torch.cuda.CUDAGraph()
    weights = torch.zeros(3, 2, 300, device="cuda")
    with torch.cuda.graph(graph):
        out = smha.cache_attention(q, k, v, n, prefix=prefix, weights=weights)
    for lengths in ([300, 7, 128], [1, 0, 300], [64, 65, 33]):
        n.copy_(int32(lengths))
        q.copy_(torch.randn_like(q))
        expect = torch.zeros_like(weights)
        eager = smha.cache_attention(q, k, v, n, prefix=prefix, weights=expect)
        weights.zero_()
        out.fill_(math.nan)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager) and torch.equal(weights, expect), lengths


@pytest.mark.gpu
def test_the_way_through_python_is_the_native_one(monkeypatch):
    """The calls that the native path leaves to Python: the same bits."""
    from paper_2506_06095_amd import cache
    q, k, v, prefix = make(3, 8, 2, 2, 700, 64, layout="bshd", P=300)
    n = int32([700, 1, 333])

    def run():
        w = torch.zeros(3, 2, 700, device="cuda")
        kk, vv = k.clone(), v.clone()
        pos = torch.arange(700, dtype=torch.int32, device="cuda").expand(3, 2, 700).contiguous()
        out = smha.cache_attention(q, kk, vv, n, prefix=prefix, weights=w)
        near = smha.cache_attention(q, kk, vv, n, window=50, n_sink=4)
        return (out, near, *smha.cache_evict(kk, vv, w, pos, n, 200, 16), kk, vv)

    native = run()
    monkeypatch.setattr(cache, "_attention", lambda *args: None)
    monkeypatch.setattr(cache, "_evict", lambda *args: None)
    assert all(torch.equal(a, b) for a, b in zip(native, run()))


@pytest.mark.gpu
def test_a_cache_past_32_bits():
    """Keys and values of more than 4 GiB in all, 1 GiB a head, and accounts to match: the last sequence's last head, whose every offset is past 2^31
    elements, against the formula on the GPU in 64 bits."""
    B, Hkv, Sk, d = 2, 2, 8 << 20, 64
    gen = torch.Generator(device="cuda").manual_seed(4)
    k, v = (torch.empty(B, Hkv, Sk, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    k[1, 1].normal_(generator=gen)
    v[1, 1].normal_(generator=gen)
    q = torch.zeros(B, 4, 1, d, dtype=torch.bfloat16, device="cuda")
    q[1, 2:] = torch.randn(2, 1, d, generator=gen, device="cuda").bfloat16()
    weights = torch.zeros(B, Hkv, Sk, device="cuda")
    lengths = [1, Sk - 3]
    k[0, :, 0] = v[0, :, 0] = k[1, 0] = v[1, 0] = 0
    out = smha.cache_attention(q, k, v, int32(lengths), weights=weights)
    u, received = 2.0 ** -8, torch.zeros(Sk, dtype=torch.float64, device="cuda")
    for h in (2, 3):
        K, V = k[1, 1, :lengths[1]].double(), v[1, 1, :lengths[1]].double()
        p = torch.softmax(K @ q[1, h, 0].double() / 8, 0)
        want, bound = p @ V, (u + F) * (p @ V.abs())
        assert bool(((out[1, h, 0].double() - want).abs() <= bound * (1 + u) + u * want.abs()).all())
        received[:lengths[1]] += p
        del K, V
    # (the log-sum-exp of eight million terms, in 32 bits: each of the 4096 lanes' sums of some thousand is off by at most as many half steps)
    assert bool(((weights[1, 1].double() - received).abs() <= (F + 4096 * 2.0 ** -24) * received).all())
    w2, pos, n = smha.cache_evict(k, v, weights, torch.arange(Sk, dtype=torch.int32, device="cuda").expand(B, Hkv, Sk).contiguous(), int32(lengths), 1000, 0)
    kept = torch.sort(weights[1, 1, :lengths[1]], descending=True, stable=True).indices[:1000].sort().values
    assert n.tolist() == [1, 1000] and torch.equal(pos[1, 1, :1000].long().sort().values, kept) and torch.equal(w2[1, 1, :1000], weights[1, 1][pos[1, 1, :1000].long()])


# --- eviction

def plain_evict(k, v, w, pos, lengths, budget, recent):
    """Head by head; k, v, w, pos on the CPU, changed in place."""
    B, Hkv, Sk = w.shape
    for b in range(B):
        n = min(max(int(lengths[b]), 0), Sk)
        end = min(n, budget)
        for h in range(Hkv):
            if n > budget:
                newest = int(pos[b, h, :n].max())

                def rank(j):
                    x = float(w[b, h, j])
                    x = math.inf if int(pos[b, h, j]) > newest - recent else -math.inf if math.isnan(x) else x
                    return (-x, j)

                kept = sorted(sorted(range(n), key=rank)[:end])
                stays = set(kept)
                to = [j for j in range(end) if j not in stays]
                at = [j for j in kept if j >= end]
                for t in (k, v, w, pos):
                    t[b, h, to] = t[b, h, at]
            w[b, h, end:], pos[b, h, end:] = 0, -1
    return torch.tensor([min(max(int(n), 0), Sk, budget) for n in lengths], dtype=torch.int32)


def evict_inputs(B, Hkv, Sk, d, seed=1, dtype=torch.float16, values="spread"):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    k, v = (torch.randn(B, Hkv, Sk, d, generator=gen, device="cuda").to(dtype) for _ in range(2))
    w = torch.randn(B, Hkv, Sk, generator=gen, device="cuda").exp()
    if values == "ties":
        w = torch.randint(3, w.shape, generator=gen, device="cuda").float() - 1
        w[w == 0] *= -1  # (both zeros)
    if values == "odd":
        w -= 1
        w[..., ::7], w[..., 1::11], w[..., 2::13] = math.nan, math.inf, -math.inf
    pos = torch.rand(B, Hkv, Sk, generator=gen, device="cuda").argsort(-1).to(torch.int32)
    return k, v, w, pos


EVICT = [
    # B, Hkv, Sk, d, lengths, budget, recent, values
    (1, 1, 1, 8, [1], 1, 0, "spread"),
    (2, 2, 100, 64, [100, 37], 37, 5, "spread"),
    (3, 2, 257, 128, [257, 0, 256], 256, 300, "ties"),       # more recent keys than the budget
    (2, 3, 513, 80, [513, 300], 64, 0, "ties"),
    (2, 2, 1300, 64, [1300, 1025], 1, 1, "odd"),
    (2, 2, 4097, 32, [4097, 4096], 4000, 64, "odd"),
    (1, 2, 10000, 64, [9999], 2048, 128, "ties"),
    (1, 2, 20000, 16, [20000], 17000, 20, "spread"),
    (1, 1, 40000, 8, [39999], 20000, 7, "ties"),             # more slots than a workgroup holds in registers
    (1, 2, 300, 64, [300], 1000, 3, "spread"),               # nothing to do
    (3, 1, 130, 64, [500, -7, 130], 100, 10, "spread"),      # lengths outside the cache
    (2, 2, 1024, 72, [1024, 700], 512, 30, "spread"),        # as many moves as one workgroup makes, and one more
    (1, 3, 1026, 64, [1026], 513, 0, "ties"),
    (1, 2, 40000, 8, [40000], 39500, 7, "spread"),
]


@pytest.mark.gpu
@pytest.mark.parametrize("in_place", [0, 3, 2], ids=["", "in_place", "weights_and_positions_in_place"])
@pytest.mark.parametrize("case", EVICT, ids=lambda c: "x".join(str(x) for x in (*c[:4], *c[5:])))
def test_eviction_is_the_plain_selection(case, in_place):
    B, Hkv, Sk, d, lengths, budget, recent, values = case
    k, v, w, pos = evict_inputs(B, Hkv, Sk, d, values=values)
    n = int32(lengths)
    want = [t.cpu().clone() for t in (k, v, w, pos)]
    want.append(plain_evict(*want, lengths, budget, recent))
    if n.max() > Sk or n.min() < 0:
        assert want[-1].tolist() == [min(max(x, 0), Sk, budget) for x in lengths]
    given = [t.clone() for t in (w, pos, n)]
    to = (w, pos, n if in_place == 3 else torch.full_like(n, -5)) if in_place else None
    out = smha.cache_evict(k, v, w, pos, n, budget, recent, out=to)
    if in_place:
        assert all(a is b for a, b in zip(out, to))
    assert all(torch.equal(a.view(torch.int32), b.view(torch.int32)) for a, b in list(zip((w, pos, n), given))[in_place:])
    for name, a, b in zip(("k", "v", "weights", "positions", "lengths"), (k, v, *out), want):
        a = a.cpu()
        same = (a == b) | (a.isnan() & b.isnan()) if a.is_floating_point() else a == b
        assert bool(same.all()), (name, int((~same).sum()))


@pytest.mark.gpu
def test_eviction_of_a_token_major_cache_on_another_stream_and_captured():
    k, v, w, pos = evict_inputs(2, 3, 400, 64, seed=3)
    kt, vt = (t.transpose(1, 2).contiguous().transpose(1, 2) for t in (k, v))
    n = int32([400, 350])
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    first = smha.cache_evict(k, v, w, pos, n, 300, 10)
    torch.cuda.synchronize()
    second = smha.cache_evict(kt, vt, w, pos, n, 300, 10, stream=side)
    side.synchronize()
    assert torch.equal(k, kt) and torch.equal(v, vt) and all(torch.equal(a, b) for a, b in zip(first, second))
    graph = torch.cuda.CUDAGraph()
    ins = evict_inputs(2, 3, 400, 64, seed=4)
    with torch.cuda.graph(graph):
        got = smha.cache_evict(*ins, n, 300, 10)
    for seed, lengths in ((4, [400, 350]), (5, [301, 5]), (6, [0, 399])):
        n.copy_(int32(lengths))
        fresh = evict_inputs(2, 3, 400, 64, seed=seed)
        for a, b in zip(ins, fresh):
            a.copy_(b)
        eager = smha.cache_evict(*fresh, n, 300, 10)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((*ins[:2], *got), (*fresh[:2], *eager))), seed


@pytest.mark.gpu
def test_a_serving_loop():
    """Prefill, then tokens one by one with accounts kept, and evictions whenever the cache has grown by 16: every step's attention is that
    of the formula on the keys that the cache holds, every eviction the plain selection, and the last tokens are always there."""
    B, H, Hkv, d, budget, slack, recent = 2, 8, 2, 64, 48, 16, 8
    room, prompt = budget + slack, 50
    gen = torch.Generator(device="cuda").manual_seed(9)

    def new(heads, rows):
        return torch.randn(B, heads, rows, d, generator=gen, device="cuda").half()

    k, v = torch.zeros(B, Hkv, room, d, dtype=torch.float16, device="cuda"), torch.zeros(B, Hkv, room, d, dtype=torch.float16, device="cuda")
    pk, pv = new(Hkv, prompt), new(Hkv, prompt)
    k[:, :, :prompt], v[:, :, :prompt] = pk, pv
    weights = torch.zeros(B, Hkv, room, device="cuda")
    positions = torch.full((B, Hkv, room), -1, dtype=torch.int32, device="cuda")
    positions[:, :, :prompt] = torch.arange(prompt, dtype=torch.int32, device="cuda")
    n = int32([prompt] * B)
    # the prompt's own pass, and the accounts that its last queries open
    q = new(H, prompt)
    smha.sink_attention(q, pk, pv)
    smha.cache_attention(q[:, :, -8:].contiguous(), k, v, n, weights=weights)
    assert abs(float(weights.sum()) - B * H * 8) < 1e-2
    evictions = 0
    for step in range(60):
        at = int(n[0])
        if at == room:
            want = [t.cpu().clone() for t in (k, v, weights, positions)]
            want.append(plain_evict(*want, n.tolist(), budget, recent))
            smha.cache_evict(k, v, weights, positions, n, budget, recent, out=(weights, positions, n))
            assert all(torch.equal(a.cpu(), b) for a, b in zip((k, v, weights, positions, n), want))
            at = budget
            evictions += 1
        q, nk, nv = new(H, 1), new(Hkv, 1), new(Hkv, 1)
        k[:, :, at:at + 1], v[:, :, at:at + 1] = nk, nv
        positions[:, :, at] = prompt + step
        n += 1
        before = weights.clone()
        out = smha.cache_attention(q, k, v, n, weights=weights)
        ref, bound, received = reference(q, k, v, n.tolist())
        check(out, ref, bound, f"step {step}")
        sum_ = before.cpu().double() + received
        check(weights, sum_, F * received + 2.0 ** -24 * sum_, f"weights of step {step}")
    assert evictions >= 3
    live = positions[:, :, :int(n[0])].cpu()
    assert bool((live >= 0).all()) and all(len(set(row.tolist())) == len(row) for head in live for row in head)
    assert all(set(range(prompt + 60 - recent, prompt + 60)) <= set(row.tolist()) for head in live for row in head)


def test_refusals():
    """On the CPU: what the C ABI says to arguments that do not fit, before it looks for a GPU."""
    import ctypes as C
    from paper_2506_06095_amd.binding import _load
    lib = _load()
    ptr = C.c_void_p(4096)
    invalid, unsupported, shape = 1, 2, 3

    def forward(q=ptr, lengths=ptr, pk=None, B=1, H=4, Hkv=2, T=1, Sk=8, P=0, d=64, dtype=0, ks=None, window=0, n_sink=0, ws=ptr, size=1 << 40, out=None):
        s, out = ((C.c_int64 * 3)(*x) if x else None for x in (ks, out))
        return lib.smha_cache_forward(q, ptr, ptr, pk, pk, ptr, None, lengths, B, H, Hkv, T, Sk, P, d, dtype, None, s, None, None, None, out, None, window, n_sink,
                                      0.0, ws, size, None)

    assert forward(q=None) == invalid and forward(lengths=None) == invalid and forward(Sk=4000, ws=None) == invalid
    assert forward(Sk=4000, size=1000) == invalid
    few = C.c_size_t(7)
    assert lib.smha_cache_workspace(1, 4, 2, 1, 8, 0, 64, 0, 0, 0, C.byref(few)) == 0 and few.value == 0  # (few keys: nothing to keep)
    assert forward(B=0) == invalid and forward(T=0) == invalid and forward(P=-1) == invalid and forward(P=5) == invalid and forward(window=-1) == invalid
    assert forward(H=3) == shape
    assert forward(d=136) == unsupported and forward(d=20) == unsupported and forward(dtype=2) == unsupported
    assert forward(P=5, pk=ptr, window=3) == unsupported
    assert forward(ks=(1024, 512, 32)) == unsupported and forward(ks=(1024, 512, 68)) == unsupported
    assert forward(q=C.c_void_p(4104)) == unsupported and forward(Sk=1 << 25) == unsupported

    assert forward(B=2, out=(0, 64, 64)) == unsupported and forward(out=(256, 0, 64)) == unsupported  # heads written in one place
    assert forward(B=1 << 12, H=1 << 12, Hkv=1 << 12) == unsupported  # more workgroups than a launch has

    def evict(k=ptr, B=1, Hkv=2, Sk=8, d=64, budget=4, recent=1, ks=None, size=1 << 30):
        s = (C.c_int64 * 3)(*ks) if ks else None
        return lib.smha_cache_evict(k, *[ptr] * 7, B, Hkv, Sk, d, budget, recent, s, None, ptr, size, None)

    assert evict(k=None) == invalid and evict(budget=0) == invalid and evict(recent=-1) == invalid and evict(Sk=0) == invalid and evict(size=4) == invalid
    assert evict(d=12) == unsupported and evict(B=40000) == unsupported and evict(ks=(1024, 512, 32)) == unsupported and evict(k=C.c_void_p(4104)) == unsupported
    need = C.c_size_t(0)
    assert lib.smha_cache_evict_workspace(2, 3, 100, 64, 60, 0, C.byref(need)) == 0 and need.value == 2 * 3 * (1 + 2 * 40) * 4
    assert lib.smha_cache_workspace(1, 4, 2, 1, 8, 0, 64, 0, 0, 0, None) == invalid


@pytest.mark.gpu
def test_refusals_of_the_binding():
    q, k, v, prefix = make(2, 4, 2, 1, 16, 64, P=8)
    n = int32([16, 3])
    for bad, match in (
        (lambda: smha.cache_attention(q, k, v, None), "lengths"),
        (lambda: smha.cache_attention(q, k, v, n.long()), "lengths"),
        (lambda: smha.cache_attention(q, k, v, n[:1]), "lengths"),
        (lambda: smha.cache_attention(q, k[:, :1].expand(-1, 3, -1, -1), v[:, :1].expand(-1, 3, -1, -1), n), "multiple"),
        (lambda: smha.cache_attention(q, k, v, n, prefix=(prefix[0], prefix[1][:1])), "prefix"),
        (lambda: smha.cache_attention(q, k, v, n, weights=torch.zeros(2, 2, 15, device="cuda")), "weights"),
        (lambda: smha.cache_attention(q, k, v, n, weights=torch.zeros(2, 1, 16, device="cuda").expand(2, 2, 16)), "overlap"),
        (lambda: smha.cache_attention(q.requires_grad_(), k, v, n), "gradients"),
        (lambda: smha.cache_evict(k[:1].expand(2, -1, -1, -1), v, torch.zeros(2, 2, 16, device="cuda"), torch.zeros(2, 2, 16, dtype=torch.int32, device="cuda"), n, 4), "overlap"),
        (lambda: smha.cache_evict(k, v, torch.zeros(2, 2, 16, device="cuda"), torch.zeros(2, 2, 16, device="cuda"), n, 4), "positions"),
    ):
        with pytest.raises(ValueError, match=match):
            bad()
        q.requires_grad_(False)
    with pytest.raises(smha.SmhaError):
        smha.cache_attention(q, k, v, n, prefix=prefix, window=4)
    with pytest.raises(smha.SmhaError):
        smha.cache_attention(*make(2, 4, 2, 1, 2000, 64)[:3], n, workspace=torch.empty(8, dtype=torch.uint8, device="cuda"))
