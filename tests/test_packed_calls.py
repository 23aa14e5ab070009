"""Calls on a cache held in 4 bits that are easy to get wrong around the kernels: tensors that share memory, sizes that are refused, tensors of other kinds, threads."""
import pytest

torch = pytest.importorskip("torch")

import paper_2506_06095_amd as smha  # noqa: E402

# What the C ABI says, on the CPU: status 1 invalid, 5 a HIP error (a call that was not refused and found no GPU).

BASE = 1 << 20
no_gpu = pytest.mark.skipif(torch.cuda.is_available(), reason="the addresses are not real")


def abi():
    import ctypes as C
    from paper_2506_06095_amd.binding import _load
    return C, _load()


def strides(C, s):
    return (C.c_int64 * 3)(*s) if s else None


def written(n, steps, row):
    """The first bytes of the rows of [n] with strides of `steps` bytes."""
    return {(b * steps[0] + h * steps[1] + t * steps[2] + i) for b in range(n[0]) for h in range(n[1]) for t in range(n[2]) for i in range(row)}


# 2 x 3 heads of 5 rows: strides in rows, of the keys and of the values (None: alike), and the distances in rows at which they are looked at
LAYOUTS = [
    ((15, 5, 1), None),      # packed
    ((30, 5, 1), None),      # room for other heads between sequences
    ((60, 20, 1), None),
    ((30, 10, 2), None),     # rows in turn
    ((30, 1, 6), None),      # tokens before heads, keys and values side by side
    ((5, 20, 1), None),      # heads outermost
    ((1, 2, 7), None),
    ((17, 5, 1), None),
    ((15, 5, 1), (30, 10, 2)),
    ((30, 10, 2), (30, 1, 6)),
]


@no_gpu
@pytest.mark.parametrize("call", ["write", "read"])
@pytest.mark.parametrize("layout", LAYOUTS, ids=str)
def test_two_tensors_that_are_written_must_not_share_memory(layout, call):
    """Against the rows' bytes, one by one, where both have the same strides; where they do not, calls whose tensors reach into one another are refused. Those that lie
    apart as a whole are taken, however they are laid out."""
    C, lib = abi()
    n, d = (2, 3, 5), 64
    row = 40 if call == "write" else 128  # bytes
    ks, vs = layout[0], layout[1] or layout[0]
    ksb, vsb = ([s * row for s in x] for x in (ks, vs))
    reach = [sum(s * (m - 1) for s, m in zip(x, n)) + row for x in (ksb, vsb)]
    keys, seen = written(n, ksb, row), set()
    for at in [r * row for r in range(-70, 71)] + ([4, -4, row // 2, -row // 2 - 4, reach[0] - 4, reach[0], -reach[1], 4 - reach[1]] if call == "write" else [16, -16, reach[0]]):
        if at == 0:
            continue
        values = {at + x for x in written(n, vsb, row)}
        shared = bool(keys & values) if layout[1] is None else at < reach[0] and -at < reach[1]
        k, v = C.c_void_p(BASE), C.c_void_p(BASE + at)
        if call == "write":
            got = lib.smha_packed_write(C.c_void_p(1 << 24), C.c_void_p(1 << 25), k, v, None, None, C.c_void_p(4096), None, *n[:2], 1, n[2], d, 0, None, None, strides(C, ksb), strides(C, vsb), None)
        else:
            got = lib.smha_packed_read(C.c_void_p(1 << 24), C.c_void_p(1 << 25), k, v, C.c_void_p(4096), None, *n, 9, d, 0, None, None, strides(C, [s // 2 for s in ksb]),
                                       strides(C, [s // 2 for s in vsb]), None)
        assert got == (1 if shared else 5), (at, got)
        seen.add(shared)
    assert seen == {True, False}


@no_gpu
def test_strides_of_one_row_do_not_matter():
    """Dimensions of one: whatever their strides are, packed tensors beside one another are taken."""
    C, lib = abi()
    for ks, vs in ((None, (7 * 4, 40, 40)), ((4, 4, 40), None), ((0, 0, 40), (400, 8, 400))):
        for at, want in ((40, 5), (-40, 5), (36, 1), (-36, 1)):
            got = lib.smha_packed_write(C.c_void_p(1 << 24), C.c_void_p(1 << 25), C.c_void_p(BASE), C.c_void_p(BASE + at), None, None, C.c_void_p(4096), None, 1, 1, 1, 1, 64, 0, None, None,
                                        strides(C, ks), strides(C, vs), None)
            assert got == want, (ks, vs, at)


@no_gpu
def test_values_go_to_memory_of_their_own():
    """K_values and V_values: not over one another, the cache, or new tokens, but for those that are read in the same places."""
    C, lib = abi()
    B, Hkv, T, Sk, d = 2, 3, 4, 9, 64
    size, cache = B * Hkv * T * d * 2, B * Hkv * Sk * 40
    at = {"kn": 1 << 20, "vn": 2 << 20, "k": 3 << 20, "v": 4 << 20, "kv": 5 << 20, "vv": 6 << 20}

    def write(kns=None, vns=None, **places):
        p = {n: C.c_void_p(x) for n, x in {**at, **places}.items()}
        return lib.smha_packed_write(p["kn"], p["vn"], p["k"], p["v"], p["kv"], p["vv"], C.c_void_p(4096), None, B, Hkv, T, Sk, d, 0, strides(C, kns), strides(C, vns), None, None, None)

    packed = (Hkv * T * d, T * d, d)
    assert write() == 5
    assert write(kv=at["kn"], vv=at["vn"]) == 5 and write(kns=packed, vns=packed, kv=at["kn"], vv=at["vn"]) == 5
    assert write(kv=at["vn"], vv=at["kn"]) == 5                       # (every lane has read both by then)
    assert write(kns=(T * Hkv * d, d, Hkv * d), kv=at["kn"]) == 1     # read in another order
    assert write(kns=(0, 0, 0 + d), kv=at["kn"]) == 1
    for name in ("kv", "vv"):
        assert write(**{name: at["kv" if name == "vv" else "vv"]}) == 1
        for other, bytes_ in (("kv" if name == "vv" else "vv", size), ("kn", size), ("vn", size), ("k", cache), ("v", cache)):
            for far in (16, bytes_ - 16, -16, 16 - size):
                assert write(**{name: at[other] + far}) == 1, (name, other, far)
            for far in ((bytes_ + 15) // 16 * 16, -size):
                assert write(**{name: at[other] + far}) == 5, (name, other, far)


@pytest.mark.gpu
def test_caches_in_one_tensor_and_over_one_another():
    both = torch.zeros(2, 40, 6, 80, dtype=torch.uint8, device="cuda")
    kn, vn = (torch.randn(2, 2, 3, 128, device="cuda").half() for _ in range(2))
    n = torch.tensor([40, 20], dtype=torch.int32, device="cuda")
    k, v = (both[:, :, i:i + 2].transpose(1, 2) for i in (0, 3))
    smha.packed_write(kn, vn, k, v, n)
    apart = smha.packed_cache(2, 2, 40, 128)
    smha.packed_write(kn, vn, *apart, n)
    assert torch.equal(k, apart[0]) and torch.equal(v, apart[1])
    before = both.clone()
    for v in (both[:, :, 1:3].transpose(1, 2), both[:, :, :2].transpose(1, 2)):
        for stream in (None, torch.cuda.current_stream()):
            with pytest.raises(smha.SmhaError):
                smha.packed_write(kn, vn, k, v, n, stream=stream)
    out = torch.empty(2, 3, 40, 128, dtype=torch.float16, device="cuda")
    with pytest.raises(smha.SmhaError):
        smha.packed_read(*apart, n, out=(out[:, :2], out[:, 1:]))
    assert torch.equal(both, before)


@pytest.mark.gpu
@pytest.mark.parametrize("way", ["native", "python"])
def test_sizes_are_refused_before_anything_is_allocated(way):
    """(Outputs of such calls would be gigabytes.)"""
    k, v = smha.packed_cache(2, 2, 40, 128)
    n = torch.tensor([40, 20], dtype=torch.int32, device="cuda")
    stream = torch.cuda.current_stream() if way == "python" else None
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.memory_allocated()

    def refused(call):
        with pytest.raises(smha.SmhaError) as e:
            call()
        assert e.value.status == 2 and torch.cuda.max_memory_allocated() - before < 1 << 20

    # more than 2^27 rows, of heads below 2 GiB; heads of 2 GiB; more rows than there are
    kc, vc = (t[:1, :1].expand(32, 2, 40, 80) for t in (k, v))
    many = n[:1].repeat(32)
    refused(lambda: smha.packed_read(kc, vc, many, tokens=(1 << 21) + 1, stream=stream))
    refused(lambda: smha.packed_read(k, v, n, tokens=1 << 23, stream=stream))
    refused(lambda: smha.packed_read(k, v, n, tokens=1 << 22, dtype=torch.float32, stream=stream))
    for tokens in (1 << 27, (1 << 31) - 1):
        refused(lambda: smha.packed_read(k[:1], v[:1], n[:1], tokens=tokens, stream=stream))
    wide = torch.zeros(1, 1, 1, 128, dtype=torch.float16, device="cuda")
    new = wide.expand(2, 2, 1 << 23, 128)  # (a stride of 0 between tokens is refused too)
    refused(lambda: smha.packed_write(new, new, k, v, n, values=True, stream=stream))
    q = wide.expand(2, 4, 1 << 22, 128)
    refused(lambda: smha.packed_attention(q, k, v, n, stream=stream))


@pytest.mark.gpu
def test_the_largest_read_that_is_taken():
    """2^27 rows in all, of which few are there; the same by both ways."""
    k, v = smha.packed_cache(1, 1, 40, 8)
    kn = torch.randn(1, 1, 40, 8, device="cuda").half()
    n = torch.tensor([40], dtype=torch.int32, device="cuda")
    want = smha.packed_write(kn, kn * 2, k, v, n, values=True)
    kc, vc = (t.expand(8, 1, 40, 8) for t in (k, v))
    many = n.repeat(8)
    for stream in (None, torch.cuda.current_stream()):
        got = smha.packed_read(kc, vc, many, tokens=1 << 24, stream=stream)
        for g, w in zip(got, want):
            assert g.shape == (8, 1, 1 << 24, 8) and all(torch.equal(g[b, :, :40], w[0]) for b in range(8)) and not bool(g[:, :, 40:].any())
        del got
    with pytest.raises(smha.SmhaError):
        smha.packed_read(kc, vc, many, tokens=(1 << 24) + 1)


def inputs():
    gen = torch.Generator(device="cuda").manual_seed(5)
    B, H, Hkv, T, Sk, d = 2, 8, 2, 3, 3000, 128
    kn, vn = (torch.randn(B, Hkv, Sk, d, generator=gen, device="cuda").half() for _ in range(2))
    q = torch.randn(B, H, T, d, generator=gen, device="cuda").half()
    n = torch.tensor([Sk, Sk - 100], dtype=torch.int32, device="cuda")
    k, v = smha.packed_cache(B, Hkv, Sk, d)
    smha.packed_write(kn, vn, k, v, n)
    return q, kn, vn, k, v, n


@pytest.mark.gpu
def test_tensors_of_other_kinds_and_modes():
    """Subclasses and calls under a mode, which the native way leaves to the other: the same results."""
    q, kn, vn, k, v, n = inputs()
    want = smha.packed_attention(q, k, v, n), *smha.packed_read(k, v, n), *smha.packed_write(kn, vn, k, v, n, values=True), k.clone(), v.clone()

    class Sub(torch.Tensor):
        pass

    class Mode(torch.utils._python_dispatch.TorchDispatchMode):
        def __torch_dispatch__(self, func, types, args=(), kwargs=None):
            return func(*args, **(kwargs or {}))

    def passes(*tensors):
        q, kn, vn, k, v, n = tensors
        return smha.packed_attention(q, k, v, n), *smha.packed_read(k, v, n), *smha.packed_write(kn, vn, k, v, n, values=True), k, v

    def same(got):
        assert len(got) == len(want) and all(torch.equal(a.as_subclass(torch.Tensor), b) for a, b in zip(got, want))

    same(passes(*(t.as_subclass(Sub) for t in (q, kn, vn, k, v, n))))
    k.zero_()
    v.zero_()
    smha.packed_write(kn, vn, k, v, n)
    with Mode():
        same(passes(q, kn, vn, k, v, n))
    with torch.inference_mode():
        same(passes(q, kn, vn, k, v, n))
    with pytest.raises(ValueError):
        smha.packed_attention(torch.nn.Parameter(q), k, v, n)
    with torch.no_grad():
        assert torch.equal(smha.packed_attention(torch.nn.Parameter(q), k, v, n), want[0])
    with pytest.raises(RuntimeError):
        torch.vmap(lambda t: smha.packed_attention(t, k, v, n))(q[None])


@pytest.mark.gpu
def test_threads_with_streams_of_their_own():
    import threading
    q, kn, vn, k, v, n = inputs()
    want = smha.packed_attention(q, k, v, n)
    got, failed = [None] * 4, []
    torch.cuda.synchronize()

    def work(i):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                mine = smha.packed_cache(2, 2, 3000, 128)
                for _ in range(20):
                    smha.packed_write(kn, vn, *mine, n)
                    got[i] = smha.packed_attention(q, *mine, n)
                torch.cuda.current_stream().synchronize()
        except Exception as e:  # noqa: BLE001
            failed.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed and all(torch.equal(g, want) for g in got)
