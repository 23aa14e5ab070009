"""Calls of the operators beside the plan that are easy to get wrong around the kernels: how names, gradients, layouts and sizes are taken and refused."""
import subprocess
import sys

import pytest

torch = pytest.importorskip("torch")

import paper_2506_06095_amd as smha  # noqa: E402


def test_a_name_is_looked_up_once():
    """In a fresh process: the package resolves an operator's name at its first use and then holds it."""
    code = ("import paper_2506_06095_amd as smha\n"
            "names = sorted(smha._OPERATORS)\n"
            "assert not any(n in vars(smha) for n in names)\n"
            "first = [getattr(smha, n) for n in names]\n"
            "assert all(vars(smha).get(n) is f for n, f in zip(names, first))\n"
            "try:\n    smha.no_such_operator\nexcept AttributeError:\n    pass\nelse:\n    raise SystemExit('found')\n")
    subprocess.run([sys.executable, "-c", code], check=True, cwd=smha.__path__[0] + "/..")


@pytest.mark.parametrize("when", ["at first", "when the call path is known"])
def test_a_first_call_from_two_threads(monkeypatch, when):
    """Another thread's call in the middle of the first one: it finds the native function, neither an unfinished state nor a second build."""
    import threading
    from paper_2506_06095_amd import binding
    builds = []
    monkeypatch.setattr(binding, "_native", None)
    monkeypatch.setattr(binding, "_native_module", None, raising=False)
    monkeypatch.setattr(binding._build, "extension_current", lambda: False)
    monkeypatch.setattr(binding._build, "build_extension", lambda: builds.append(threading.get_ident()))
    got, others = [], []

    def call():
        try:
            got.append(binding.native_call("sink_attention"))
        except Exception as e:  # noqa: BLE001
            got.append(e)

    def first():
        def at_line(frame, event, arg):
            if frame.f_code is binding._load_native.__code__ and not others and (when == "at first" or binding._native is not None):
                others.append(threading.Thread(target=call))
                others[0].start()
                others[0].join(0.2)  # (it may have to wait until the first is done)
            return at_line
        sys.settrace(at_line)
        call()
        sys.settrace(None)

    thread = threading.Thread(target=first)
    thread.start()
    thread.join()
    others[0].join()
    assert len(got) == 2 and all(callable(f) and f.__name__ == "sink_attention" for f in got), got
    assert len(builds) == 1


def test_the_native_functions_are_those_of_the_module_in_use(monkeypatch, tmp_path):
    """Where the native module cannot be had, calls go the general way; once it can, they are its own again."""
    from paper_2506_06095_amd import binding
    native = binding.native_call("cache_evict")
    assert native.__name__ == "cache_evict"
    with monkeypatch.context() as m:
        m.setattr(binding, "_native", None)
        m.setattr(binding._build, "EXT", str(tmp_path / "_smha_torch.so"))
        m.setenv("CXX", "false")
        with pytest.warns(RuntimeWarning, match="native call path"):
            assert binding.native_call("cache_evict")() is None
    assert binding.native_call("cache_evict") is native


# What the C ABI says, on the CPU: status 1 invalid, 2 unsupported, 3 shape.

def abi():
    import ctypes as C
    from paper_2506_06095_amd.binding import _load
    return C, _load(), C.c_void_p(4096)


def test_eviction_refuses_heads_that_lie_in_one_place():
    """Each head moves rows of its own: two that share memory would move them at once."""
    C, lib, ptr = abi()

    def evict(ks, vs=None, B=2):
        ks, vs = ((C.c_int64 * 3)(*s) if s else None for s in (ks, vs))
        return lib.smha_cache_evict(ptr, *[ptr] * 7, B, 2, 8, 64, 4, 1, ks, vs, ptr, 1 << 30, None)

    for bad in ((0, 512, 64), (1024, 0, 64), (1024, 56, 64)):
        assert evict(bad) == 2 and evict(None, bad) == 2, bad
    assert evict((0, 0, 64), B=1) == 2  # (one sequence, but two heads in one place)


# {batch, head, token} strides of 2 x 2 heads of 8 rows of 64, some of whose rows share memory though every step is wide enough for a row
OVERLAPPING = [(512, 512, 64), (1024, 448, 64), (512, 960, 64), (64, 512, 64), (128, 64, 64), (1024, 512, 1024), (1536, 128, 128)]
# and those of layouts whose rows do not: packed, heads outermost, token-major, batch within tokens, with room between, heads of a wider tensor
APART = [(1024, 512, 64), (512, 1024, 64), (1024, 64, 128), (64, 128, 256), (4096, 1024, 72), (8192, 64, 1024)]


@pytest.mark.parametrize("strides", OVERLAPPING + APART, ids=str)
def test_written_rows_must_not_overlap(strides):
    """(Without a GPU, a call that is not refused ends with status 5, a HIP error.)"""
    if torch.cuda.is_available():
        pytest.skip("the addresses are not real")
    C, lib, ptr = abi()
    s = (C.c_int64 * 3)(*strides)
    args = (2, 2, 2, 8, 8, 64, 0)
    got = [lib.smha_sink_forward(ptr, ptr, ptr, ptr, None, None, *args, None, None, None, s, None, None, 4, 0, 0.0, None)]
    for at in (5, 6, 7):  # dq, dk, dv
        st = [None] * 8
        st[at] = s
        got.append(lib.smha_sink_backward(*[ptr] * 10, *args, *st, None, None, 4, 0, 0.0, ptr, 1 << 30, None))
    got.append(lib.smha_cache_forward(ptr, ptr, ptr, None, None, ptr, None, ptr, 2, 2, 2, 8, 8, 0, 64, 0, None, None, None, None, None, s, None, 0, 0, 0.0, None, 0, None))
    for k, v in ((s, None), (None, s)):
        got.append(lib.smha_cache_evict(ptr, *[ptr] * 7, 2, 2, 8, 64, 4, 1, k, v, ptr, 1 << 30, None))
    assert got == [2 if strides in OVERLAPPING else 5] * 7


def test_accounts_that_overlap_are_refused():
    """Accounts are read, added to and written without atomics: a key's belongs to one head of one sequence."""
    if torch.cuda.is_available():
        pytest.skip("the addresses are not real")
    C, lib, ptr = abi()

    def weigh(strides, B=2, Hkv=2, Sk=8):
        return lib.smha_cache_forward(ptr, ptr, ptr, None, None, ptr, ptr, ptr, B, 2 * Hkv, Hkv, 1, Sk, 0, 64, 0, *[None] * 6, (C.c_int64 * 2)(*strides), 0, 0, 0.0, ptr, 1 << 40,
                                      None)

    for bad in ((0, 8), (16, 0), (8, 8), (16, 7), (-16, 8), (16, -8), (12, 8)):
        assert weigh(bad) == 2, bad
    for good in ((16, 8), (8, 16), (100, 9)):
        assert weigh(good) == 5, good
    assert weigh((0, 8), B=1) == 5 and weigh((8, 0), Hkv=1) == 5


def test_sizes_whose_products_pass_64_bits_are_refused():
    """No memory holds them, but their products come out small; and a workspace's size is only told for calls that are taken."""
    C, lib, ptr = abi()
    need = C.c_size_t(7)
    big, top = 1 << 30, (1 << 31) - 1
    for sizes in ((big, big, 1, 1 << 26, 8, 0), (big, big, big, 1 << 26, 8, 0), (1 << 22, 1 << 22, 1, 1 << 22, 8, 0), (1, 1, 1, 1, top, 0), (1, 1, 1, 1, 1, top),
                  (1, 1, 1, 1 << 27, 8, 0), (1, 1, 1, 1, 1 << 27, 0)):
        for weigh in (0, 1):
            assert lib.smha_cache_workspace(*sizes, 8, 0, 0, weigh, C.byref(need)) == 2, sizes
        assert lib.smha_cache_forward(*[ptr] * 6, None, ptr, *sizes, 8, 0, *[None] * 7, 0, 0, 0.0, ptr, 1 << 62, None) == 2, sizes
    for Sq, Sk in ((8, top), (top, 8), (1 << 27, 8), (8, 1 << 27), (1 << 29, 1 << 29)):
        assert lib.smha_sink_workspace(1, 1, 1, Sq, Sk, 8, 4, 0, C.byref(need)) == 2, (Sq, Sk)
        assert lib.smha_sink_forward(*[ptr] * 4, None, None, 1, 1, 1, Sq, Sk, 8, 0, *[None] * 6, 4, 0, 0.0, None) == 2, (Sq, Sk)
    assert need.value == 7
    # the longest heads that 2 GiB hold at 8 columns
    assert lib.smha_sink_workspace(1, 1, 1, 8, (1 << 27) - 129, 8, 4, 0, C.byref(need)) == 0
    assert lib.smha_cache_workspace(1, 1, 1, 1, (1 << 27) - 65, 0, 8, 4, 0, 0, C.byref(need)) == 0


def sink_workspace(*sizes):
    C, lib, _ = abi()
    need = C.c_size_t(0)
    assert lib.smha_sink_workspace(*sizes, C.byref(need)) == 0
    return need.value


def test_a_long_document_with_sinks_needs_little_more_than_one_without():
    """Places for partial sums belong to key tiles that are cut: here the one with sinks, whose up to 400 parts in all (twelve steps at least, equally
    shared) are 2 x 128 x columns x 4 bytes each."""
    for B, H, Hkv, S, d, window in ((1, 32, 32, 131072, 128, 1024), (4, 32, 8, 32768, 128, 512), (1, 32, 8, 131072, 128, 1024), (2, 16, 16, 65536, 64, 256)):
        without, with_ = (sink_workspace(B, H, Hkv, S, S, d, window, n) for n in (0, 4))
        assert without == 2 * B * H * S * 4  # lse and delta of every query
        assert with_ - without <= (400 + B * Hkv) * 2 * 128 * d * 4, (B, H, S, with_ - without)


@pytest.mark.gpu
@pytest.mark.parametrize("case", [
    # B, H, Hkv, S, d, window, n_sink: tiles that are cut are
    (1, 2, 2, 1000, 64, 16, 4),      # the sinks' alone
    (2, 3, 3, 700, 80, 30, 130),     # two of them
    (2, 4, 2, 1000, 128, 100, 3),    # all
    (1, 2, 2, 600, 64, 0, 0),        # all, without sinks
    (1, 1, 1, 150, 32, 16, 2),       # none
], ids=str)
def test_a_backward_pass_keeps_to_its_workspace(case):
    from test_sink import check, reference, tensors
    B, H, Hkv, S, d, window, n_sink = case
    q, k, v, g = tensors(B, H, Hkv, S, S, d, torch.bfloat16)
    want = reference(q, k, v, g, window, n_sink, None, None, 0.0)
    need = sink_workspace(B, H, Hkv, S, S, d, window, n_sink)
    out, rest, lse = torch.empty_like(q), torch.empty_like(q), torch.empty(B, H, S, device="cuda")
    grads = [torch.full_like(t, float("nan")) for t in (q, k, v)]
    smha.smha_sink_forward(q, k, v, out, lse, window, n_sink, O_rest=rest)
    room = torch.full((need + 4096,), 0xAB, dtype=torch.uint8, device="cuda")
    smha.smha_sink_backward(q, k, v, out, lse, g, *grads, window, n_sink, workspace=room[:need], O_rest=rest)
    for name, got in zip(("out", "dq", "dk", "dv"), (out, *grads)):
        check(got, want[name], name)
    assert bool((room[need:] == 0xAB).all())


@pytest.mark.gpu
def test_a_window_counts_slots_also_after_an_eviction():
    """As documented: eviction moves recent keys to slots that were freed, where a window does not look for them; without one every key that stayed is seen."""
    from test_cache import check, evict_inputs, int32, make, reference
    k, v, w, _ = evict_inputs(2, 2, 80, 64)
    positions = torch.arange(80, dtype=torch.int32, device="cuda").expand(2, 2, 80).contiguous()
    q = make(2, 4, 2, 1, 80, 64)[0]
    w, positions, n = smha.cache_evict(k, v, w, positions, int32([80, 61]), 32, 16)
    recent = positions[:, :, :32] >= (n.new_tensor([80, 61]) - 16)[:, None, None]
    assert bool((recent.sum(-1) == 16).all()) and not bool(recent[:, :, 16:].all())  # (they are there, but not in the last slots)
    for window, n_sink in ((0, 0), (16, 0), (16, 4)):
        want, bound, _ = reference(q, k, v, n.tolist(), window, n_sink)
        check(smha.cache_attention(q, k, v, n, window=window, n_sink=n_sink), want, bound, f"window {window}")


def test_a_warning_of_the_first_call_may_call_again(monkeypatch, tmp_path):
    """What shows the warning that there is no native path (a log, say) may itself make a call."""
    import threading
    import warnings
    from paper_2506_06095_amd import binding
    monkeypatch.setattr(binding, "_native", None)
    monkeypatch.setattr(binding._build, "EXT", str(tmp_path / "_smha_torch.so"))
    monkeypatch.setenv("CXX", "false")
    shown = []

    def show(*args, **kwargs):
        shown.append(binding.native_call("cache_evict")())

    def call():
        with warnings.catch_warnings():
            warnings.simplefilter("always")
            warnings.showwarning = show
            binding.native_call("cache_evict")

    thread = threading.Thread(target=call, daemon=True)
    thread.start()
    thread.join(20)
    assert not thread.is_alive() and shown == [None]
