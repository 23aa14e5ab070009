"""A cache held in 4 bits: packing against the format's definition, byte for byte; reading back, bit for bit; attention against its formula in 64 bits on
the values that the rows stand for; all of them together as a serving loop runs them; and refusals.

Tolerance of an output of attention: u |O| (its rounding) + sum_j (2^-11 P + 2^-25) |V| (the probabilities' rounding to binary16, whatever the type;
relative to a reference that is no larger than the largest score, they sum to 1 at least) + F sum_j P |V|, with u half a step of the type and F = 2e-5
for sums and exponentials in 32 bits (scores stay below 60, whose exponents are rounded by 60 log2(e) 2^-24 = 5e-6, and are sums of 128 products
of which no partial sum passes 60 sqrt(128): another 60 * 2^-24 * 2).  Keys and values are what the rows stand for, exactly.
"""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2506_06095_amd as smha  # noqa: E402

F = 2e-5
TYPES = pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])


# --- the format, from its definition, on numpy arrays

def row_bytes(d):
    return 4 * ((d + 31) // 32) + d // 2


def pack_group(x):
    """(s, m, codes) of one group's columns (a list of at most 32 numbers)."""
    if any(math.isnan(v) for v in x):
        return np.float16(0), np.float16("nan"), [0] * len(x)
    x = [max(-65280.0, min(65280.0, float(v))) for v in x]
    m = np.float16(min(x))
    if float(m) > min(x):
        m = np.nextafter(m, np.float16(-np.inf))
    m = np.float16(0) if m == 0 else m
    s = np.float16(max(0.0, (max(x) - float(m)) / 15))
    while s > 0 and 15 * float(np.nextafter(s, np.float16(0))) + float(m) >= max(x):
        s = np.nextafter(s, np.float16(0))
    while 15 * float(s) + float(m) < max(x):
        s = np.nextafter(s, np.float16(np.inf))
    borders = [float(m) + (k + 0.5) * float(s) for k in range(15)] if s > 0 else [math.inf] * 15  # exact: 41 binary digits at most
    return s, m, [sum(v >= b for b in borders) for v in x]


def pack_rows(x):
    """[..., d] float64 -> [..., row] uint8."""
    d = x.shape[-1]
    out = np.zeros((*x.shape[:-1], row_bytes(d)), np.uint8)
    G = (d + 31) // 32
    for at in np.ndindex(*x.shape[:-1]):
        words = [0] * (d // 8)
        heads = []
        for g in range(G):
            s, m, codes = pack_group(x[at][32 * g:32 * g + 32].tolist())
            heads += [s, m]
            for i, c in enumerate(codes):
                col = 32 * g + i
                words[col // 8] |= c << (16 * (col % 2) + 4 * (col % 8 // 2))
        out[at] = np.frombuffer(np.array(heads, "<f2").tobytes() + np.array(words, "<u4").tobytes(), np.uint8)
    return out


def unpack_rows(rows, d):
    """[..., row] uint8 -> [..., d]: the binary16 values, as float64."""
    G = (d + 31) // 32
    rows = np.ascontiguousarray(rows)
    head = rows[..., :4 * G].copy().view("<f2").astype(np.float64)
    word = rows[..., 4 * G:].copy().view("<u4")
    out = np.empty((*rows.shape[:-1], d))
    for col in range(d):
        code = (word[..., col // 8] >> (16 * (col % 2) + 4 * (col % 8 // 2))) & 15
        with np.errstate(invalid="ignore", over="ignore"):
            out[..., col] = (code * head[..., col // 32 * 2] + head[..., col // 32 * 2 + 1]).astype(np.float16)
    return out


def test_the_format_by_hand():
    s, m, codes = pack_group([0.0, 15.0, 7.5, 7.49, 14.5, 3.0])
    assert (s, m, codes) == (1, 0, [0, 15, 8, 7, 15, 3])       # a tie goes up
    assert pack_group([0.25] * 32)[:2] == (0, 0.25) and pack_group([0.25] * 32)[2] == [0] * 32
    s, m, codes = pack_group([1e-9, 2e-9])                      # below binary16: a base of 0, the smallest step
    assert (s, m, codes) == (np.float16(2.0 ** -24), 0, [0, 0])
    s, m, codes = pack_group([-1e-9, 0.0])
    assert (s, m, codes) == (np.float16(2.0 ** -24), np.float16(-(2.0 ** -24)), [1, 1])
    s, m, codes = pack_group([-math.inf, math.inf])
    assert (s, m, codes) == (8704, -65280, [0, 15]) and np.isfinite(np.float16(15.0 * 8704 - 65280))
    row = pack_rows(np.arange(8.0)[None] * 15 / 7)
    assert row.shape == (1, 8) and unpack_rows(row, 8)[0].tolist() == [0, 2, 4, 6, 9, 11, 13, 15]
    assert row[0, 4:].tolist() == [0x40, 0xD9, 0x62, 0xFB]      # columns 0 2 | 4 6 | 1 3 | 5 7


def test_a_row_is_five_bits_a_column_and_says_how_many():
    assert [smha.smha_packed_row(d) for d in (8, 32, 64, 80, 128)] == [8, 20, 40, 52, 80]
    widths = [smha.smha_packed_row(d) for d in range(8, 129, 8)]
    assert widths == [row_bytes(d) for d in range(8, 129, 8)] and len(set(widths)) == 16
    for d in (0, 4, 12, 136):
        with pytest.raises(smha.SmhaError):
            smha.smha_packed_row(d)


# --- on the GPU

def int32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def rows_of(t):
    return t.float().cpu().double().numpy()


def new_tokens(B, Hkv, T, d, dtype, layout="bhsd", seed=1, scale=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def new():
        shape = (B, T, Hkv, d) if layout == "bshd" else (B, Hkv, T, d)
        t = (torch.randn(shape, generator=gen, device="cuda") * scale).to(dtype)
        return t.transpose(1, 2) if layout == "bshd" else t
    return new(), new()


def old_cache(B, Hkv, Sk, d, seed=2):
    """Bytes of any kind."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return tuple(torch.randint(0, 256, (B, Hkv, Sk, row_bytes(d)), generator=gen, device="cuda", dtype=torch.uint8) for _ in range(2))


WRITES = [
    # B, Hkv, T, Sk, d, lengths, offsets, layout
    (1, 1, 1, 1, 8, [1], None, "bhsd"),
    (1, 2, 1, 256, 64, [256], None, "bhsd"),
    (5, 3, 1, 9, 128, [0, 1, 5, 9, 12], None, "bhsd"),              # none, the first, the last, more than there are
    (3, 2, 7, 10, 80, [3, 10, 7], None, "bshd"),                    # more tokens than keys
    (3, 2, 7, 10, 96, [3, 10, -4], [0, 2, 0], "bshd"),              # padded behind
    (4, 1, 6, 12, 40, [12, 12, 12, 12], [-3, 9, 50, -50], "bhsd"),  # partly before the cache and past it, wholly
    (2, 4, 33, 40, 32, [40, 35], [7, 0], "bhsd"),
    (2, 1, 3, 8, 24, [8, 7], [2147483647, -2147483648], "bhsd"),    # places past 32 bits
    (70, 1, 2, 5, 16, [i % 6 for i in range(70)], None, "bhsd"),
    (1, 2, 21, 30, 120, [30], None, "bshd"),
]


def slots(lengths, offsets, b, T, Sk):
    """(token, slot) pairs that are kept."""
    n = min(max(lengths[b], 0), Sk)
    at = n - T if offsets is None else offsets[b]
    return [(t, at + t) for t in range(T) if 0 <= at + t < n]


@pytest.mark.gpu
@TYPES
@pytest.mark.parametrize("case", WRITES, ids=lambda c: "x".join(str(x) for x in c[:5]))
def test_written_rows_are_the_format(case, dtype):
    B, Hkv, T, Sk, d, lengths, offsets, layout = case
    kn, vn = new_tokens(B, Hkv, T, d, dtype, layout)
    for values in (False, True):
        k, v = old_cache(B, Hkv, Sk, d)
        before = (k.cpu().numpy().copy(), v.cpu().numpy().copy())
        versions = k._version, v._version
        got = smha.packed_write(kn, vn, k, v, int32(lengths), offsets=None if offsets is None else int32(offsets), values=values)
        assert k._version > versions[0] and v._version > versions[1]
        assert (got is None) == (not values)
        for i, (new, cache) in enumerate(((kn, k), (vn, v))):
            want, rows = before[i], pack_rows(rows_of(new))
            kept = np.zeros((B, Hkv, T, d), bool)
            for b in range(B):
                for t, slot in slots(lengths, offsets, b, T, Sk):
                    want[b, :, slot] = rows[b, :, t]
                    kept[b, :, t] = True
            assert np.array_equal(cache.cpu().numpy(), want)
            if values:
                stands = torch.from_numpy(np.where(kept, unpack_rows(rows, d), 0.0)).to(torch.float32).to(dtype)
                assert got[i].is_contiguous() and torch.equal(got[i].cpu(), stands)


@pytest.mark.gpu
@TYPES
def test_values_at_borders_are_packed_exactly(dtype):
    """Ties, constants, signed zeros, values that differ from a border by less than 32 bits hold, the type's largest and smallest, infinities, NaN."""
    rng = np.random.default_rng(5)
    tiny, top = torch.finfo(dtype).smallest_normal, torch.finfo(dtype).max
    sub = float(torch.tensor(1, dtype=torch.int16).view(dtype))
    groups = [[0.0] * 32, [-0.0] * 32, [0.0, -0.0] * 16, [-0.0, 0.0] * 16, [0.1] * 32, [-7.25] * 32, [sub] * 32, [-sub, sub] * 16, [tiny, -tiny] * 16,
              [top, -top] * 16, [math.inf] + [1.0] * 31, [-math.inf, math.inf] * 16, [1.0] * 31 + [math.nan], [math.nan] * 32, [math.inf, math.nan] * 16,
              [65504.0, -3.0] * 16, [top] * 32, [1e-8] * 16 + [-1e-8] * 16]
    for _ in range(200):  # multiples of a step: (k + 1/2) s is hit often, also where s was rounded up
        n = int(rng.integers(1, 31))
        unit = 2.0 ** rng.integers(-20, 8)
        groups.append((rng.integers(-n, n + 1, 32) * unit / 2).tolist())
    for _ in range(100):  # a wide range with values next to 0 or to a border
        x = rng.standard_normal(32) * 10.0 ** rng.integers(-6, 4)
        x[rng.integers(0, 32, 8)] *= 1e-6
        groups.append(x.tolist())
    for _ in range(50):   # 0 .. 15 steps and halves about a base, with the smallest values of the type added
        base, step = float(rng.integers(-20, 20)), 2.0 ** rng.integers(-3, 3)
        groups.append([base, base + 15 * step] + [base + (rng.integers(0, 15) + 0.5) * step for _ in range(29)] + [sub])
    x = torch.tensor(groups, dtype=torch.float64).to(torch.float32).to(dtype)
    rows = x.reshape(1, 1, -1, 32)
    T = rows.shape[2]
    k, v = smha.packed_cache(1, 1, T, 32)
    got = smha.packed_write(rows.cuda(), rows.flip(2).cuda(), k, v, int32([T]), values=True)
    want = pack_rows(rows_of(rows))
    assert np.array_equal(k.cpu().numpy(), want) and np.array_equal(v.cpu().numpy(), want[:, :, ::-1])
    stands = unpack_rows(want, 32)
    assert np.array_equal(got[0].float().cpu().numpy(), torch.from_numpy(stands).float().to(dtype).float().numpy(), equal_nan=True)
    # within half a step and half a last place of binary16
    inside = np.clip(rows_of(rows), -65280, 65280)
    step = want[..., :2].copy().view("<f2").astype(np.float64)
    finite = ~np.isnan(inside).any(-1)
    off = np.abs(stands - inside)[finite]
    assert bool((off <= (step / 2 + np.maximum(2.0 ** -11 * np.abs(stands), 2.0 ** -25))[finite]).all()) and np.isfinite(stands[finite]).all()
    assert np.isnan(stands[~finite]).all()


def pack_many(x):
    """[n, 32] float64 -> (s, m, codes), as pack_group, all rows at once (finite ones, within 65280)."""
    lo, hi = x.min(1), x.max(1)
    m = lo.astype(np.float16)
    m = np.where(m > lo, np.nextafter(m, np.float16(-np.inf)), m) + np.float16(0)
    s = ((hi - m.astype(np.float64)) / 15).astype(np.float16)
    for _ in range(2):
        less = np.nextafter(s, np.float16(0))
        s = np.where((s > 0) & (15 * less.astype(np.float64) + m >= hi), less, s)
    for _ in range(2):
        s = np.where(15 * s.astype(np.float64) + m < hi, np.nextafter(s, np.float16(np.inf)), s)
    codes = np.zeros(x.shape, np.int64)
    for k in range(15):
        codes += (x >= (m.astype(np.float64) + (k + 0.5) * s.astype(np.float64))[:, None]) & (s > 0)[:, None]
    return s, m, codes


@pytest.mark.gpu
@TYPES
def test_many_groups_are_packed_exactly(dtype):
    """Groups of all kinds, most of whose waves hold no value near a border, and groups of which every value is near one."""
    rng = np.random.default_rng(11)
    n = 1 << 15
    size = 10.0 ** rng.uniform(-5, 3, (n, 1))
    x = rng.standard_normal((n, 32)) * size + rng.standard_normal((n, 1)) * size * (rng.random((n, 1)) < 0.5) * 20
    x[: n // 2, 1:] = np.round(x[: n // 2, 1:] / size[: n // 2] * 8) * size[: n // 2] / 8  # few values to a group
    x = torch.from_numpy(np.clip(x, -60000, 60000)).float().to(dtype)
    # values at a border and next to it: base + (k + 1/2) s and its neighbours, of groups that have these s and base
    s, m, _ = pack_many(x[n // 2:n // 2 + n // 4].double().numpy())
    k = rng.integers(0, 15, (n // 4, 30)) + 0.5
    x[n // 2:n // 2 + n // 4, 2:] = torch.from_numpy(m.astype(np.float64)[:, None] + k * s.astype(np.float64)[:, None]).float().to(dtype)
    s, m, codes = pack_many(x.double().numpy())
    word = np.zeros((n, 4), np.uint32)
    for col in range(32):
        word[:, col // 8] |= codes[:, col].astype(np.uint32) << np.uint32(16 * (col % 2) + 4 * (col % 8 // 2))
    want = np.concatenate([np.stack([s, m], 1).astype("<f2").view(np.uint8).reshape(n, 4), word.astype("<u4").view(np.uint8).reshape(n, 16)], 1)
    k4, v4 = smha.packed_cache(1, 1, n, 32)
    rows = x.reshape(1, 1, n, 32).cuda()
    smha.packed_write(rows, rows.flip(2), k4, v4, int32([n]))
    assert np.array_equal(k4[0, 0].cpu().numpy(), want) and np.array_equal(v4[0, 0].cpu().numpy(), want[::-1])


def test_the_two_references_of_the_format_agree():
    rng = np.random.default_rng(3)
    x = np.round(rng.standard_normal((200, 32)) * 8) / 8 * 10.0 ** rng.integers(-6, 4, (200, 1))
    s, m, codes = pack_many(x)
    for i in range(200):
        a, b, c = pack_group(x[i].tolist())
        assert (a, b, c) == (s[i], m[i], codes[i].tolist())


READS = [
    # B, Hkv, T, Sk, d, lengths, offsets
    (1, 1, 1, 1, 8, [1], None),
    (2, 3, 40, 40, 64, [40, 17], None),
    (3, 2, 9, 30, 80, [30, 4, 0], None),
    (3, 2, 9, 30, 128, [30, 33, -1], [25, -4, 0]),
    (2, 1, 50, 20, 104, [20, 13], [3, -2]),                  # more than there are
    (2, 1, 3, 8, 24, [8, 7], [2147483647, -2147483648]),
]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16, torch.float32], ids=["f16", "bf16", "f32"])
@pytest.mark.parametrize("case", READS, ids=lambda c: "x".join(str(x) for x in c[:5]))
def test_what_is_read_is_what_the_rows_stand_for(case, dtype):
    """On rows of any bytes (all of them stand for something, infinities and NaN too)."""
    B, Hkv, T, Sk, d, lengths, offsets = case
    k, v = old_cache(B, Hkv, Sk, d)
    at = None if offsets is None else int32(offsets)
    got = smha.packed_read(k, v, int32(lengths), offsets=at, tokens=T, dtype=dtype)
    for out, cache in zip(got, (k, v)):
        stands = unpack_rows(cache.cpu().numpy(), d)
        want = np.zeros((B, Hkv, T, d))
        for b in range(B):
            for t, slot in slots(lengths, offsets if offsets else [0] * B, b, T, Sk):
                want[b, :, t] = stands[b, :, slot]
        want = torch.from_numpy(want).float().to(dtype)
        assert out.dtype == dtype and torch.equal(out.cpu().nan_to_num(nan=12345.0), want.nan_to_num(nan=12345.0))
        assert torch.equal(out.cpu().isnan(), want.isnan())
    # into tensors of other strides
    into = tuple(torch.full((B, T, Hkv, 2, 128), -1.0, dtype=dtype, device="cuda") for _ in range(2))
    views = tuple(t[:, :, :, 1, :d].transpose(1, 2) for t in into)
    back = smha.packed_read(k, v, int32(lengths), offsets=at, tokens=T, dtype=dtype, out=views)
    assert back[0] is views[0] and back[1] is views[1]
    for a, b, t in zip(got, views, into):
        assert torch.equal(a.nan_to_num(), b.nan_to_num()) and bool((t[:, :, :, 0] == -1).all()) and bool((t[:, :, :, 1, d:] == -1).all())


@pytest.mark.gpu
def test_all_slots_are_read_by_default():
    k, v = smha.packed_cache(2, 2, 37, 64)
    kn, vn = new_tokens(2, 2, 37, 64, torch.float16)
    stands = smha.packed_write(kn, vn, k, v, int32([37, 37]), values=True)
    got = smha.packed_read(k, v, int32([37, 37]))
    assert all(torch.equal(a, b) and a.dtype == torch.float16 for a, b in zip(stands, got))


# --- attention

def reference(q, k, v, lengths, window=0, n_sink=0, scale=0.0):
    """(out, its bound) in 64 bits on the CPU, on the values that the rows stand for."""
    (B, H, T, d), (Hkv, Sk) = q.shape, k.shape[1:3]
    u, z = torch.finfo(q.dtype).eps / 2, 2.0 ** -25 if q.dtype == torch.float16 else 0.0
    scale = scale if scale > 0 else d ** -0.5
    q = q.cpu().double()
    k, v = (torch.from_numpy(unpack_rows(t.cpu().numpy(), d)) for t in (k, v))
    out, tol = torch.zeros_like(q), torch.zeros_like(q)
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
            s = (q[b, h] @ K.T * scale).masked_fill(~seen, -math.inf)
            P = torch.where(seen, torch.exp(s - torch.logsumexp(s, 1).nan_to_num(neginf=0.0)[:, None]), 0.0)
            out[b, h] = P @ V
            tol[b, h] = torch.where(seen, (2.0 ** -11 + F) * P + 2.0 ** -25, 0.0) @ V.abs()
    return out, tol * (1 + u) + u * out.abs() + z


def check(got, want, bound, what="output"):
    got = got.detach().cpu().double()
    ok = torch.isfinite(got) & ((got - want).abs() <= bound)
    assert got.shape == want.shape and bool(ok.all()), f"{what}: {int((~ok).sum())} of {ok.numel()} off, worst {float(((got - want).abs() - bound).max())}"


def filled(B, Hkv, Sk, d, seed=3):
    """A cache whose every slot holds a key."""
    k, v = smha.packed_cache(B, Hkv, Sk, d)
    kn, vn = new_tokens(B, Hkv, Sk, d, torch.float16, seed=seed)
    smha.packed_write(kn, vn, k, v, int32([Sk] * B))
    return k, v


def queries(B, H, T, d, dtype, layout="bhsd", seed=4):
    return new_tokens(B, H, T, d, dtype, layout, seed)[0]


CASES = [
    # B, H, Hkv, T, Sk, d, window, n_sink, lengths, layout
    (1, 1, 1, 1, 1, 64, 0, 0, [1], "bhsd"),
    (1, 8, 2, 1, 256, 64, 64, 4, [256], "bhsd"),
    (3, 4, 4, 1, 100, 128, 0, 0, [0, 1, 100], "bshd"),               # an empty sequence, one key
    (2, 6, 2, 3, 333, 80, 50, 7, [333, 2], "bhsd"),                  # fewer keys than tokens
    (2, 16, 2, 5, 700, 128, 100, 40, [699, 130], "bshd"),            # 40 rows on a key head
    (2, 16, 1, 4, 97, 32, 0, 0, [97, 33], "bhsd"),                   # 64 rows
    (1, 16, 2, 40, 120, 64, 60, 3, [119], "bhsd"),                   # 320 rows
    (1, 4, 1, 1, 20000, 128, 0, 0, [19999], "bhsd"),                 # many segments
    (2, 4, 2, 1, 9000, 64, 4096, 130, [9000, 8999], "bhsd"),
    (70, 2, 1, 1, 64, 8, 0, 0, [(7 * i) % 65 for i in range(70)], "bhsd"),   # more sequences than lanes
    (150, 4, 2, 2, 300, 64, 33, 2, [(31 * i) % 301 for i in range(150)], "bhsd"),
    (70, 2, 1, 1, 2000, 64, 0, 0, [(29 * i) % 2001 for i in range(70)], "bhsd"),
    (70, 4, 4, 1, 1400, 128, 0, 0, [(1400 - 21 * i) for i in range(67)] + [0, 1, 2], "bshd"),
    (2, 2, 1, 1, 50, 64, 1, 0, [50, 49], "bhsd"),                    # a window of one key
    (1, 2, 1, 130, 130, 128, 0, 0, [130], "bhsd"),                   # a whole prompt
    (2, 4, 2, 129, 257, 72, 0, 0, [257, 100], "bshd"),               # a chunk; a sequence shorter than it
    (1, 8, 1, 70, 1000, 104, 200, 70, [1000], "bhsd"),               # 560 rows in a window
    (1, 3, 1, 11, 66, 16, 5, 2, [66], "bhsd"),                       # 33 rows, three heads a key head
    (2, 12, 4, 90, 4000, 128, 0, 0, [4000, 1931], "bhsd"),           # 270 rows, long
    (1, 17, 1, 1, 77, 40, 0, 0, [77], "bhsd"),                       # 17 rows
    (1, 5, 1, 13, 3000, 56, 0, 0, [2999], "bhsd"),                   # 65 rows
    (3, 2, 2, 300, 700, 64, 128, 0, [700, 299, 1], "bshd"),
    (90, 2, 1, 1, 3000, 64, 0, 0, [3000 if i == 50 else 5 + 7 * i for i in range(90)], "bhsd"),   # one long sequence among short ones, counted in LDS
    (70, 8, 1, 5, 900, 128, 0, 0, [900 - 13 * i for i in range(69)] + [0], "bhsd"),                # 40 rows of each of 70 sequences
    (300, 1, 1, 1, 1700, 32, 0, 0, [(1701 * i) // 300 for i in range(300)], "bhsd"),
    (4200, 2, 2, 1, 40, 8, 0, 0, [i % 41 for i in range(4200)], "bhsd"),                           # too many sequences to count
    (3, 16, 1, 100, 1500, 64, 0, 0, [1500, 90, 700], "bhsd"),                                     # 13 tiles of 128 rows, cut
    (20, 4, 1, 100, 2000, 64, 0, 0, [2000 - 101 * i for i in range(19)] + [30], "bhsd"),           # 4 tiles of rows of 20 sequences, counted in LDS
    (300, 4, 4, 1, 1700, 8, 0, 0, [1700 if i == 77 else 40 - i % 40 for i in range(300)], "bhsd"), # groups that fill the chip, of which some are cut
    (1, 32, 2, 1024, 1100, 64, 100, 3, [1100], "bshd"),                                            # one sequence's that do
]


@pytest.mark.gpu
@TYPES
@pytest.mark.parametrize("case", CASES, ids=lambda c: "x".join(str(x) for x in c[:8]))
def test_attention_is_the_formula(case, dtype):
    B, H, Hkv, T, Sk, d, window, n_sink, lengths, layout = case
    k, v = filled(B, Hkv, Sk, d)
    q = queries(B, H, T, d, dtype, layout)
    want, bound = reference(q, k, v, lengths, window, n_sink)
    out = smha.packed_attention(q, k, v, int32(lengths), window=window, n_sink=n_sink)
    check(out, want, bound)
    again = torch.full_like(out, math.nan)
    assert smha.packed_attention(q, k, v, int32(lengths), window=window, n_sink=n_sink, out=again) is again
    assert torch.equal(again, out)


@pytest.mark.gpu
@pytest.mark.parametrize("H, T", [(16, 1), (32, 10)])   # 1 and 20 rows on a key head, with more tiles than are cut into the chip's segments once
def test_long_caches_as_the_16_bit_operator_reads_them(H, T):
    """Both operators are within the bound above of the formula on the same binary16 values; sum P |V| by the 16-bit operator on |V|, which is half a percent off at most."""
    B, Hkv, Sk, d = 2, 16, 110000, 128
    k, v = filled(B, Hkv, Sk, d)
    lengths = int32([Sk, Sk - 9999])
    q = queries(B, H, T, d, torch.float16) * 3
    got = smha.packed_attention(q, k, v, lengths)
    assert torch.equal(smha.packed_attention(q, k, v, lengths), got)
    keys, values = smha.packed_read(k, v, lengths)
    want = smha.cache_attention(q, keys, values, lengths).double()
    size = smha.cache_attention(q, keys, values.abs(), lengths).double() * 1.005
    rows = values.abs().double().sum(2).repeat_interleave(H // Hkv, 1)[:, :, None]
    bound = 2 * ((2.0 ** -11 + F) * size + 2.0 ** -25 * rows + 2.0 ** -11 * (want.abs() * 1.01) + 2.0 ** -25)
    assert bool(((got.double() - want).abs() <= bound).all())


@pytest.mark.gpu
@pytest.mark.parametrize("T, Sk", [(2, 600), (2, 6000), (30, 600), (30, 9000), (90, 9000)])   # few rows whole and cut, 120 rows, 360
def test_what_is_not_seen_may_hold_anything(T, Sk):
    k, v = filled(2, 2, Sk, 128)
    q = queries(2, 8, T, 128, torch.float16)
    n, window, n_sink = Sk - 45, 100, 5
    want = smha.packed_attention(q, k, v, int32([n, 1]), window=window, n_sink=n_sink)
    first = n - T - window + 1  # the first key in the first token's window
    for t in (k, v):
        t[0, :, n:] = 0xFF  # (steps, bases and so values that are NaN)
        t[0, :, n_sink:first] = 0xFF
        t[1, :, 1:] = 0xFF
    assert bool(torch.isfinite(want).all())
    assert torch.equal(smha.packed_attention(q, k, v, int32([n, 1]), window=window, n_sink=n_sink), want)
    assert bool((want[1, :, :T - 1] == 0).all()) and bool((want[1, :, T - 1] != 0).any())


@pytest.mark.gpu
@TYPES
@pytest.mark.parametrize("T, Sk", [(1, 300), (1, 5000), (20, 300)])
def test_a_query_of_nan_stays_nan_alone(T, Sk, dtype):
    k, v = filled(1, 2, Sk, 64)
    q = queries(1, 4, T, 64, dtype)
    want = smha.packed_attention(q, k, v, int32([Sk]))
    q[0, 1, 0, 5] = math.nan
    got = smha.packed_attention(q, k, v, int32([Sk]))
    assert bool(got[0, 1, 0].isnan().all())
    got[0, 1, 0] = want[0, 1, 0]
    assert torch.equal(got, want)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 12, 40])
def test_queries_of_any_size_are_brought_to_binary16(T):
    """bfloat16 queries times a power of two, and the scale by its inverse: the same bits, far past what binary16 holds."""
    k, v = filled(2, 2, 777, 96)
    q = queries(2, 6, T, 96, torch.bfloat16)
    want = smha.packed_attention(q, k, v, int32([777, 300]), scale=0.125)
    for p in (-90, -30, 17, 60):
        assert torch.equal(smha.packed_attention(q * 2.0 ** p, k, v, int32([777, 300]), scale=0.125 * 2.0 ** -p), want)
    assert torch.equal(smha.packed_attention(torch.zeros_like(q), k, v, int32([777, 300])), smha.packed_attention(q, k, v, int32([777, 300]), scale=1e-38))


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128, 72])
@pytest.mark.parametrize("T, Sk", [(1, 90), (1, 4000), (20, 4000)])
def test_caches_of_any_strides(d, T, Sk):
    """Keys and values side by side, tokens before heads, a head's first byte aligned to 4 and no more."""
    B, Hkv, R = 2, 3, row_bytes(d)
    both = torch.randint(0, 256, (B, Sk, Hkv, 2, R + 12), dtype=torch.uint8, device="cuda")
    k, v = (both[:, :, :, i, 4:4 + R].transpose(1, 2) for i in range(2))
    packed = smha.packed_cache(B, Hkv, Sk, d)
    kn, vn = new_tokens(B, Hkv, Sk, d, torch.bfloat16, "bshd")
    around = both.clone()
    for cache in ((k, v), packed):
        smha.packed_write(kn, vn, *cache, int32([Sk, Sk - 7]), offsets=int32([0, 0]))
    for i, t in enumerate(packed):
        around[0, :, :, i, 4:4 + R] = t[0].transpose(0, 1)
        around[1, :Sk - 7, :, i, 4:4 + R] = t[1, :, :Sk - 7].transpose(0, 1)
    assert torch.equal(both, around)  # and nothing beside the rows is written
    for a, b in zip(smha.packed_read(k, v, int32([Sk, Sk - 7])), smha.packed_read(*packed, int32([Sk, Sk - 7]))):
        assert torch.equal(a, b)
    q = queries(B, 6, T, d, torch.float16)
    want = smha.packed_attention(q, *packed, int32([Sk, Sk - 7]))
    assert torch.equal(smha.packed_attention(q, k, v, int32([Sk, Sk - 7])), want)
    # one row of heads read by all sequences (strides of 0)
    shared = [t[:1].expand(B, Hkv, Sk, R) for t in packed]
    assert torch.equal(smha.packed_attention(q, *shared, int32([Sk, Sk]))[0], want[0])


@pytest.mark.gpu
def test_caches_past_32_bits():
    """A head of nearly 2 GiB, of which the end is read; and batches further apart than 2^32 bytes."""
    d, R = 128, 80
    Sk = (2 ** 31 - R) // R - 65
    k, v = (torch.empty(1, 1, Sk, R, dtype=torch.uint8, device="cuda") for _ in range(2))
    kn, vn = new_tokens(1, 1, 200, d, torch.float16)
    smha.packed_write(kn, vn, k, v, int32([Sk]))
    small = smha.packed_cache(1, 1, 200, d)
    smha.packed_write(kn, vn, *small, int32([200]))
    assert torch.equal(k[:, :, Sk - 200:], small[0]) and torch.equal(v[:, :, Sk - 200:], small[1])
    got = smha.packed_read(k, v, int32([Sk]), offsets=int32([Sk - 200]), tokens=200)
    assert all(torch.equal(a, b) for a, b in zip(got, smha.packed_read(*small, int32([200]))))
    for T in (1, 40):
        q = queries(1, 4, T, d, torch.float16)
        want, bound = reference(q, *small, [200], window=100)
        check(smha.packed_attention(q, k, v, int32([Sk]), window=100), want, bound)
    del k, v
    k, v = (torch.empty(5, 1, 2 ** 30 // 4 // 4, R, dtype=torch.uint8, device="cuda")[:, :, :300] for _ in range(2))  # 5 GiB apart in all
    assert k.stride(0) * 4 > 2 ** 32
    kn, vn = new_tokens(5, 1, 300, d, torch.float16)
    smha.packed_write(kn, vn, k, v, int32([300] * 5))
    small = smha.packed_cache(5, 1, 300, d)
    smha.packed_write(kn, vn, *small, int32([300] * 5))
    assert torch.equal(k, small[0]) and torch.equal(v, small[1])
    q = queries(5, 4, 2, d, torch.float16)
    assert torch.equal(smha.packed_attention(q, k, v, int32([300] * 5)), smha.packed_attention(q, *small, int32([300] * 5)))
    assert all(torch.equal(a, b) for a, b in zip(smha.packed_read(k, v, int32([300] * 5)), smha.packed_read(*small, int32([300] * 5))))


@pytest.mark.gpu
@TYPES
def test_a_serving_loop(dtype):
    """Prompts of different lengths written at once, padded behind, and attended to; then tokens one by one, then three at once. Every output is the formula's on
    what the cache stands for by then, and what was written before stays."""
    B, H, Hkv, Sk, d = 3, 8, 2, 200, 80
    prompts = [150, 1, 77]
    k, v = smha.packed_cache(B, Hkv, Sk, d)
    lengths = int32(prompts)
    kn, vn = new_tokens(B, Hkv, 150, d, dtype, "bshd")
    kv, vv = smha.packed_write(kn, vn, k, v, lengths, offsets=int32([0] * B), values=True)
    # the prompt's own attention on what was kept of it: by the 16-bit operator, and (its last 9 tokens) on the packed cache
    q = queries(B, H, 150, d, dtype)
    out = smha.sink_attention(q, kv, vv, offsets=int32([0] * B), lengths=lengths)
    late = torch.stack([q[b, :, max(0, n - 9):n] if n >= 9 else torch.cat([q[b, :, n:9], q[b, :, :n]], 1) for b, n in enumerate(prompts)])
    want, bound = reference(late, k, v, prompts)
    got = smha.packed_attention(late, k, v, lengths)
    check(got, want, bound)
    # Apart by both ways' roundings of probabilities and outputs (half a step of the largest value each) and by the rounding of values to bfloat16; that of keys moves a
    # score by u sum |q| |k| / sqrt(d) at most, and so a probability by a factor of exp(2 of that).
    eps, top = torch.finfo(dtype).eps, float(vv.abs().max())
    shift = 0.0 if dtype == torch.float16 else eps / 2 * float((late.float().abs() @ kv.float().abs().repeat_interleave(H // Hkv, 1).mT).max()) / math.sqrt(d)
    for b, n in enumerate(prompts):
        t = min(n, 9)
        assert float((got[b, :, 9 - t:].float() - out[b, :, n - t:n].float()).abs().max()) <= (3 * eps + math.expm1(2 * shift)) * top
    at = prompts
    for step, T in enumerate([1, 1, 1, 3, 1]):
        lengths += T
        at = [n + T for n in at]
        kn, vn = new_tokens(B, Hkv, T, d, dtype, seed=10 + step)
        kept = k.clone()
        kv, vv = smha.packed_write(kn, vn, k, v, lengths, values=True)
        for b, n in enumerate(at):
            assert torch.equal(k[b, :, :n - T], kept[b, :, :n - T]) and torch.equal(k[b, :, n:], kept[b, :, n:])
            assert torch.equal(smha.packed_read(k, v, lengths, dtype=dtype)[1][b, :, n - T:n], vv[b])
        q = queries(B, H, T, d, dtype, seed=20 + step)
        for window, n_sink in ((0, 0), (40, 3)):
            want, bound = reference(q, k, v, at, window, n_sink)
            check(smha.packed_attention(q, k, v, lengths, window=window, n_sink=n_sink), want, bound, f"step {step}")


@pytest.mark.gpu
@pytest.mark.parametrize("Sk, H, T", [(100, 4, 1), (4000, 4, 1), (4000, 8, 3), (4000, 8, 40)])   # whole; cut; 12 rows; 160 rows
def test_a_captured_step_follows_lengths_and_inputs(Sk, H, T):
    B, Hkv, d = 3, 2, 128
    k, v = filled(B, Hkv, Sk, d)
    lengths = int32([Sk - 40, 50, T])
    kn, vn = new_tokens(B, Hkv, T, d, torch.float16)
    q = queries(B, H, T, d, torch.float16)

    def step():
        smha.packed_write(kn, vn, k, v, lengths)
        return smha.packed_attention(q, k, v, lengths), *smha.packed_read(k, v, lengths, offsets=lengths - 8, tokens=8)

    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        step()
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for i in range(4):
        lengths += 7
        kn.add_(0.25)
        q.mul_(-1.0)
        before = k.clone(), v.clone()
        graph.replay()
        replayed = [t.clone() for t in got]
        after = k.clone(), v.clone()
        torch.cuda.synchronize()
        k.copy_(before[0])
        v.copy_(before[1])
        assert not torch.equal(k, after[0])
        for a, b in zip(replayed, step()):
            assert torch.equal(a, b), i
        assert torch.equal(k, after[0]) and torch.equal(v, after[1])


@pytest.mark.gpu
@pytest.mark.parametrize("Sk", [100, 4000])
def test_other_streams_workspaces_and_the_way_through_python(Sk):
    k, v = filled(2, 2, Sk, 64)
    q = queries(2, 8, 2, 64, torch.bfloat16)
    lengths = int32([Sk, Sk // 2])
    want = smha.packed_attention(q, k, v, lengths)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = smha.packed_attention(q, k, v, lengths, stream=side)
    values = smha.packed_read(k, v, lengths, stream=side, dtype=torch.float32)
    side.synchronize()
    assert torch.equal(got, want) and all(torch.equal(a, b) for a, b in zip(values, smha.packed_read(k, v, lengths, dtype=torch.float32)))
    with torch.cuda.stream(side):
        got = smha.packed_attention(q, k, v, lengths)
    side.synchronize()
    assert torch.equal(got, want)
    need = smha.smha_packed_workspace(2, 8, 2, 2, Sk, 64)
    assert (need == 0) == (Sk == 100)
    out, workspace = torch.empty_like(q), torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    smha.packed_attention(q, k, v, lengths, out=out, workspace=workspace, stream=torch.cuda.current_stream().cuda_stream)
    assert torch.equal(out, want)
    if need:
        with pytest.raises(smha.SmhaError):
            smha.packed_attention(q, k, v, lengths, out=out, workspace=workspace[:-16])
    with pytest.raises(ValueError):
        smha.packed_attention(q, k, v, lengths, stream=side.cuda_stream)
    # an output of other strides
    wide = torch.zeros(2, 2, 8, 128, dtype=q.dtype, device="cuda")
    into = wide[..., :64].transpose(1, 2)
    assert smha.packed_attention(q, k, v, lengths, out=into) is into and torch.equal(into, want) and bool((wide[..., 64:] == 0).all())
    kn, vn = new_tokens(2, 2, 3, 64, torch.float16)
    a, b = smha.packed_cache(2, 2, Sk, 64), smha.packed_cache(2, 2, Sk, 64)
    one = smha.packed_write(kn, vn, *a, lengths, values=True)
    two = smha.packed_write(kn, vn, *b, lengths, values=True, stream=torch.cuda.current_stream())
    assert all(torch.equal(x, y) for x, y in zip((*a, *one), (*b, *two)))


@pytest.mark.gpu
def test_results_do_not_depend_on_the_order_of_workgroups():
    k, v = filled(5, 2, 6000, 128)
    for H, T in ((8, 1), (16, 3), (16, 8), (16, 60)):
        q = queries(5, H, T, 128, torch.float16)
        lengths = int32([6000, 5, 3000, 1, 4999])
        first = smha.packed_attention(q, k, v, lengths)
        assert all(torch.equal(smha.packed_attention(q, k, v, lengths), first) for _ in range(5))


@pytest.mark.gpu
def test_refusals():
    k, v = smha.packed_cache(2, 2, 40, 64)
    kn, vn = new_tokens(2, 2, 3, 64, torch.float16)
    q = queries(2, 4, 3, 64, torch.float16)
    n = int32([40, 20])
    with pytest.raises(ValueError):
        smha.packed_write(kn.float(), vn.float(), k, v, n)
    with pytest.raises(ValueError):
        smha.packed_write(kn, vn.bfloat16(), k, v, n)
    with pytest.raises(ValueError):
        smha.packed_write(kn[..., :56], vn[..., :56], k, v, n)
    with pytest.raises(ValueError):
        smha.packed_write(kn[:1], vn[:1], k, v, n)
    with pytest.raises(ValueError):
        smha.packed_write(kn, vn, k, v, None)
    with pytest.raises(ValueError):
        smha.packed_write(kn, vn, k, v, n.long())
    with pytest.raises(ValueError):
        smha.packed_write(kn, vn, k, v, n, offsets=n[:1])
    with pytest.raises(ValueError):
        smha.packed_write(kn, vn, k.to(torch.int8), v.to(torch.int8), n)
    with pytest.raises(ValueError):
        smha.packed_write(kn, vn, k[..., :39], v[..., :39], n)         # no row has as many bytes
    with pytest.raises(ValueError):
        smha.packed_write(kn, vn, k[:1].expand_as(k), v, n)            # sequences in one place
    with pytest.raises(smha.SmhaError):
        smha.packed_write(kn, vn, k, k, n)
    overlapping = torch.zeros(2000, dtype=torch.uint8, device="cuda").as_strided((2, 2, 9, 40), (440, 44, 44, 1))
    with pytest.raises(smha.SmhaError):
        smha.packed_write(kn, vn, overlapping, v[:, :, :9], n)         # heads a key apart
    with pytest.raises(ValueError):
        smha.packed_write(kn.clone().requires_grad_(), vn, k, v, n)    # its gradient would be lost
    with torch.no_grad():
        smha.packed_write(kn.clone().requires_grad_(), vn, k, v, n)
    with torch.autograd.forward_ad.dual_level():
        dual = torch.autograd.forward_ad.make_dual(kn.float(), kn.float()).to(torch.float16)
        with pytest.raises(NotImplementedError):
            smha.packed_write(dual, vn, k, v, n)
        dual = torch.autograd.forward_ad.make_dual(q.float(), q.float()).to(torch.float16)
        with pytest.raises(NotImplementedError):
            smha.packed_attention(dual, k, v, n)
    misplaced = torch.zeros(3, 2, 40, 42, dtype=torch.uint8, device="cuda")[:2, :, :, 2:]
    with pytest.raises(smha.SmhaError):
        smha.packed_read(misplaced, misplaced, n)                      # not whole words apart
    with pytest.raises(ValueError):
        smha.packed_read(k, v, n, dtype=torch.float64)
    with pytest.raises(ValueError):
        smha.packed_read(k, v, n, tokens=-1)
    with pytest.raises(smha.SmhaError):
        smha.packed_read(k, v, n, tokens=0)
    with pytest.raises(ValueError):
        smha.packed_read(k, v, n, out=(torch.empty(2, 2, 40, 64, device="cuda"),) * 2)
    same = torch.empty(2, 2, 40, 64, dtype=torch.float16, device="cuda")
    with pytest.raises(smha.SmhaError):
        smha.packed_read(k, v, n, out=(same, same))
    with pytest.raises(ValueError):
        smha.packed_attention(q[:, :3], k, v, n)
    with pytest.raises(ValueError):
        smha.packed_attention(q.float(), k, v, n)
    with pytest.raises(ValueError):
        smha.packed_attention(q, k, v, n, window=-1)
    with pytest.raises(ValueError):
        smha.packed_attention(q.clone().requires_grad_(), k, v, n)
    with pytest.raises(ValueError):
        smha.cache_attention(q, k, v, n)                               # (of 16-bit caches)
    with pytest.raises(ValueError):
        smha.packed_attention(q, k, v.cpu(), n)
    with pytest.raises(ValueError):
        smha.packed_cache(1, 1, 1, 64, device="cpu")
    assert smha.packed_attention(q, k, v, n).shape == q.shape


# What the C ABI says, on the CPU: status 1 invalid, 2 unsupported, 3 shape.

def abi():
    import ctypes as C
    from paper_2506_06095_amd.binding import _load
    return C, _load(), C.c_void_p(4096), C.c_void_p(8192)


def i64(C, *values):
    return (C.c_int64 * len(values))(*values)


def test_the_abi_refuses_writes():
    C, lib, p, q = abi()

    def status(kn=p, k=p, v=q, kv=None, vv=None, n=p, B=2, Hkv=2, T=3, Sk=40, d=64, dtype=0, kns=None, ks=None):
        return lib.smha_packed_write(kn, p, k, v, kv, vv, n, None, B, Hkv, T, Sk, d, dtype, kns, None, ks, None, None)

    for kw in (dict(kn=None), dict(k=None), dict(n=None), dict(v=p), dict(kv=p), dict(vv=p), dict(B=0), dict(Hkv=0), dict(T=0), dict(Sk=0), dict(B=-1), dict(T=-2 ** 31)):
        assert status(**kw) == 1, kw
    for kw in (dict(d=0), dict(d=12), dict(d=136), dict(dtype=2), dict(T=1 << 27), dict(Sk=1 << 27), dict(Sk=1 << 26), dict(B=1 << 24, Hkv=2), dict(B=1 << 14, Hkv=1 << 10, T=16),
               dict(kn=C.c_void_p(4104)), dict(k=C.c_void_p(4098)), dict(kv=p, vv=C.c_void_p(4104)),
               dict(ks=i64(C, 3200, 1600, 36)),          # rows over one another
               dict(ks=i64(C, 3200, 40, 40)),            # heads over rows
               dict(ks=i64(C, 3202, 1600, 40)),          # not whole words
               dict(ks=i64(C, 0, 1600, 40)),             # sequences in one place
               dict(ks=i64(C, -3200, 1600, 40)), dict(ks=i64(C, 1 << 40, 1 << 36, 1 << 31)), dict(ks=i64(C, 1 << 62, 1 << 62, 1 << 62)),
               dict(kns=i64(C, 384, 192, 60)), dict(kns=i64(C, 384, 190, 64)), dict(kns=i64(C, 384, -192, 64)), dict(kns=i64(C, 384, 192, 1 << 30))):
        assert status(**kw) == 2, kw


def test_the_abi_refuses_reads():
    C, lib, p, q = abi()

    def status(k=p, ko=p, vo=q, n=p, B=2, Hkv=2, T=3, Sk=40, d=64, dtype=0, ks=None, os=None):
        return lib.smha_packed_read(k, q, ko, vo, n, None, B, Hkv, T, Sk, d, dtype, ks, None, os, None, None)

    for kw in (dict(k=None), dict(ko=None), dict(vo=p), dict(n=None), dict(T=0)):
        assert status(**kw) == 1, kw
    for kw in (dict(d=20), dict(dtype=3), dict(ko=C.c_void_p(4104)), dict(k=C.c_void_p(4097)), dict(ks=i64(C, 3200, 1600, 20)), dict(os=i64(C, 384, 0, 64)),
               dict(os=i64(C, 384, 192, 68)), dict(dtype=2, os=i64(C, 384, 192, 66)), dict(dtype=2, os=i64(C, 1 << 40, 1 << 34, 1 << 28))):
        assert status(**kw) == 2, kw


def test_the_abi_refuses_attention():
    C, lib, p, q = abi()

    def status(Q=p, k=p, o=p, n=p, B=2, H=4, Hkv=2, T=3, Sk=40, d=64, dtype=0, qs=None, ks=None, os=None, window=0, n_sink=0, ws=None, size=0):
        return lib.smha_packed_forward(Q, k, q, o, n, B, H, Hkv, T, Sk, d, dtype, qs, ks, None, os, window, n_sink, 0.0, ws, size, None)

    for kw in (dict(Q=None), dict(k=None), dict(o=None), dict(n=None), dict(B=0), dict(H=0), dict(T=0), dict(window=-1), dict(n_sink=-1),
               dict(Sk=20000), dict(Sk=20000, size=1 << 30), dict(Sk=20000, ws=p, size=100)):   # a workspace is needed
        assert status(**kw) == 1, kw
    assert status(H=5) == 3
    for kw in (dict(d=4), dict(dtype=2), dict(Q=C.c_void_p(4104)), dict(o=C.c_void_p(4104)), dict(k=C.c_void_p(4098)), dict(ws=C.c_void_p(4104), size=16), dict(T=1 << 27),
               dict(B=1 << 20, H=32, Hkv=32), dict(T=1 << 22, H=4), dict(os=i64(C, 0, 192, 64)), dict(os=i64(C, 768, 64, 64)), dict(qs=i64(C, 768, 192, 68)), dict(ks=i64(C, 3200, 1600, 42))):
        assert status(**kw) == 2, kw
    need = C.c_size_t(77)
    assert lib.smha_packed_workspace(2, 4, 2, 3, 20000, 64, 0, 0, None) == 1
    assert lib.smha_packed_workspace(2, 5, 2, 3, 20000, 64, 0, 0, C.byref(need)) == 3 and need.value == 77
    assert lib.smha_packed_workspace(2, 4, 2, 3, 100, 64, 0, 0, C.byref(need)) == 0 and need.value == 0
    assert lib.smha_packed_workspace(2, 4, 2, 3, 20000, 64, 0, 0, C.byref(need)) == 0 and 0 < need.value < 1 << 24


def test_workspaces_stay_small():
    """What a call needs is bounded by what the chip holds at once, whatever the sizes are."""
    for B, H, Hkv, T, Sk in ((1, 8, 8, 1, 1 << 24), (64, 64, 8, 1, 1 << 17), (4096, 16, 1, 1, 1 << 14), (64, 64, 1, 100, 1 << 14), (1, 128, 1, 1, 1 << 24)):
        assert smha.smha_packed_workspace(B, H, Hkv, T, Sk, 128) < 256 << 20
