"""Attention on a cache held in 4 bits where one key has nearly all of the weight and very many others share what is left: the first key of a text often takes
that part, and outputs are then sums of weights that are small beside the largest.

Tolerance: as in test_packed.py, u |O| (the output's rounding) + F sum_j P |V| (sums and exponentials in 32 bits), and for the probabilities' rounding to
binary16 2^-11 P + 2^-32 a key.  They are stored times 2^7, relative to a reference that is no larger than the row's largest score, so that they add up to 2^7
at least: half a step of binary16 is 2^-11 of a normal value, and 2^-25 of others, which is 2^-32 of the sum.  The largest is 2^4 over the reference's, and so
2^11, and binary16 holds 2^15.99.
"""
import math

import pytest

torch = pytest.importorskip("torch")

import paper_2506_06095_amd as smha  # noqa: E402
from test_packed import F, TYPES, check, int32, row_bytes, unpack_rows  # noqa: E402


def dominated(B, H, Hkv, T, Sk, d, dtype, seed=1):
    """A cache whose first key, whose value is 0, is 2^21 to 2^31 times as heavy as each of the others, whose values are 0.5 to 1.5; scale: log(2)."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    keys = torch.zeros(B, Hkv, Sk, d, dtype=torch.float16, device="cuda")
    values = torch.rand(B, Hkv, Sk, d, generator=gen, device="cuda").add_(0.5).to(torch.float16)
    keys[..., 0] = -10 * torch.rand(B, Hkv, Sk, generator=gen, device="cuda").to(torch.float16)  # (in powers of two below 2^-21)
    keys[:, :, 0, 0] = 0
    keys[:, :, 1:, 32 % d] = -21
    values[:, :, 0] = 0
    k, v = smha.packed_cache(B, Hkv, Sk, d)
    smha.packed_write(keys, values, k, v, int32([Sk] * B))
    q = torch.zeros(B, H, T, d, dtype=dtype, device="cuda")
    q[..., 0] = 1
    q[..., 32 % d] = 1
    return q, k, v


def formula(q, k, v, scale):
    """(out, its bound) in 64 bits, on the values that the rows stand for."""
    (B, H, T, d), (Hkv, Sk) = q.shape, k.shape[1:3]
    u = torch.finfo(q.dtype).eps / 2
    z = 2.0 ** -25 if q.dtype == torch.float16 else 0.0
    seen = torch.arange(Sk)[None, :] <= torch.arange(T)[:, None] + Sk - T
    out, tol = torch.zeros(q.shape, dtype=torch.float64), torch.zeros(q.shape, dtype=torch.float64)
    for b in range(B):
        for c in range(Hkv):
            K, V = (torch.from_numpy(unpack_rows(t[b, c].cpu().numpy(), d)) for t in (k, v))
            for h in range(c * (H // Hkv), (c + 1) * (H // Hkv)):
                P = torch.softmax((q[b, h].cpu().double() @ K.T * scale).masked_fill(~seen, -math.inf), 1)
                out[b, h] = P @ V
                tol[b, h] = torch.where(seen, (2.0 ** -11 + F) * P + 2.0 ** -32, 0.0) @ V.abs()
    return out, tol * (1 + u) + u * out.abs() + z


@pytest.mark.gpu
@TYPES
@pytest.mark.parametrize("B, H, Hkv, T, Sk, d", [
    (1, 256, 256, 1, 8000, 64),    # a row a key head, whole
    (1, 256, 256, 1, 2000, 128),
    (1, 256, 256, 20, 3000, 64),   # 20 rows
    (1, 256, 256, 50, 3000, 64),   # 50
    (1, 256, 256, 100, 3000, 64),  # 100
    (1, 4, 1, 1, 60000, 64),       # cut
    (2, 4, 1, 30, 9000, 128),
], ids=str)
def test_small_weights_are_not_lost(B, H, Hkv, T, Sk, d, dtype):
    assert row_bytes(d) == smha.smha_packed_row(d)
    q, k, v = dominated(B, H, Hkv, T, Sk, d, dtype)
    want, bound = formula(q, k, v, math.log(2))
    check(smha.packed_attention(q, k, v, int32([Sk] * B), scale=math.log(2)), want, bound)


@pytest.mark.gpu
@TYPES
@pytest.mark.parametrize("T, Sk", [(1, 500), (1, 9000), (20, 500), (20, 9000), (50, 900), (100, 900)])
@pytest.mark.parametrize("size", [2.0 ** 20, 2.0 ** 22, 2.0 ** 24])
def test_scores_that_32_bits_hold_in_whole_steps(T, Sk, size, dtype):
    """Scores up to 2^26 in powers of two, of which 32 bits leave whole numbers: outputs stay averages of the values (their weights, relative to a reference that is a few steps
    off, have to fit binary16)."""
    gen = torch.Generator(device="cuda").manual_seed(7)
    B, H, Hkv, d = 2, 4, 2, 64
    k, v = smha.packed_cache(B, Hkv, Sk, d)
    keys, values = (torch.randn(B, Hkv, Sk, d, generator=gen, device="cuda").to(torch.float16) for _ in range(2))
    smha.packed_write(keys, values, k, v, int32([Sk] * B))
    q = torch.randn(B, H, T, d, generator=gen, device="cuda").to(dtype)
    out = smha.packed_attention(q, k, v, int32([Sk] * B), scale=size / (8 * math.log2(math.e) * 4)).double()
    top = smha.packed_read(k, v, int32([Sk] * B))[1].double()
    low, high = (t.repeat_interleave(H // Hkv, 1)[:, :, None] for t in (top.amin(2), top.amax(2)))
    slack = (2.0 ** -11 + torch.finfo(dtype).eps / 2 + F) * torch.maximum(low.abs(), high.abs())
    assert bool(((out >= low - slack) & (out <= high + slack)).all())


@pytest.mark.gpu
@TYPES
@pytest.mark.parametrize("B, H, Hkv, T, Sk, d, window, n_sink, lengths", [
    (2, 4, 2, 1, 700, 96, 0, 0, [700, 33]),
    (1, 8, 1, 3, 5000, 96, 1000, 5, [4999]),
    (2, 6, 2, 20, 900, 96, 0, 0, [900, 450]),
    (1, 8, 2, 50, 800, 96, 300, 40, [800]),
    (2, 4, 2, 1, 700, 88, 0, 0, [700, 1]),
    (1, 4, 1, 40, 500, 112, 0, 0, [499]),
    (1, 4, 2, 9, 500, 48, 100, 0, [500]),
    (1, 4, 1, 40, 500, 24, 0, 0, [500]),
    (1, 3, 1, 2, 500, 120, 0, 0, [499]),
], ids=str)
def test_heads_of_other_widths(B, H, Hkv, T, Sk, d, window, n_sink, lengths, dtype):
    """(The bound of test_packed.py, which is the wider one.)"""
    from test_packed import filled, queries, reference
    k, v = filled(B, Hkv, Sk, d)
    q = queries(B, H, T, d, dtype)
    want, bound = reference(q, k, v, lengths, window, n_sink)
    check(smha.packed_attention(q, k, v, int32(lengths), window=window, n_sink=n_sink), want, bound)
