"""Attention with sinks: what is sharper than the bounds that a whole pass has room for.

Keys of a head that are all alike give equal scores, so that probabilities before the division are exactly 1 and no rounding of theirs is in the way: an
output is a mean, in 32 bits, and what is left of its rounding (O_rest) and of delta = sum dO O can be seen.  u: half a step of the inputs' type; z: half
the smallest step of binary16; F = 2e-5 for sums, exponentials and the log-sum-exp in 32 bits.
"""
import math

import pytest

torch = pytest.importorskip("torch")

import paper_2506_06095_amd as smha  # noqa: E402
from paper_2506_06095_amd import sink  # noqa: E402
from test_sink import CASES, F, int32, reference, rounding, tensors, visible  # noqa: E402

TYPES = pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])


def means(B, H, Hkv, Sq, Sk, d, dtype, layout):
    """Inputs whose keys are alike and whose values lie one step or none over a value that they share: outputs lie between two numbers of the type,
    and dP - delta is as small as what rounding O leaves out of delta."""
    q, k, v, g = tensors(B, H, Hkv, Sq, Sk, d, dtype, layout)
    k[:] = k[:, :, :1].clone()
    up = torch.rand(v.shape, generator=torch.Generator(device="cuda").manual_seed(8), device="cuda") < 0.5
    v[:] = torch.where(up, v[:, :, :1].contiguous().view(torch.int16) + 1, v[:, :, :1].contiguous().view(torch.int16)).view(dtype)
    return q, k, v, g


SHAPES = [
    # B, H, Hkv, Sq, Sk, d, window, n_sink, offsets, lengths, layout
    (1, 2, 1, 1, 5, 64, 0, 0, None, None, "bhsd"),
    (2, 4, 2, 130, 130, 64, 9, 2, None, [130, 61], "bhsd"),
    (2, 3, 3, 100, 140, 80, 20, 3, [40, -30], [140, 90], "bshd"),
    (1, 4, 1, 200, 200, 96, 0, 0, None, None, "bshd"),
    (3, 2, 2, 70, 70, 128, 5, 1, None, [0, 1, 70], "bhsd"),
    (1, 4, 2, 90, 90, 32, 30, 4, None, None, "bshd"),
    (5, 8, 4, 300, 300, 80, 12, 2, None, [300, 1, 150, 0, 299], "bhsd"),    # more than 8192 queries, whose dS is multiplied rounded
    (5, 8, 2, 300, 300, 128, 40, 2, None, None, "bshd"),
]


def expected(q, k, v, g, window, n_sink, offsets, lengths, fine):
    """(name: value, bound) in 64 bits.  Bounds: O + O_rest is off by F of its sum and by the rest's own rounding, u^2 |O|, which delta takes on; dS by that, by
    its rounding (twice u, squared, where both halves are multiplied) and z; dQ and dK by their roundings."""
    (B, H, Sq, d), (Hkv, Sk) = q.shape, k.shape[1:3]
    u, z = rounding(q.dtype)
    q, k, v, g = (t.detach().cpu().double() for t in (q, k, v, g))
    zero = torch.zeros_like
    val = {"out": zero(q), "dq": zero(q), "dk": zero(k)}
    tol = {n: zero(t) for n, t in val.items()}
    for b in range(B):
        seen = visible(Sq, Sk, Sk - Sq if offsets is None else offsets[b], Sk if lengths is None else lengths[b], window, n_sink)
        some = seen.any(1)
        for h in range(H):
            c = h * Hkv // H
            Q, G, K, V = q[b, h], g[b, h], k[b, c], v[b, c]
            P = seen.double() / seen.sum(1, keepdim=True).clamp(min=1)
            O = P @ V
            val["out"][b, h], tol["out"][b, h] = O, (F + u * u) * (P @ V.abs()) + z * some[:, None]
            dS = P * (G @ V.T - (G * O).sum(1, keepdim=True))
            mag = (G.abs() @ V.abs().T + (G.abs() * O.abs()).sum(1, keepdim=True))
            e = P * (2 * (F + u * u) * mag + z * G.abs().sum(1, keepdim=True)) + torch.where(seen, (u * u if fine else u) * dS.abs() + z, 0.0)
            val["dq"][b, h], tol["dq"][b, h] = d ** -0.5 * dS @ K, d ** -0.5 * e @ K.abs()
            val["dk"][b, c] += d ** -0.5 * dS.T @ Q
            tol["dk"][b, c] += d ** -0.5 * e.T @ Q.abs()
    for n in ("dq", "dk"):
        tol[n] += u * (val[n].abs() + tol[n]) + z
    return {n: (val[n], tol[n]) for n in val}


def off(got, want):
    """How many bounds of the worst the error is (the largest of all elements; infinite for what is not finite)."""
    got = got.detach().cpu().double()
    value, bound = want
    ratio = torch.where(got == value, 0.0, (got - value).abs() / bound)
    return float(torch.where(torch.isfinite(got), ratio, math.inf).max())


@pytest.mark.gpu
@TYPES
@pytest.mark.parametrize("case", SHAPES, ids=lambda c: "x".join(str(x) for x in c[:8]))
def test_what_rounding_the_output_left_out(case, dtype):
    """O + O_rest is the output in 32 bits, also where O has strides of its own; with it delta, dQ and dK are as exact, and without it they are not."""
    B, H, Hkv, Sq, Sk, d, window, n_sink, offsets, lengths, layout = case
    q, k, v, g = means(B, H, Hkv, Sq, Sk, d, dtype, layout)
    want = expected(q, k, v, g, window, n_sink, offsets, lengths, B * H * Sq <= 8192)
    at, n = int32(offsets), int32(lengths)
    for out in (torch.full((B, H, Sq, d), math.nan, dtype=dtype, device="cuda"), torch.full((B, Sq, H, d + 8), math.nan, dtype=dtype, device="cuda")[..., :d].transpose(1, 2)):
        rest, lse = torch.full((B, H, Sq, d), math.nan, dtype=dtype, device="cuda"), torch.empty(B, H, Sq, device="cuda")
        smha.smha_sink_forward(q, k, v, out, lse, window, n_sink, at, n, O_rest=rest)
        assert off(out.double() + rest.double(), want["out"]) <= 1
        grads = [torch.full_like(t, math.nan) for t in (q, k, v)]
        smha.smha_sink_backward(q, k, v, out, lse, g, *grads, window, n_sink, at, n, O_rest=rest)
        assert off(grads[0], want["dq"]) <= 1 and off(grads[1], want["dk"]) <= 1
        if Sq > 1:
            assert off(out, want["out"]) > 1  # (the bounds tell: what rounding leaves out is more than they allow)
            smha.smha_sink_backward(q, k, v, out, lse, g, *grads, window, n_sink, at, n)
            assert off(grads[0], want["dq"]) > 1


@pytest.mark.gpu
@TYPES
@pytest.mark.parametrize("native", [True, False], ids=["native", "python"])
@pytest.mark.parametrize("case", SHAPES, ids=lambda c: "x".join(str(x) for x in c[:8]))
def test_a_pass_of_autograd_keeps_it(monkeypatch, case, dtype, native):
    if not native:
        monkeypatch.setattr(sink, "_call", lambda *args: None)
    B, H, Hkv, Sq, Sk, d, window, n_sink, offsets, lengths, layout = case
    q, k, v, g = means(B, H, Hkv, Sq, Sk, d, dtype, layout)
    want = expected(q, k, v, g, window, n_sink, offsets, lengths, B * H * Sq <= 8192)
    x = [t.requires_grad_() for t in (q, k, v)]
    dq, dk, _ = torch.autograd.grad(smha.sink_attention(*x, window, n_sink, offsets=int32(offsets), lengths=int32(lengths)), x, g)
    assert off(dq, want["dq"]) <= 1 and off(dk, want["dk"]) <= 1


@pytest.mark.gpu
@pytest.mark.parametrize("case", CASES, ids=lambda c: "x".join(str(x) for x in c[:8]))
def test_lse_is_minus_infinity_where_a_query_sees_nothing(case):
    """And nowhere else, where it is within its bound."""
    B, H, Hkv, Sq, Sk, d, window, n_sink, offsets, lengths, layout = case
    q, k, v, g = tensors(B, H, Hkv, Sq, Sk, d, torch.float16, layout)
    value, bound = reference(q, k, v, g, window, n_sink, offsets, lengths, 0.0)["lse"]
    lse = torch.full((B, H, Sq), math.nan, device="cuda")
    smha.smha_sink_forward(q, k, v, torch.empty_like(q), lse, window, n_sink, int32(offsets), int32(lengths))
    lse, empty = lse.cpu().double(), torch.isneginf(value)
    assert bool((lse[empty] == -math.inf).all())
    assert bool(((lse - value).abs() <= bound)[~empty].all())


@pytest.mark.gpu
@TYPES
@pytest.mark.parametrize("d", [64, 128])
def test_both_halves_of_ds_make_one_number(dtype, d):
    """Queries of zeros see three keys of equal weight, one of which is not zero: a row of dQ is one dS times one key and shows dS's error beside its own
    rounding.  dS to twice its digits is off by u^2 and by what 32 bits leave of dP - delta; one step of the type, as where the halves are taken from two
    roundings of a tie (one value in 2^14), would be up to two u.  64 x 128 queries, twelve times."""
    (u, z), H, S = rounding(dtype), 64, 128
    for seed in range(12):
        q, k, v, g = tensors(1, H, H, S, S, d, dtype, seed=100 + seed)
        q.zero_()
        k[:, :, 1::3] = k[:, :, 2::3] = 0
        x = [t.requires_grad_() for t in (q, k, v)]
        (dq,) = torch.autograd.grad(smha.sink_attention(*x, 3), x[:1], g)
        K, V, G = (t.detach().cpu().double() for t in (k, v, g))
        seen = visible(S, S, 0, S, 3, 0)
        P = seen.double() / seen.sum(1, keepdim=True)
        O = P @ V
        dS = P * (G @ V.mT - (G * O).sum(-1, keepdim=True))
        e = P * 2 * (F + u * u) * (G.abs() @ V.abs().mT + (G * O).abs().sum(-1, keepdim=True)) + torch.where(seen, u * u * dS.abs() + 2 * z, 0.0)
        dQ, bound = d ** -0.5 * dS @ K, d ** -0.5 * e @ K.abs()
        assert off(dq, (dQ, bound + u * (dQ.abs() + bound) + z)) <= 1, seed


@pytest.mark.gpu
@TYPES
@pytest.mark.parametrize("case", [
    (1, 2, 1, 96, 20000, 64, 0, 0),        # weights of 5e-5, which binary16 holds with fewer digits (z)
    (1, 2, 2, 200, 6000, 128, 4096, 128),
    (1, 4, 1, 3000, 3000, 64, 1024, 4),
], ids=str)
def test_gradients_over_long_windows(case, dtype):
    B, H, Hkv, Sq, Sk, d, window, n_sink = case
    q, k, v, g = tensors(B, H, Hkv, Sq, Sk, d, dtype)
    want = reference(q, k, v, g, window, n_sink, None, None, 0.0)
    x = [t.requires_grad_() for t in (q, k, v)]
    out = smha.sink_attention(*x, window, n_sink)
    for name, got in zip(("out", "dq", "dk", "dv"), (out, *torch.autograd.grad(out, x, g))):
        worst = off(got, want[name])
        print(name, worst, float((got.detach().cpu().double() - want[name][0]).norm() / want[name][0].norm()))
        assert worst <= 1, name
