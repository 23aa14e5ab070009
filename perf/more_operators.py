"""A cache held in 4 bits: keys and values packed as they are written, read back, and attended to. The calls whose speed is tracked, their inputs, and
what they compute in plain operations.

A packed row stands for the d columns of one key or value. Its columns are taken 32 at a time (the last group may be shorter); each group has a step s and a
base m, both binary16, and a code c of 4 bits for each column, which stands for the binary16 nearest to c s + m. The row is bytes: (s, m) of every
group, then the codes, eight columns to a 32-bit word, columns 0, 2, 4, 6 in its lower half and 1, 3, 5, 7 in its upper, from the lowest bits on.

Kinds of case:

  write    keys and values of new tokens go into their slots; what they stand for from then on comes back
  read     slots of the cache as 16-bit keys and values
  attend   new tokens of every sequence (one, a few, or a chunk of a prompt) against its packed cache, all of it or a window and sinks
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False  # run() calls the framework's operators, not their plain form

_TORCH = {"f16": torch.float16, "bf16": torch.bfloat16}
_MOST = 65280.0  # values of a larger magnitude are packed as this


def _case(kind, B, H, Hkv, d, dtype, **kw):
    case = dict(kind=kind, B=B, H=H, Hkv=Hkv, d=d, dtype=dtype, T=1, Sk=0, window=0, n_sink=0, ragged=0.0, aligned="right", layout="bhsd", len_seed=1)
    return dict(case, **kw)


def listed():
    return [
        # the token that one short chat has just made: latency
        _case("write", 1, 2, 2, 64, "f16", Sk=256, name="write_tiny"),
        # one token each of a full batch, caches of uneven length
        _case("write", 64, 8, 8, 128, "bf16", Sk=4096, ragged=0.9, name="write_step"),
        # prompts of a small model, of odd length and head size, each at its cache's end
        _case("write", 3, 12, 12, 80, "f16", T=1537, Sk=2000, ragged=0.4, name="write_odd"),
        # four long prompts at once, padded behind, their tensors straight from a projection
        _case("write", 4, 8, 8, 128, "bf16", T=8192, Sk=8192, ragged=0.3, aligned="left", layout="bshd", name="write_prompt"),
        # a few hundred keys back, for a look at them or for another kind of attention
        _case("read", 2, 4, 4, 64, "f16", T=333, Sk=512, ragged=0.5, name="read_small"),
        # whole caches back
        _case("read", 4, 8, 8, 128, "bf16", T=16384, Sk=16384, ragged=0.3, name="read_caches"),
        # one token of one short sequence: latency
        _case("attend", 1, 8, 2, 64, "f16", Sk=256, name="attend_tiny"),
        # one token each of a full batch on caches of uneven length
        _case("attend", 32, 32, 8, 128, "bf16", Sk=8192, ragged=0.9, name="attend_batch"),
        # one token each of two long documents
        _case("attend", 2, 32, 8, 128, "f16", Sk=65536, name="attend_long"),
        # three tokens each (a guess and its check) within a window and a few sinks, an odd head size
        _case("attend", 16, 20, 4, 80, "bf16", T=3, Sk=16384, window=2048, n_sink=4, ragged=0.5, layout="bshd", name="attend_window"),
        # eight drafted tokens each, eight heads on every key head: 64 rows read the same keys
        _case("attend", 8, 64, 8, 128, "f16", T=8, Sk=8192, ragged=0.5, name="attend_draft"),
        # a chunk of two long prompts against what is cached of them (the largest call)
        _case("attend", 2, 32, 8, 128, "bf16", T=1024, Sk=16384, ragged=0.3, name="attend_chunk"),
    ]


def _loguniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """A length in [lo, hi], log-uniform; half of them a multiple of 64, the rest as they fall."""
    n = _loguniform(rng, lo, hi)
    return max(lo, n // 64 * 64) if rng.random() < 0.5 else n


def draw(rng):
    top = {c["name"]: work(c) for c in listed()}
    flops, nbytes = top["attend_chunk"]["flops"], top["read_caches"]["bytes"]
    while True:
        kind = rng.choice(["write", "write", "read", "attend", "attend", "attend", "attend"])
        H, Hkv = rng.choice([(2, 2), (8, 2), (12, 12), (16, 4), (16, 16), (20, 4), (32, 8), (16, 1), (64, 8)])
        d = rng.choice([64, 64, 128, 128, 128, 32, 72, 80, 96])
        B, Sk = _loguniform(rng, 1, 64), _size(rng, 64, 65536)
        kw = dict(layout="bshd" if rng.random() < 0.3 else "bhsd", ragged=rng.choice([0.0, 0.3, 0.9]), len_seed=rng.randrange(1, 1 << 30))
        if kind == "attend":
            T = min(rng.choice([1, 1, 1, 2, 3, 5, 8, _loguniform(rng, 9, 64), _size(rng, 64, 1024)]), Sk)
            if rng.random() < 0.3:
                kw.update(window=_size(rng, 32, 4096), n_sink=rng.choice([0, 4, 64]))
        elif kind == "write":
            T = rng.choice([1, _size(rng, 1, min(Sk, 8192))])
            kw.update(aligned=rng.choice(["left", "right"]))
        else:
            T = _size(rng, 64, Sk)
        case = _case(kind, B, H if kind == "attend" else Hkv, Hkv, d, rng.choice(["f16", "bf16"]), T=T, Sk=Sk, **kw)
        w = work(case)
        # (the plain form holds caches in 64 and all scores in 32 bits)
        if w["flops"] <= flops and w["bytes"] <= nbytes and B * Hkv * Sk * d <= 32 * 8 * 8192 * 128 and B * case["H"] * T * Sk <= 2 * 32 * 1024 * 16384:
            return case


# --- inputs

def _lengths(case):
    """Keys in every sequence (new tokens included)."""
    r = random.Random(case["len_seed"])
    low = max(1 if case["aligned"] == "left" else min(case["T"], case["Sk"]), int(round(case["Sk"] * (1 - case["ragged"]))))
    return [r.randint(low, case["Sk"]) if case["ragged"] else case["Sk"] for _ in range(case["B"])]


def _offsets(case):
    """The first new token's slot in every sequence."""
    return [0 if case["aligned"] == "left" or case["kind"] == "read" else n - case["T"] for n in _lengths(case)]


def _row(d):
    """Bytes of a packed row."""
    return (d + 31) // 32 * 4 + d // 2


def _tensor(case, heads, rows, g, keys=False):
    """Normal values; keys have a few columns that are far larger than the others, or far from zero."""
    B, d = case["B"], case["d"]
    shape = (B, rows, heads, d) if case["layout"] == "bshd" else (B, heads, rows, d)
    x = torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)
    if keys:
        pick = torch.rand((2, d), generator=g, device="cuda")
        x = x * (1 + 3 * (pick[0] > 0.95)) + 4 * torch.randn(d, generator=g, device="cuda") * (pick[1] > 0.95)
    x = x.to(_TORCH[case["dtype"]])
    return x.transpose(1, 2) if case["layout"] == "bshd" else x


def _filled(case, g, keys):
    """A cache [B, Hkv, Sk, row] of packed values."""
    B, Hkv, Sk, d = (case[n] for n in ("B", "Hkv", "Sk", "d"))
    cache = torch.empty((B, Hkv, Sk, _row(d)), dtype=torch.uint8, device="cuda")
    for b in range(B):
        cache[b:b + 1] = _packed(_tensor(dict(case, B=1, layout="bhsd"), Hkv, Sk, g, keys))
    return cache


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    state = {"case": case, "lengths": torch.tensor(_lengths(case), dtype=torch.int32, device="cuda")}
    if case["kind"] == "write":
        shape = (case["B"], case["Hkv"], case["Sk"], _row(case["d"]))
        state["k"], state["v"] = (torch.zeros(shape, dtype=torch.uint8, device="cuda") for _ in range(2))
        state["k_new"], state["v_new"] = _tensor(case, case["Hkv"], case["T"], g, True), _tensor(case, case["Hkv"], case["T"], g)
        if case["aligned"] == "left":
            state["offsets"] = torch.tensor(_offsets(case), dtype=torch.int32, device="cuda")
        return state
    state["k"], state["v"] = _filled(case, g, True), _filled(case, g, False)
    if case["kind"] == "attend":
        state["q"] = _tensor(case, case["H"], case["T"], g)
    return state


# --- one pass

def run(state):
    case = state["case"]
    if own:
        return _run_own(state, case)
    with torch.no_grad():
        return {"write": _plain_write, "read": _plain_read, "attend": _plain_attention}[case["kind"]](state, case)


def _run_own(state, case):
    import paper_2506_06095_amd as smha
    if case["kind"] == "write":
        return smha.packed_write(state["k_new"], state["v_new"], state["k"], state["v"], state["lengths"], offsets=state.get("offsets"), values=True)
    if case["kind"] == "read":
        return smha.packed_read(state["k"], state["v"], state["lengths"], tokens=case["T"], dtype=_TORCH[case["dtype"]])
    return smha.packed_attention(state["q"], state["k"], state["v"], state["lengths"], window=case["window"], n_sink=case["n_sink"])


def _next(h, up):
    """The next larger (or smaller) binary16 of finite ones."""
    bits = h.view(torch.int16)
    away = (h >= 0) if up else (h <= 0)  # from zero
    zero = torch.full_like(bits, 1 if up else -32767)  # the smallest of the other sign, or this one
    return torch.where(h == 0, zero, torch.where(away, bits + 1, bits - 1)).view(torch.float16)


def _packed(x):
    """[..., d] -> [..., row] uint8. (In 64 bits: sums and products of a code, a step and a base are exact there, and so are comparisons.)"""
    d = x.shape[-1]
    G = (d + 31) // 32
    x = x.double().clamp(-_MOST, _MOST)
    if d % 32:
        x = torch.cat([x, x[..., -1:].expand(*x.shape[:-1], 32 - d % 32)], -1)
    x = x.reshape(*x.shape[:-1], G, 32)
    lo, hi = x.amin(-1), x.amax(-1)
    m = (lo + 0.0).half()
    m = torch.where(m.double() > lo, _next(m, False), m)
    s = ((hi - m.double()) / 15).half()
    s = torch.where(15 * s.double() + m.double() < hi, _next(s, True), s)
    down = _next(s, False)
    s = torch.where((s > 0) & (15 * down.double() + m.double() >= hi), down, s)
    sd, md = s.double()[..., None], m.double()[..., None]
    code = torch.zeros_like(x, dtype=torch.int32)
    for k in range(15):
        code += (x >= md + (k + 0.5) * sd) & (sd > 0)
    code = code.reshape(*code.shape[:-2], G * 32)[..., :d].reshape(*code.shape[:-2], d // 8, 4, 2)
    shift = torch.tensor([[4 * i, 16 + 4 * i] for i in range(4)], device=x.device)
    word = (code.long() << shift).sum((-1, -2))
    word = torch.where(word >= 1 << 31, word - (1 << 32), word).to(torch.int32)
    head = torch.stack([s, m], -1).reshape(*s.shape[:-1], 2 * G)
    return torch.cat([head.view(torch.uint8), word.contiguous().view(torch.uint8)], -1)


def _values(rows, d):
    """[..., row] uint8 -> [..., d] of the binary16 values that they stand for, in 32 bits."""
    G = (d + 31) // 32
    head = rows[..., :4 * G].contiguous().view(torch.float16).double().reshape(*rows.shape[:-1], G, 2)
    word = rows[..., 4 * G:].contiguous().view(torch.int32)
    shift = torch.tensor([4 * (i // 2) + 16 * (i % 2) for i in range(8)], device=rows.device, dtype=torch.int32)
    code = ((word[..., None] >> shift) & 15).reshape(*rows.shape[:-1], d)
    group = torch.arange(d, device=rows.device) // 32
    x = head[..., 0][..., group].mul_(code).add_(head[..., 1][..., group])
    # one rounding to 11 digits, steps of 2^-24 at least (a cast goes through 32 bits, and may round twice)
    step = ((torch.frexp(x).exponent - 11).clamp_min(-24).long() + 1023 << 52).view(torch.float64)  # (2 to that, by its digits)
    return x.div_(step).round_().mul_(step).float()


def _plain_write(state, case):
    B, T, d = case["B"], case["T"], case["d"]
    lengths = state["lengths"]
    at = state["offsets"] if "offsets" in state else lengths - T
    slot = at[:, None] + torch.arange(T, device="cuda")
    there = (slot >= 0) & (slot < lengths[:, None])
    b, t = there.nonzero(as_tuple=True)
    out = []
    for new, cache in ((state["k_new"], state["k"]), (state["v_new"], state["v"])):
        rows = _packed(new)
        cache[b, :, slot[b, t]] = rows[b, :, t]
        values = torch.zeros(new.shape, dtype=torch.float32, device="cuda")
        values[b, :, t] = _values(rows[b, :, t], d)
        out.append(values.to(new.dtype))
    return tuple(out)


def _plain_read(state, case):
    T, d = case["T"], case["d"]
    there = (torch.arange(T, device="cuda") < state["lengths"][:, None])[:, None, :, None]
    return tuple((_values(state[n][:, :, :T], d) * there).to(_TORCH[case["dtype"]]) for n in ("k", "v"))


def _plain_attention(state, case):
    B, H, Hkv, T, Sk, d = (case[n] for n in ("B", "H", "Hkv", "T", "Sk", "d"))
    G = H // Hkv
    q = state["q"].float().reshape(B, Hkv, G * T, d)
    s = (q @ _values(state["k"], d).mT).reshape(B, Hkv, G, T, Sk).mul_(d ** -0.5)
    p = (state["lengths"][:, None] - T + torch.arange(T, device="cuda"))[:, :, None]
    j = torch.arange(Sk, device="cuda")
    seen = j <= p
    if case["window"]:
        seen &= (p - j < case["window"]) | (j < case["n_sink"])
    s.masked_fill_(~seen[:, None, None], -math.inf)
    s -= s.amax(-1, keepdim=True).clamp_min(torch.finfo(torch.float32).min)
    s.exp_()
    s /= s.sum(-1, keepdim=True).clamp_min(torch.finfo(torch.float32).tiny)
    return (s.reshape(B, Hkv, G * T, Sk) @ _values(state["v"], d)).reshape(B, H, T, d).to(_TORCH[case["dtype"]])


# --- what a pass cannot do without

def work(case):
    B, H, Hkv, T, Sk, d = (case[n] for n in ("B", "H", "Hkv", "T", "Sk", "d"))
    lengths, row, window, sink = _lengths(case), _row(d), case["window"], case["n_sink"]
    if case["kind"] == "write":
        tokens = sum(max(0, min(n, at + T) - max(at, 0)) for n, at in zip(lengths, _offsets(case)))
        return {"bytes": 2 * Hkv * (tokens * (2 * d + row) + B * T * 2 * d), "flops": 0}
    if case["kind"] == "read":
        return {"bytes": 2 * Hkv * (sum(min(n, T) for n in lengths) * row + B * T * 2 * d), "flops": 0}
    pairs = keys = 0
    for n in lengths:
        p = np.arange(max(n - T, 0), n, dtype=np.int64)
        first = np.maximum(p - (window or Sk + 1) + 1, 0)
        pairs += int((p + 1 - first + np.minimum(first, sink)).sum())
        keys += int(n - first[0] + min(first[0], sink))
    return {"bytes": 2 * row * Hkv * keys + 2 * 2 * d * B * H * T, "flops": 4 * d * H * pairs}


# --- the definition in 64 bits

def exact(case, seed):
    with torch.no_grad():
        state = prepare(case, seed)
        return {"write": _exact_write, "read": _exact_read, "attend": _exact_attention}[case["kind"]](state, case)


def _unpack64(rows, d):
    """The values of packed rows (a uint8 array), one column of 32 at a time."""
    G = (d + 31) // 32
    out = np.empty((*rows.shape[:-1], d))
    word = np.ascontiguousarray(rows[..., 4 * G:]).view("<u4")
    head = np.ascontiguousarray(rows[..., :4 * G]).view("<f2").astype(np.float64)
    for c in range(d):
        code = word[..., c // 8] >> np.uint32(4 * (c % 8 // 2) + 16 * (c % 2)) & np.uint32(15)
        out[..., c] = (code * head[..., c // 32 * 2] + head[..., c // 32 * 2 + 1]).astype(np.float16)
    return out


def _round64(x):
    """What a group of columns (an array [..., up to 32]) stands for once it is packed."""
    x = np.clip(x, -_MOST, _MOST)
    lo, hi = x.min(-1, keepdims=True), x.max(-1, keepdims=True)
    m = lo.astype(np.float16)
    m = np.where(m > lo, np.nextafter(m, np.float16(-np.inf)), m).astype(np.float64)
    s = ((hi - m) / 15).astype(np.float16)
    s = np.nextafter(s, np.float16(0))  # no larger than the one that is wanted, and no more than two below it
    for _ in range(2):
        s = np.where(15 * s.astype(np.float64) + m < hi, np.nextafter(s, np.float16(np.inf)), s)
    s = s.astype(np.float64)
    code = np.clip(np.rint((x - m) / np.where(s > 0, s, 1)), 0, 15)
    code -= x < m + (code - 0.5) * s
    code += (x >= m + (code + 0.5) * s) & (s > 0)
    return (code * s + m).astype(np.float16).astype(np.float64)


def _exact_write(state, case):
    T = case["T"]
    out = []
    for n in ("k_new", "v_new"):
        x = state[n].float().cpu().numpy()
        y = np.zeros(x.shape)
        for b, (length, at) in enumerate(zip(_lengths(case), _offsets(case))):
            t0, t1 = max(0, -at), max(0, min(T, length - at))
            for c in range(0, case["d"], 32):
                y[b, :, t0:t1, c:c + 32] = _round64(x[b, :, t0:t1, c:c + 32].astype(np.float64))
        out.append(torch.from_numpy(y))
    return tuple(out)


def _exact_read(state, case):
    out = []
    for n in ("k", "v"):
        y = np.zeros((case["B"], case["Hkv"], case["T"], case["d"]))
        for b, length in enumerate(_lengths(case)):
            t = min(length, case["T"])
            y[b, :, :t] = _unpack64(state[n][b, :, :t].cpu().numpy(), case["d"])
        out.append(torch.from_numpy(y))
    return tuple(out)


def _exact_attention(state, case):
    B, H, Hkv, T, d = (case[n] for n in ("B", "H", "Hkv", "T", "d"))
    out = torch.zeros((B, H, T, d), dtype=torch.float64, device="cuda")
    for b, n in enumerate(_lengths(case)):
        t0 = max(0, T - n)  # the first token that is there
        i = torch.arange(n - T + t0, n, device="cuda")[:, None]
        j = torch.arange(n, device="cuda")[None, :]
        hidden = j > i
        if case["window"]:
            hidden |= (j <= i - case["window"]) & (j >= case["n_sink"])
        for c in range(Hkv):
            k, v = (torch.from_numpy(_unpack64(state[x][b, c, :n].cpu().numpy(), d)).cuda() for x in ("k", "v"))
            for h in range(c * (H // Hkv), (c + 1) * (H // Hkv)):
                s = torch.where(hidden, -math.inf, state["q"][b, h, t0:].double() @ k.T / math.sqrt(d))
                out[b, h, t0:] = torch.softmax(s, 1) @ v
    return out
