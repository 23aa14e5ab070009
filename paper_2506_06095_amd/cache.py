"""Attention of new tokens on a cache, and eviction from it: binding of smha_cache_*.

Argument checks and allocation only; include/smha.h says what the entry points compute.
"""
from __future__ import annotations

import contextlib
import ctypes as C

import torch

from .binding import SmhaError, _load, native_call
from .sink import _CODES, _check_int, _check_no_tangents, _check_per_sequence, _check_qkv, _handle, _on_device, _strides, _written


_attention = _evict = None  # functions of _smha_torch


def _allocating_on(stream, given):
    """What makes torch allocate for the stream that a call runs on; `given`: nothing has to be allocated."""
    if stream is None or given:
        return contextlib.nullcontext()
    if not isinstance(stream, torch.cuda.Stream):
        raise ValueError("a call on a bare stream handle needs its workspace and outputs")
    return torch.cuda.stream(stream)


def _check_no_gradients(name, *tensors):
    """Gradients would be lost, or leaves written."""
    if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in tensors):
        raise ValueError(f"{name} has no gradients, and writes no tensor that requires them")
    _check_no_tangents(name, *tensors)


def _check_workspace(workspace, like):
    if workspace.dtype != torch.uint8 or workspace.device != like.device or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous uint8 tensor on the same GPU")


def smha_cache_workspace(B: int, H: int, Hkv: int, T: int, Sk: int, P: int, d: int, window: int = 0, n_sink: int = 0, weigh: bool = False) -> int:
    """Bytes of device memory that cache_attention needs."""
    need = C.c_size_t(0)
    st = _load().smha_cache_workspace(B, H, Hkv, T, Sk, P, d, _check_int(window, "window"), _check_int(n_sink, "n_sink"), int(weigh), C.byref(need))
    if st != 0:
        raise SmhaError(st, "smha_cache_workspace")
    return need.value


def cache_attention(q, k, v, lengths, *, window: int = 0, n_sink: int = 0, prefix=None, weights=None, out=None, scale: float = 0.0, workspace=None, stream=None):
    """Attention of the last T tokens of every sequence on its cache: [B,H,T,d] like q.

    q [B,H,T,d]: the new tokens, whose keys and values are in the cache; k, v [B,Hkv,Sk,d], H a multiple of Hkv; float16 or bfloat16, d a
    multiple of 8 up to 128.  lengths: int32 [B] on the GPU, keys of every sequence, the new tokens' included.  Token t of sequence b stands at
    lengths[b] - T + t (below 0: no such token, its output is zero) and sees the keys up to itself: the last `window` of them (0: all) and the
    first `n_sink`.  These are slots of the cache: after cache_evict, which moves keys, a window no longer holds the most recent tokens (without
    a window the order of keys does not matter).
    prefix: (keys, values), each [Hkv,P,d]: tokens before those of every sequence, which all of them see (not with a window).
    weights: float32 [B,Hkv,Sk]; each key's attention, summed over the tokens and the heads that share it, is added to it.
    scale: 0 or less for 1/sqrt(d).  No gradients (sink_attention has them): no tensor given may require any.  Values that a token of the sequence
    sees have to be finite (those before the window, past the length and in the cache's free slots may be anything).  workspace: a uint8 tensor of smha_cache_workspace bytes, by default one is allocated."""
    if out is None and workspace is None and stream is None:  # the native way, for every call that it takes (csrc/torch_binding.cpp)
        global _attention
        if _attention is None:
            _attention = native_call("cache_attention")
        pk, pv = prefix if prefix is not None else (None, None)
        got = _attention(q, k, v, lengths, window, n_sink, pk, pv, weights, float(scale))
        if got is not None:
            if type(got) is int:
                raise SmhaError(got, "smha_cache_forward")
            return got
    _check_qkv(q, k, v)
    _check_no_gradients("cache_attention", q, k, v, *(() if prefix is None else prefix), weights, out)
    (B, H, T, d), (Hkv, Sk) = q.shape, k.shape[1:3]
    if lengths is None:
        raise ValueError("lengths must be given")
    n = _check_per_sequence(lengths, "lengths", q)
    window, n_sink = _check_int(window, "window"), _check_int(n_sink, "n_sink")
    P, pk, pv, pks, pvs = 0, None, None, None, None
    if prefix is not None:
        pk, pv = prefix
        if pk.dim() != 3 or pk.shape != pv.shape or pk.shape[0] != Hkv or pk.shape[2] != d or pk.dtype != q.dtype or pv.dtype != q.dtype:
            raise ValueError("prefix must be a pair of [Hkv,P,d] tensors of q's type")
        if pk.device != q.device or pv.device != q.device:
            raise ValueError("tensors must be on one GPU")
        P = pk.shape[1]
        pks, pvs = _prefix_strides(pk), _prefix_strides(pv)
    ws = None
    if weights is not None:
        if weights.shape != (B, Hkv, Sk) or weights.dtype != torch.float32 or weights.device != q.device or weights.stride(2) != 1:
            raise ValueError("weights must be a float32 [B,Hkv,Sk] tensor on the same GPU, its keys contiguous")
        if not weights.is_contiguous():
            if (B > 1 and weights.stride(0) < Sk) or (Hkv > 1 and weights.stride(1) < Sk):
                raise ValueError("rows of weights must not overlap")
            ws = (C.c_int64 * 2)(weights.stride(0), weights.stride(1))
    if out is not None and (out.shape != q.shape or out.dtype != q.dtype or out.device != q.device):
        raise ValueError("out must be like q")
    with _on_device(q), _allocating_on(stream, workspace is not None and out is not None):
        if out is None:
            out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        if workspace is None:
            workspace = torch.empty(smha_cache_workspace(B, H, Hkv, T, Sk, P, d, window, n_sink, weights is not None), dtype=torch.uint8, device=q.device)
        else:
            _check_workspace(workspace, q)
        st = _load().smha_cache_forward(q.data_ptr(), k.data_ptr(), v.data_ptr(), pk.data_ptr() if P else None, pv.data_ptr() if P else None, out.data_ptr(),
                                        weights.data_ptr() if weights is not None else None, n, B, H, Hkv, T, Sk, P, d, _CODES[q.dtype], _strides(q), _strides(k),
                                        _strides(v), pks, pvs, _strides(out), ws, window, n_sink, float(scale), workspace.data_ptr(), workspace.numel(),
                                        _handle(stream, q.device))
    if st != 0:
        raise SmhaError(st, "smha_cache_forward")
    _written(out, weights)
    return out


def _prefix_strides(t):
    if t.is_contiguous():
        return None
    n, s = t.shape, t.stride()
    if s[2] != 1 and n[2] != 1:
        raise ValueError("the head's columns must be contiguous")
    return (C.c_int64 * 2)(s[0] if n[0] > 1 else 0, s[1] if n[1] > 1 else n[2])


def smha_cache_evict_workspace(B: int, Hkv: int, Sk: int, d: int, budget: int, recent: int) -> int:
    """Bytes of device memory that cache_evict needs."""
    need = C.c_size_t(0)
    st = _load().smha_cache_evict_workspace(B, Hkv, Sk, d, _check_int(budget, "budget"), _check_int(recent, "recent"), C.byref(need))
    if st != 0:
        raise SmhaError(st, "smha_cache_evict_workspace")
    return need.value


def cache_evict(k, v, weights, positions, lengths, budget: int, recent: int = 0, *, out=None, workspace=None, stream=None):
    """Brings every key head of every sequence down to `budget` keys; returns (weights, positions, lengths) as they are then.

    k, v [B,Hkv,Sk,d] as in cache_attention, changed in place; weights float32 and positions int32 [B,Hkv,Sk], lengths int32 [B], contiguous.  Where a
    sequence has more than `budget` keys, those of a head stay that are among the `recent` last positions (position > highest - recent), then
    those of the largest weight, the lower slot first among equals (recent keys count as of infinite weight, NaN as of the lowest).  Keys keep
    their slots, except that those that stay past the budget move, in order, to the slots before it that were freed: slots are then not in
    the order of positions, and the window of cache_attention, which counts slots, is not one of tokens any more.  Slots from the
    new length on get weight 0 and position -1, and keep their keys.
    out: the three tensors to write to, by default new ones; they may be the inputs themselves.  No gradients."""
    if out is None and workspace is None and stream is None:
        global _evict
        if _evict is None:
            _evict = native_call("cache_evict")
        got = _evict(k, v, weights, positions, lengths, budget, recent)
        if got is not None:
            if type(got) is int:
                raise SmhaError(got, "smha_cache_evict")
            return got
    if k.dim() != 4 or k.shape != v.shape or k.dtype not in _CODES or v.dtype != k.dtype:
        raise ValueError("k, v must be [B,Hkv,Sk,d], float16 or bfloat16, alike")
    if not k.is_cuda or v.device != k.device:
        raise ValueError("tensors must be on one GPU")
    B, Hkv, Sk, d = k.shape
    _check_no_gradients("cache_evict", k, v, weights, *(() if out is None else out))
    for t in (k, v):
        s = t.stride()
        if any(size > 1 and step < d for size, step in zip((B, Hkv, Sk), s)):
            raise ValueError("k and v are changed in place: their keys must not overlap")
    budget, recent = _check_int(budget, "budget"), _check_int(recent, "recent")
    given = (weights, positions, lengths)
    for t, name, dtype, shape in zip(given, ("weights", "positions", "lengths"), (torch.float32, torch.int32, torch.int32), ((B, Hkv, Sk), (B, Hkv, Sk), (B,))):
        if t.dtype != dtype or t.shape != shape or t.device != k.device or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {shape} on the same GPU")
    if out is not None:
        if len(out) != 3:
            raise ValueError("out must be three tensors like weights, positions and lengths")
        for t, like in zip(out, given):
            if t.dtype != like.dtype or t.shape != like.shape or t.device != k.device or not t.is_contiguous():
                raise ValueError("out must be three tensors like weights, positions and lengths")
    with _on_device(k), _allocating_on(stream, workspace is not None and out is not None):
        if out is None:
            out = tuple(torch.empty_like(t) for t in given)
        if workspace is None:
            workspace = torch.empty(smha_cache_evict_workspace(B, Hkv, Sk, d, budget, recent), dtype=torch.uint8, device=k.device)
        else:
            _check_workspace(workspace, k)
        st = _load().smha_cache_evict(k.data_ptr(), v.data_ptr(), *(t.data_ptr() for t in given), *(t.data_ptr() for t in out), B, Hkv, Sk, d, budget, recent,
                                      _strides(k), _strides(v), workspace.data_ptr(), workspace.numel(), _handle(stream, k.device))
    if st != 0:
        raise SmhaError(st, "smha_cache_evict")
    _written(k, v, *out)
    return tuple(out)
