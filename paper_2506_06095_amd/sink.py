"""Attention within a causal window and a few first keys that stay visible (sinks), with its gradients: binding of smha_sink_*.

Argument checks, allocation and autograd only; include/smha.h says what the entry points compute.
"""
from __future__ import annotations

import contextlib
import ctypes as C

import torch

from .binding import SMHA_BF16, SMHA_F16, SmhaError, _current_raw_stream, _load, native_call

_CODES = {torch.float16: SMHA_F16, torch.bfloat16: SMHA_BF16}
_PACKED = None


def _strides(t):
    """{batch, head, token} strides for the C ABI, None where the tensor is packed.  (What the stride of a dimension of size 1 says is
    never used, and need not fit.)"""
    if t.is_contiguous():
        return _PACKED
    n, s = t.shape, t.stride()
    if s[3] != 1 and n[3] != 1:
        raise ValueError("the head's columns must be contiguous")
    return (C.c_int64 * 3)(s[0] if n[0] > 1 else 0, s[1] if n[1] > 1 else 0, s[2] if n[2] > 1 else n[3])


def _on_device(t):
    """What runs a call on the tensor's device, which need not be the current one."""
    return contextlib.nullcontext() if t.device.index == torch.cuda.current_device() else torch.cuda.device(t.device)


def _handle(stream, device):
    if stream is None:
        return _current_raw_stream(torch, device)
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _check_qkv(q, k, v):
    if q.dim() != 4 or k.dim() != 4 or k.shape != v.shape or q.shape[0] != k.shape[0] or q.shape[3] != k.shape[3]:
        raise ValueError("q must be [B,H,Sq,d] and k, v [B,Hkv,Sk,d]")
    if k.shape[1] < 1 or q.shape[1] % k.shape[1]:
        raise ValueError("the number of heads must be a multiple of the number of key heads")
    if q.dtype not in _CODES or k.dtype != q.dtype or v.dtype != q.dtype:
        raise ValueError("q, k, v must be float16 or bfloat16, all alike")
    if not q.is_cuda or k.device != q.device or v.device != q.device:
        raise ValueError("tensors must be on one GPU")


def _check_no_tangents(name, *tensors):
    """Tangents of outputs would be missing."""
    if any(t is not None and torch.autograd.forward_ad.unpack_dual(t).tangent is not None for t in tensors):
        raise NotImplementedError(f"{name} has no derivatives in forward mode")


def _check_per_sequence(t, name, like):
    """The pointer of an int32 [B] tensor, None for None."""
    if t is None:
        return None
    if t.dtype != torch.int32 or t.shape != (like.shape[0],) or t.device != like.device or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous int32 [B] tensor on the same GPU")
    return t.data_ptr()


def _check_int(value, name):
    """An integer that the C ABI's int holds."""
    value = int(value)
    if not 0 <= value < 1 << 31:
        raise ValueError(f"{name} must be at least 0 and below 2^31")
    return value


def _written(*tensors):
    """Autograd refuses to go back through what was saved of a tensor that was written since."""
    for t in tensors:
        if t is not None and not t.is_inference():
            torch.autograd.graph.increment_version(t)


def _check_rest(rest, like):
    if rest is not None and (rest.shape != like.shape or rest.dtype != like.dtype or rest.device != like.device or not rest.is_contiguous()):
        raise ValueError("O_rest must be a contiguous tensor like O")
    return rest.data_ptr() if rest is not None else None


def smha_sink_forward(Q, K, V, O, lse=None, window: int = 0, n_sink: int = 0, offsets=None, lengths=None, scale: float = 0.0, stream=None,
                      O_rest=None) -> None:
    """O [B,H,Sq,d] and, where they are given, lse (float32 [B,H,Sq], contiguous) and O_rest (like O, contiguous: what O's rounding left out,
    for the backward pass) of Q [B,H,Sq,d], K, V [B,Hkv,Sk,d].  Enqueues on `stream`
    (default: torch's current stream of Q's device); does not synchronise."""
    _check_qkv(Q, K, V)
    B, H, Sq, d = Q.shape
    if O.shape != Q.shape or O.dtype != Q.dtype or O.device != Q.device:
        raise ValueError("O must be like Q")
    if lse is not None and (lse.shape != (B, H, Sq) or lse.dtype != torch.float32 or lse.device != Q.device or not lse.is_contiguous()):
        raise ValueError("lse must be a contiguous float32 [B,H,Sq] tensor on the same GPU")
    at, n = _check_per_sequence(offsets, "offsets", Q), _check_per_sequence(lengths, "lengths", Q)
    with _on_device(Q):
        st = _load().smha_sink_forward(Q.data_ptr(), K.data_ptr(), V.data_ptr(), O.data_ptr(), lse.data_ptr() if lse is not None else None,
                                       _check_rest(O_rest, Q), B, H, K.shape[1], Sq, K.shape[2], d, _CODES[Q.dtype], _strides(Q), _strides(K), _strides(V), _strides(O), at, n,
                                       _check_int(window, "window"), _check_int(n_sink, "n_sink"), float(scale), _handle(stream, Q.device))
    if st != 0:
        raise SmhaError(st, "smha_sink_forward")
    _written(O, lse, O_rest)


def smha_sink_workspace(B: int, H: int, Hkv: int, Sq: int, Sk: int, d: int, window: int = 0, n_sink: int = 0) -> int:
    """Bytes of device memory that smha_sink_backward needs."""
    need = C.c_size_t(0)
    st = _load().smha_sink_workspace(B, H, Hkv, Sq, Sk, d, _check_int(window, "window"), _check_int(n_sink, "n_sink"), C.byref(need))
    if st != 0:
        raise SmhaError(st, "smha_sink_workspace")
    return need.value


def smha_sink_backward(Q, K, V, O, lse, dO, dQ, dK, dV, window: int = 0, n_sink: int = 0, offsets=None, lengths=None, scale: float = 0.0, workspace=None,
                       stream=None, O_rest=None) -> None:
    """dQ, dK, dV (like Q, K, V) from what smha_sink_forward took and gave and the gradient dO of O.  workspace: a uint8 tensor of
    smha_sink_workspace bytes; by default one is allocated.  (In binary16, dS is rounded to it like the gradients themselves: gradients of O have to be
    scaled so that they and their products with V keep within its range.)"""
    _check_qkv(Q, K, V)
    B, H, Sq, d = Q.shape
    for t, like, name in ((O, Q, "O"), (dO, Q, "dO"), (dQ, Q, "dQ"), (dK, K, "dK"), (dV, V, "dV")):
        if t.shape != like.shape or t.dtype != Q.dtype or t.device != Q.device:
            raise ValueError(f"{name} has another shape, type or device than what it belongs to")
    if lse.shape != (B, H, Sq) or lse.dtype != torch.float32 or lse.device != Q.device or not lse.is_contiguous():
        raise ValueError("lse must be a contiguous float32 [B,H,Sq] tensor on the same GPU")
    at, n = _check_per_sequence(offsets, "offsets", Q), _check_per_sequence(lengths, "lengths", Q)
    window, n_sink = _check_int(window, "window"), _check_int(n_sink, "n_sink")
    with _on_device(Q):
        if workspace is None:
            if stream is not None and not isinstance(stream, torch.cuda.Stream):
                raise ValueError("a call on a bare stream handle needs a workspace")
            with torch.cuda.stream(stream) if stream is not None else contextlib.nullcontext():
                workspace = torch.empty(smha_sink_workspace(B, H, K.shape[1], Sq, K.shape[2], d, window, n_sink), dtype=torch.uint8, device=Q.device)
        elif workspace.dtype != torch.uint8 or workspace.device != Q.device or not workspace.is_contiguous():
            raise ValueError("workspace must be a contiguous uint8 tensor on the same GPU")
        st = _load().smha_sink_backward(*(t.data_ptr() for t in (Q, K, V, O)), _check_rest(O_rest, Q), *(t.data_ptr() for t in (lse, dO, dQ, dK, dV)), B, H, K.shape[1], Sq, K.shape[2], d, _CODES[Q.dtype],
                                        *(_strides(t) for t in (Q, K, V, O, dO, dQ, dK, dV)), at, n, window, n_sink, float(scale),
                                        workspace.data_ptr(), workspace.numel(), _handle(stream, Q.device))
    if st != 0:
        raise SmhaError(st, "smha_sink_backward")
    _written(dQ, dK, dV)


def _takes(t):
    """Whether the kernels can read a tensor as it lies (autograd may hand on gradients that are expanded or transposed or of more than 2 GiB between a
    head's first and last row, and hooks of saved tensors may give those back with other strides)."""
    if t.data_ptr() % 16:
        return False
    if t.is_contiguous():
        return True
    (b, h, rows, d), s = t.shape, t.stride()
    pitch = s[2] if rows > 1 else d
    return s[3] == 1 and all(n == 1 or step % 8 == 0 for n, step in zip((b, h, rows), s)) and pitch >= d and ((rows + 128) * pitch + d) * 2 < 1 << 31


def _readable(t):
    return t if _takes(t) else t.clone(memory_format=torch.contiguous_format)


class _SinkAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, window, n_sink, offsets, lengths, scale):
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        lse = torch.empty(q.shape[:3], dtype=torch.float32, device=q.device)
        rest = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        smha_sink_forward(q, k, v, out, lse, window, n_sink, offsets, lengths, scale, O_rest=rest)
        ctx.save_for_backward(q, k, v, out, rest, lse, offsets, lengths)
        ctx.rest = window, n_sink, scale
        return out

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad):
        saved = ctx.saved_tensors
        q, k, v, out = (_readable(t) for t in saved[:4])
        rest, lse, offsets, lengths = (t if t is None else t.contiguous() for t in saved[4:])
        window, n_sink, scale = ctx.rest
        dq, dk, dv = (torch.empty(t.shape, dtype=t.dtype, device=t.device) for t in (q, k, v))
        smha_sink_backward(q, k, v, out, lse, _readable(grad), dq, dk, dv, window, n_sink, offsets, lengths, scale,
                           O_rest=rest)
        return dq, dk, dv, None, None, None, None, None


_call = None  # the native way, for every call that it takes


def sink_attention(q, k, v, window: int = 0, n_sink: int = 0, *, offsets=None, lengths=None, scale: float = 0.0):
    """softmax(scale q k^T over visible keys) v, differentiable in q, k and v (once, and not in forward mode).

    q [B,H,Sq,d]; k, v [B,Hkv,Sk,d], H a multiple of Hkv; float16 or bfloat16, d a multiple of 8 up to 128.  Query i of sequence b stands at
    offsets[b] + i (default Sk - Sq + i) and exists where that is in 0 .. lengths[b] - 1 (default Sk); it sees key j iff j is not after it and
    either within the last `window` keys (0: any) or one of the first `n_sink`.  offsets, lengths: int32 [B] on the GPU, read there.  scale: 0
    or less for 1/sqrt(d).  Queries that do not exist give zeros, and neither they nor keys past a length receive or pass on gradients.
    (A pass is captured into a graph where no eager graph of the same leaves is alive, as torch wants it.)"""
    global _call
    if _call is None:
        _call = native_call("sink_attention")
    got = _call(q, k, v, window, n_sink, offsets, lengths, float(scale))
    if got is not None:
        if type(got) is int:
            raise SmhaError(got, "smha_sink_forward")
        return got
    _check_qkv(q, k, v)
    _check_no_tangents("sink_attention", q, k, v)
    if torch.is_grad_enabled() and (q.requires_grad or k.requires_grad or v.requires_grad):
        return _SinkAttention.apply(q, k, v, window, n_sink, offsets, lengths, scale)
    out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    smha_sink_forward(q, k, v, out, None, window, n_sink, offsets, lengths, scale)
    return out
