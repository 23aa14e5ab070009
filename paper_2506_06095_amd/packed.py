"""A cache held in 4 bits: packed as it is written, read back, and attended to: binding of smha_packed_*.

Argument checks and allocation only; include/smha.h says how rows are packed and what the entry points compute.
"""
from __future__ import annotations

import ctypes as C

import torch

from .binding import SMHA_F32, SmhaError, _load, native_call
from .cache import _allocating_on, _check_no_gradients, _check_workspace
from .sink import _CODES, _check_int, _check_per_sequence, _handle, _on_device, _strides, _written

_READ_CODES = {**_CODES, torch.float32: SMHA_F32}
_write = _read = _attention = None  # functions of _smha_torch


def smha_packed_row(d: int) -> int:
    """Bytes of a packed row of d columns."""
    n = C.c_int(0)
    st = _load().smha_packed_row(_check_int(d, "d"), C.byref(n))
    if st != 0:
        raise SmhaError(st, "smha_packed_row")
    return n.value


_WIDTHS = {4 * ((d + 31) // 32) + d // 2: d for d in range(8, 129, 8)}  # bytes of a row: columns (no two are the same)


def _width(k, v):
    """Columns of the rows of a packed cache."""
    if k.dim() != 4 or k.shape != v.shape or k.dtype != torch.uint8 or v.dtype != torch.uint8 or k.shape[3] not in _WIDTHS:
        raise ValueError("the cache must be two uint8 tensors [B,Hkv,Sk,row], alike, row = smha_packed_row(d)")
    if not k.is_cuda or v.device != k.device:
        raise ValueError("tensors must be on one GPU")
    return _WIDTHS[k.shape[3]]


def _check_rows_apart(*tensors):
    for t in tensors:
        if any(size > 1 and step < t.shape[3] for size, step in zip(t.shape[:3], t.stride())):
            raise ValueError("what is written must not overlap")


_MOST_ROWS, _UNSUPPORTED = 1 << 27, 2  # SMHA_PACKED_MOST_ROWS, SMHA_ERR_UNSUPPORTED


def _check_outputs_fit(where, B, Hkv, T, d, dtype):
    """What the entry points would refuse for its size is not allocated first."""
    if B * Hkv * T > _MOST_ROWS or (T + 64) * d * dtype.itemsize >= 1 << 31:
        raise SmhaError(_UNSUPPORTED, where)


def packed_cache(B: int, Hkv: int, Sk: int, d: int, *, device=None):
    """An empty cache for packed_write: two uint8 tensors [B,Hkv,Sk,smha_packed_row(d)] of zeros on the GPU (`device`: the current one).  (Any such
    tensors will do, whose rows are contiguous and whose strides are multiples of 4.)"""
    device = torch.device("cuda") if device is None else torch.device(device)
    if device.type != "cuda":
        raise ValueError("the cache must be on a GPU")
    shape = [_check_int(n, name) for n, name in ((B, "B"), (Hkv, "Hkv"), (Sk, "Sk"))] + [smha_packed_row(d)]
    return torch.zeros(shape, dtype=torch.uint8, device=device), torch.zeros(shape, dtype=torch.uint8, device=device)


def packed_write(k_new, v_new, k, v, lengths, *, offsets=None, values: bool = False, stream=None):
    """Packs new tokens' keys and values, [B,Hkv,T,d] of float16 or bfloat16, into their slots of the cache k, v (uint8 [B,Hkv,Sk,row], see
    packed_cache), which is changed in place.

    lengths: int32 [B] on the GPU, keys of every sequence, the new tokens' included.  Token t of sequence b goes to slot lengths[b] - T + t, or to
    offsets[b] + t (int32 [B] on the GPU: prompts that are padded behind have offsets of 0); where that is not in 0 .. lengths[b] - 1 the
    token is left out.  k and v may lie side by side in one tensor, but share no memory.  values: return (keys, values) like k_new and v_new as the cache stands for them from now on (tokens that are left out: zeros), for attention of
    the prompt itself on what later tokens will see; otherwise None.  Values beyond +-65280 are packed as +-65280, 32 columns among which there
    is a NaN as NaN.  No gradients."""
    if stream is None:  # the native way, for every call that it takes (csrc/torch_binding.cpp)
        global _write
        if _write is None:
            _write = native_call("packed_write")
        got = _write(k_new, v_new, k, v, lengths, offsets, values)
        if got is not None:
            if type(got) is int:
                raise SmhaError(got, "smha_packed_write")
            return None if got is True else got
    d = _width(k, v)
    if k_new.dim() != 4 or k_new.shape != v_new.shape or k_new.shape[:2] != k.shape[:2] or k_new.shape[3] != d:
        raise ValueError("k_new, v_new must be [B,Hkv,T,d], and the cache [B,Hkv,Sk,smha_packed_row(d)]")
    if k_new.dtype not in _CODES or v_new.dtype != k_new.dtype:
        raise ValueError("k_new, v_new must be float16 or bfloat16, alike")
    if k_new.device != k.device or v_new.device != k.device:
        raise ValueError("tensors must be on one GPU")
    _check_no_gradients("packed_write", k_new, v_new)
    _check_rows_apart(k, v)
    if lengths is None:
        raise ValueError("lengths must be given")
    n, at = _check_per_sequence(lengths, "lengths", k), _check_per_sequence(offsets, "offsets", k)
    (B, Hkv, T, _), Sk = k_new.shape, k.shape[2]
    if values:
        _check_outputs_fit("smha_packed_write", B, Hkv, T, d, k_new.dtype)
    with _on_device(k), _allocating_on(stream, not values):
        out = tuple(torch.empty(t.shape, dtype=t.dtype, device=t.device) for t in (k_new, v_new)) if values else None
        st = _load().smha_packed_write(k_new.data_ptr(), v_new.data_ptr(), k.data_ptr(), v.data_ptr(), *((t.data_ptr() for t in out) if values else (None, None)), n, at, B, Hkv,
                                       T, Sk, d, _CODES[k_new.dtype], *(_strides(t) for t in (k_new, v_new, k, v)), _handle(stream, k.device))
    if st != 0:
        raise SmhaError(st, "smha_packed_write")
    _written(k, v)
    return out


def packed_read(k, v, lengths, *, offsets=None, tokens=None, dtype=torch.float16, out=None, stream=None):
    """What `tokens` slots of every sequence (default: all) from slot offsets[b] (default: 0) on stand for: (keys, values), each [B,Hkv,tokens,d] of
    `dtype`, float16, float32 (the same values) or bfloat16 (rounded to it); zeros where a slot is not in 0 .. lengths[b] - 1.  k, v, lengths, offsets as in packed_write.
    out: the two tensors to write to, which share no memory, by default new ones."""
    if out is None and stream is None:
        global _read
        if _read is None:
            _read = native_call("packed_read")
        got = _read(k, v, lengths, offsets, tokens, dtype)
        if got is not None:
            if type(got) is int:
                raise SmhaError(got, "smha_packed_read")
            return got
    d = _width(k, v)
    if lengths is None:
        raise ValueError("lengths must be given")
    n, at = _check_per_sequence(lengths, "lengths", k), _check_per_sequence(offsets, "offsets", k)
    B, Hkv, Sk, _ = k.shape
    T = Sk if tokens is None else _check_int(tokens, "tokens")
    if dtype not in _READ_CODES:
        raise ValueError("dtype must be float16, bfloat16 or float32")
    if out is not None:
        if len(out) != 2 or any(t.shape != (B, Hkv, T, d) or t.dtype != dtype or t.device != k.device for t in out):
            raise ValueError("out must be two [B,Hkv,tokens,d] tensors of dtype on the same GPU")
        _check_no_gradients("packed_read", *out)
        _check_rows_apart(*out)
    if out is None:
        _check_outputs_fit("smha_packed_read", B, Hkv, T, d, dtype)
    with _on_device(k), _allocating_on(stream, out is not None):
        if out is None:
            out = tuple(torch.empty(B, Hkv, T, d, dtype=dtype, device=k.device) for _ in range(2))
        st = _load().smha_packed_read(k.data_ptr(), v.data_ptr(), out[0].data_ptr(), out[1].data_ptr(), n, at, B, Hkv, T, Sk, d, _READ_CODES[dtype],
                                      *(_strides(t) for t in (k, v, *out)), _handle(stream, k.device))
    if st != 0:
        raise SmhaError(st, "smha_packed_read")
    _written(*out)
    return tuple(out)


def smha_packed_workspace(B: int, H: int, Hkv: int, T: int, Sk: int, d: int, window: int = 0, n_sink: int = 0) -> int:
    """Bytes of device memory that packed_attention needs."""
    need = C.c_size_t(0)
    st = _load().smha_packed_workspace(B, H, Hkv, T, Sk, d, _check_int(window, "window"), _check_int(n_sink, "n_sink"), C.byref(need))
    if st != 0:
        raise SmhaError(st, "smha_packed_workspace")
    return need.value


def packed_attention(q, k, v, lengths, *, window: int = 0, n_sink: int = 0, out=None, scale: float = 0.0, workspace=None, stream=None):
    """cache_attention on a packed cache: attention of the last T tokens of every sequence, whose keys and values are in the cache already: [B,H,T,d] like q.

    q [B,H,T,d], float16 or bfloat16 (whatever the type was that the cache was packed from); k, v uint8 [B,Hkv,Sk,row] as in packed_write, H a multiple
    of Hkv; T from one token to a chunk of a prompt.  lengths, window, n_sink, scale, out, workspace (of smha_packed_workspace bytes) as in cache_attention: token t of sequence b
    stands at slot lengths[b] - T + t and sees the keys up to itself, the last `window` of them (0: all) and the first `n_sink`.  No gradients.  Keys that a token of
    the sequence sees have to stand for something finite, as what packed_write packed of finite values does (others, and free slots, may hold anything)."""
    if out is None and workspace is None and stream is None:
        global _attention
        if _attention is None:
            _attention = native_call("packed_attention")
        got = _attention(q, k, v, lengths, window, n_sink, float(scale))
        if got is not None:
            if type(got) is int:
                raise SmhaError(got, "smha_packed_forward")
            return got
    d = _width(k, v)
    if q.dim() != 4 or q.shape[0] != k.shape[0] or q.shape[3] != d:
        raise ValueError("q must be [B,H,T,d], and the cache [B,Hkv,Sk,smha_packed_row(d)]")
    if k.shape[1] < 1 or q.shape[1] % k.shape[1]:
        raise ValueError("the number of heads must be a multiple of the number of key heads")
    if q.dtype not in _CODES:
        raise ValueError("q must be float16 or bfloat16")
    if q.device != k.device:
        raise ValueError("tensors must be on one GPU")
    _check_no_gradients("packed_attention", q, out)
    (B, H, T, _), (Hkv, Sk) = q.shape, k.shape[1:3]
    if lengths is None:
        raise ValueError("lengths must be given")
    n = _check_per_sequence(lengths, "lengths", q)
    window, n_sink = _check_int(window, "window"), _check_int(n_sink, "n_sink")
    if out is not None and (out.shape != q.shape or out.dtype != q.dtype or out.device != q.device):
        raise ValueError("out must be like q")
    with _on_device(q), _allocating_on(stream, workspace is not None and out is not None):
        need = smha_packed_workspace(B, H, Hkv, T, Sk, d, window, n_sink)  # (sizes that are not taken end here)
        if workspace is None:
            workspace = torch.empty(need, dtype=torch.uint8, device=q.device)
        else:
            _check_workspace(workspace, q)
        if out is None:
            out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        st = _load().smha_packed_forward(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), n, B, H, Hkv, T, Sk, d, _CODES[q.dtype],
                                         *(_strides(t) for t in (q, k, v, out)), window, n_sink, float(scale), workspace.data_ptr(), workspace.numel(),
                                         _handle(stream, q.device))
    if st != 0:
        raise SmhaError(st, "smha_packed_forward")
    _written(out)
    return out
