"""smha: masked multi-head attention for MI355X (gfx950) behind a C ABI.

Beside plans: attention with a window and sinks (`sink`), on a cache, and eviction from it (`cache`), and a cache held in 4 bits (`packed`).

The compute lives in libsmha.so (HIP); this package is the thin ctypes binding
(`binding`, `sink`, `cache`, `packed`) and the in-tree build step (`build`).  There is no CPU fallback: if
the library is missing or no GPU is usable, calls raise.
"""
from .binding import (  # noqa: F401
    SMHA_BF16, SMHA_F16, SMHA_F32, SMHA_KERNEL_AUTO, SMHA_KERNEL_BLOCK, SMHA_KERNEL_ROW,
    SMHA_SELECTOR_CALIBRATED, SMHA_SELECTOR_PAPER_EQ1, Plan, SmhaError, library_path,
    smha_call_kernel_name, smha_forward, smha_forward_static, smha_kernel_name, smha_plan_destroy, smha_plan_export, smha_plan_from_dense,
    smha_plan_from_dense_rect,
    smha_plan_from_desc, smha_plan_info, smha_plan_prepare, smha_plan_work_order, smha_status_string)

_OPERATORS = {**{name: "sink" for name in ("sink_attention", "smha_sink_backward", "smha_sink_forward", "smha_sink_workspace")},
              **{name: "cache" for name in ("cache_attention", "cache_evict", "smha_cache_evict_workspace", "smha_cache_workspace")},
              **{name: "packed" for name in ("packed_attention", "packed_cache", "packed_read", "packed_write", "smha_packed_row", "smha_packed_workspace")}}


def __getattr__(name):  # (these modules need torch when they are imported, which plans on the host do not)
    if name in _OPERATORS:
        import importlib
        value = globals()[name] = getattr(importlib.import_module(f".{_OPERATORS[name]}", __name__), name)  # (from now on an ordinary name: this costs 8 us)
        return value
    raise AttributeError(f"module {__name__!r} has no attribute {name!r}")
