"""Spectral-LSH hot path on AMD MI355X (gfx950): HIP kernels behind the C ABI
of include/slh.h (libslh.so), with a thin ctypes binding (slh.py)."""
from .slh import (  # noqa: F401
    SLHError, load, slh_gen_params, slh_gen_start, slh_create, slh_set_option, slh_set_stream,
    slh_route, slh_feature_map, slh_lanczos, slh_simhash, slh_merge, slh_merge_async, slh_merge_wait, slh_merge_capacity,
    slh_copy_out, slh_load, slh_stage_times, slh_time_passes, slh_spectral_energy, slh_bucket_purity, slh_eigh_ritz, slh_peak_read, slh_peak_mfma, slh_merge_noalloc, compress,
)

# The attention operators' bindings are loaded when one of them is first asked for: they need torch, the host calls above
# do not.
_ATTENTION = (
    "slh_rope_table", "slh_qk_norm_rope", "slh_kv_append", "slh_attend_workspace", "slh_attend",
    "slh_attend_paged_workspace", "slh_attend_paged",
)
_CACHE = (
    "slh_kv_append_e4m3", "slh_attend_paged_e4m3_workspace", "slh_attend_paged_e4m3", "slh_attend_weights_workspace",
    "slh_attend_weights", "slh_kv_evict_workspace", "slh_kv_evict",
)
_LATER = {"attention": _ATTENTION, "cache": _CACHE}
__all__ = [n for n in globals() if not n.startswith("_")] + [*_LATER, *_ATTENTION, *_CACHE]


def __getattr__(name):
    of = next((m for m, names in _LATER.items() if name == m or name in names), None)
    if of is None:
        raise AttributeError(f"module {__name__!r} has no attribute {name!r}")
    from importlib import import_module
    module = import_module("." + of, __name__)
    globals().update({n: getattr(module, n) for n in _LATER[of]})
    return globals()[name]


def __dir__():
    return sorted({*globals(), *__all__})
