"""Spectral-LSH hot path on AMD MI355X (gfx950): HIP kernels behind the C ABI
of include/slh.h (libslh.so), with a thin ctypes binding (slh.py)."""
from .slh import (  # noqa: F401
    SLHError, load, slh_gen_params, slh_gen_start, slh_create, slh_set_option, slh_set_stream,
    slh_route, slh_feature_map, slh_lanczos, slh_simhash, slh_merge, slh_merge_async, slh_merge_wait, slh_merge_capacity,
    slh_copy_out, slh_load, slh_stage_times, slh_time_passes, slh_spectral_energy, slh_bucket_purity, slh_eigh_ritz, slh_peak_read, slh_peak_mfma, slh_merge_noalloc, compress,
)

# The attention operators' binding is loaded when one of them is first asked for: it needs torch, the host calls above
# do not.
_ATTENTION = (
    "slh_rope_table", "slh_qk_norm_rope", "slh_kv_append", "slh_attend_workspace", "slh_attend",
    "slh_attend_paged_workspace", "slh_attend_paged",
)
__all__ = [n for n in globals() if not n.startswith("_")] + ["attention", *_ATTENTION]


def __getattr__(name):
    if name != "attention" and name not in _ATTENTION:
        raise AttributeError(f"module {__name__!r} has no attribute {name!r}")
    from importlib import import_module
    module = import_module(".attention", __name__)
    globals().update({n: getattr(module, n) for n in _ATTENTION})
    return globals()[name]


def __dir__():
    return sorted({*globals(), *__all__})
