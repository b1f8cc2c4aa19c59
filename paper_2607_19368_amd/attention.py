"""Python binding of the operators behind a compressed prompt (include/slh.h): argument
checks and marshalling, as in slh.py.  Every call goes to torch's current stream, or to the
`stream` given (a torch.cuda.Stream), and returns without waiting for it.  The operators have no backward passes:
tensors that require a gradient are refused where torch records one.
"""
import math

import torch

from . import slh as B
from .slh import SLHError

_DTYPES = {torch.bfloat16: B.SLH_BF16, torch.float16: B.SLH_F16, torch.float32: B.SLH_F32}
_HALVES = (torch.bfloat16, torch.float16)


# The calls of a decode step take microseconds, so the checks here are few and flat: dtypes are
# singletons, devices are compared by index, and the stream is asked for as an integer.
_current_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda index: torch.cuda.current_stream(index).cuda_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
_recording = torch.is_grad_enabled


def _no_gradient(name):
    raise SLHError(f"{name} requires a gradient, and the operator has no backward pass: detach it or call under torch.no_grad()")


def _call(name, dev, stream, args):
    """Calls the library's function `name` on device `dev` with args and the stream."""
    f = getattr(B.load(), name)
    if _current_device() == dev:
        rc = f(*args, _current_stream(dev) if stream is None else stream.cuda_stream)
    else:
        with torch.cuda.device(dev):
            rc = f(*args, _current_stream(dev) if stream is None else stream.cuda_stream)
    if rc != B.SLH_OK:
        raise SLHError(f"{name} failed ({rc}): " + {
            B.SLH_EINVAL: "a size, stride or alignment that the library does not take",
            B.SLH_EHIP: "a kernel launch failed"}.get(rc, ""))


def _strides(st, shape):
    """Strides without those of single tokens and heads: they reach nothing, and torch leaves any value in them."""
    return [0 if n == 1 else s for n, s in zip(shape, st)]


def _first(name, t, dims):
    """(type, device index, shape, strides) of the tensor of rows that the others go by."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise SLHError(f"{name} must be a device tensor")
    if t.dtype not in _DTYPES:
        raise SLHError(f"{name}: unsupported type {t.dtype}")
    if t.requires_grad and _recording():
        _no_gradient(name)
    shape, st = t.shape, t.stride()
    if 1 in shape and (shape[0] == 1 or shape[-2] == 1):
        st = _strides(st, shape)
    if len(shape) not in dims or (st[-1] != 1 and t.numel() > 0):
        raise SLHError(f"{name} must have {' or '.join(map(str, dims))} dimensions and unit stride in the last")
    return t.dtype, t.get_device(), shape, st


def _rows(name, t, dtype, dev, shape):
    """Strides of t, a tensor of rows with unit element stride."""
    try:
        if t.dtype is not dtype or t.get_device() != dev:
            raise SLHError(f"{name} must be a {dtype} tensor on device {dev}")
    except AttributeError:
        raise SLHError(f"{name} must be a tensor") from None
    if t.shape != shape:
        raise SLHError(f"{name} must have shape {tuple(shape)}")
    if t.requires_grad and _recording():
        _no_gradient(name)
    st = t.stride()
    if 1 in shape and (shape[0] == 1 or shape[-2] == 1):
        st = _strides(st, shape)
    if st[-1] != 1 and t.numel() > 0:
        raise SLHError(f"{name} must have unit stride in the last dimension")
    return st


def _plain(name, t, dtype, dev, shape):
    """Address of t, a contiguous tensor of `shape`, or of so many dimensions."""
    try:
        if t.dtype is not dtype or t.get_device() != dev or not t.is_contiguous():
            raise SLHError(f"{name} must be a contiguous {dtype} tensor on device {dev}")
    except AttributeError:
        raise SLHError(f"{name} must be a tensor") from None
    if t.shape != shape if shape.__class__ is not int else t.dim() != shape:
        raise SLHError(f"{name} must have " + (f"{shape} dimensions" if isinstance(shape, int) else f"shape {tuple(shape)}"))
    if t.requires_grad and _recording():
        _no_gradient(name)
    return t.data_ptr()


def _empty(shape, dtype, dev, stream):
    """Memory of the stream that the call goes to."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=dev)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=dev)


def _rotation(table, pos, T, dev):
    """(table address, n_pos, rot_dim, pos address) of a rotation, or of none."""
    if table is None:
        return None, 0, 0, None
    t = _plain("table", table, torch.float32, dev, 3)
    n_pos, two, half = table.shape
    if two != 2 or pos is None:
        raise SLHError("table must have shape (*, 2, rot_dim / 2), and pos must be given with it")
    return t, n_pos, 2 * half, _plain("pos", pos, torch.int32, dev, (T,))


def slh_rope_table(n_pos, rot_dim, base=10000.0, scaling=B.SLH_ROPE_PLAIN, factor=1.0, orig_len=0,
                   beta_fast=32.0, beta_slow=1.0, device="cuda", stream=None):
    """Table [n_pos, 2, rot_dim / 2] float32 of cosines and sines for slh_qk_norm_rope and
    slh_kv_append; `scaling` is one of SLH_ROPE_PLAIN, _LINEAR, _BASE and _BANDS (include/slh.h)."""
    if n_pos < 1 or rot_dim < 16 or rot_dim > 256 or rot_dim % 16:
        raise SLHError("n_pos must be positive and rot_dim a multiple of 16 from 16 to 256")
    table = _empty((n_pos, 2, rot_dim // 2), torch.float32, device, stream)
    _call("slh_rope_table", table.get_device(), stream,
          (table.data_ptr(), n_pos, rot_dim, float(base), int(scaling), float(factor), int(orig_len),
           float(beta_fast), float(beta_slow)))
    return table


def slh_qk_norm_rope(q, k=None, q_weight=None, k_weight=None, eps=1e-6, table=None, pos=None, interleaved=False,
                     q_out=None, k_out=None, stream=None):
    """Queries [T, Hq, d] and keys [T, Hk, d] (either may be None): RMS norm per head where a
    weight [d] is given, rotation by the table's rows `pos` [T] int32 where a table is.  Returns
    (q_out, k_out), which may be the inputs themselves."""
    dtype, dev, shape, st = _first("q" if q is not None else "k", q if q is not None else k, (3,))
    T, _, d = shape
    none = (None, 0, 0, 0, None, 0, 0)
    qa = ka = none
    if q is not None:
        if q_out is None:
            q_out = _empty(shape, dtype, q.device, stream)
        so = _rows("q_out", q_out, dtype, dev, shape)
        qa = (q.data_ptr(), st[0], st[1], shape[1], q_out.data_ptr(), so[0], so[1])
    if k is not None:
        shape = k.shape
        if len(shape) != 3 or shape[0] != T or shape[2] != d:
            raise SLHError("q and k must have the same tokens and head size")
        st = _rows("k", k, dtype, dev, shape)
        if k_out is None:
            k_out = _empty(shape, dtype, k.device, stream)
        so = _rows("k_out", k_out, dtype, dev, shape)
        ka = (k.data_ptr(), st[0], st[1], shape[1], k_out.data_ptr(), so[0], so[1])
    tab, n_pos, rot, p = _rotation(table, pos, T, dev)
    wq = None if q_weight is None else _plain("q_weight", q_weight, dtype, dev, (d,))
    wk = None if k_weight is None else _plain("k_weight", k_weight, dtype, dev, (d,))
    _call("slh_qk_norm_rope", dev, stream,
          (*qa, *ka, _DTYPES[dtype], T, d, wq, wk, eps, tab, n_pos, rot, p, interleaved))
    return (q_out if q is not None else None), (k_out if k is not None else None)


def slh_kv_append(k, v, k_cache, v_cache, slots, k_weight=None, eps=1e-6, table=None, pos=None, interleaved=False,
                  stream=None):
    """Writes k and v [T, H, d] into the caches [pages, H, page, d] at rows `slots` [T] int64
    (page * page size + row; negative: left out), the keys normed and rotated on the way as
    in slh_qk_norm_rope.  Returns the caches."""
    dtype, dev, shape, ks = _first("k", k, (3,))
    vs = _rows("v", v, dtype, dev, shape)
    T, H, d = shape
    kc = _plain("k_cache", k_cache, dtype, dev, 4)
    cache = k_cache.shape
    if cache[1] != H or cache[3] != d:
        raise SLHError(f"k_cache must have shape (*, {H}, *, {d})")
    vc = _plain("v_cache", v_cache, dtype, dev, cache)
    sl = _plain("slots", slots, torch.int64, dev, (T,))
    tab, n_pos, rot, p = _rotation(table, pos, T, dev)
    wk = None if k_weight is None else _plain("k_weight", k_weight, dtype, dev, (d,))
    _call("slh_kv_append", dev, stream,
          (k.data_ptr(), ks[0], ks[1], v.data_ptr(), vs[0], vs[1], _DTYPES[dtype], T, H, d, wk, eps, tab, n_pos, rot,
           p, interleaved, kc, vc, cache[0], cache[2], sl))
    return k_cache, v_cache


def _workspace(need, dev, workspace, device, stream):
    """(tensor, address) of `need` bytes: of the workspace given, or of a new one."""
    if need <= 0:
        return None, None
    if workspace is None:
        workspace = _empty(need, torch.uint8, device, stream)
        return workspace, workspace.data_ptr()
    at = _plain("workspace", workspace, torch.uint8, dev, 1)
    if workspace.numel() < need:
        raise SLHError(f"workspace must hold {need} bytes")
    return workspace, at


def _bytes(name, dev, args):
    """What a workspace function says for device `dev`."""
    f = getattr(B.load(), name)
    if _current_device() == dev:
        return f(*args)
    with torch.cuda.device(dev):
        return f(*args)


def slh_attend_workspace(Tq, Tk, B_, Hq, Hkv, d, causal=True):
    """Bytes that slh_attend needs as workspace on the current device."""
    return int(B.load().slh_attend_workspace(Tq, Tk, B_, Hq, Hkv, d, causal))


def slh_attend(q, k, v, cu_q, cu_k=None, scale=None, causal=True, out=None, lse_out=None, workspace=None,
               stream=None):
    """Attention of packed sequences: q [Tq, Hq, d], k and v [Tk, Hkv, d] (bf16 or fp16), sequence b
    at rows cu_q[b]..cu_q[b + 1] of q and cu_k[b]..cu_k[b + 1] of k and v (int32; cu_k None: as cu_q).
    causal: a sequence's last query sees all its keys, the one before it one fewer, and so on.
    scale: 1 / sqrt(d) by default.  lse_out: [Tq, Hq] float32.  Returns out; its rows of no sequence (in front of cu_q[0],
    behind the last entry) are not written, so hold anything in a new one."""
    dtype, dev, shape, qs = _first("q", q, (3,))
    if dtype not in _HALVES:
        raise SLHError("q must be bfloat16 or float16")
    Tq, Hq, d = shape
    if not isinstance(k, torch.Tensor) or k.dim() != 3 or k.shape[2] != d:
        raise SLHError("k must have three dimensions and q's head size")
    kshape = k.shape
    ks = _rows("k", k, dtype, dev, kshape)
    vs = _rows("v", v, dtype, dev, kshape)
    Tk, Hkv, _ = kshape
    cq = _plain("cu_q", cu_q, torch.int32, dev, 1)
    n = cu_q.shape[0] - 1
    ck = cq if cu_k is None else _plain("cu_k", cu_k, torch.int32, dev, (n + 1,))
    if n < 0:
        raise SLHError("cu_q must have an entry more than there are sequences")
    if out is None:
        out = _empty(shape, dtype, q.device, stream)
    os = _rows("out", out, dtype, dev, shape)
    lse = None if lse_out is None else _plain("lse_out", lse_out, torch.float32, dev, (Tq, Hq))
    need = _bytes("slh_attend_workspace", dev, (Tq, Tk, n, Hq, Hkv, d, causal))
    workspace, ws = _workspace(need, dev, workspace, q.device, stream)
    _call("slh_attend", dev, stream,
          (q.data_ptr(), qs[0], qs[1], k.data_ptr(), ks[0], ks[1], v.data_ptr(), vs[0], vs[1], _DTYPES[dtype], Tq, Tk,
           n, Hq, Hkv, d, cq, ck, 1.0 / math.sqrt(d) if scale is None else scale, causal, out.data_ptr(), os[0],
           os[1], lse, ws, need))
    return out


def slh_attend_paged_workspace(B_, n_q, Hq, Hkv, d, max_len, prefix_len):
    """Bytes that slh_attend_paged needs as workspace on the current device."""
    return int(B.load().slh_attend_paged_workspace(B_, n_q, Hq, Hkv, d, max_len, prefix_len))


def slh_attend_paged(q, k_cache, v_cache, page_table, lens, prefix_pages=None, prefix_len=0, scale=None, out=None,
                     lse_out=None, workspace=None, stream=None):
    """The new tokens q [B, n_q, Hq, d] (or [B, Hq, d]: one each) of a batch against the paged caches
    [pages, Hkv, page, d]: sequence b's keys are the first prefix_len rows of prefix_pages (int32,
    shared by all), then the first lens[b] rows of its own pages page_table[b] (int32 [B, n]), the new
    tokens' rows the last of them.  lse_out: q's shape without d, float32.  Returns out."""
    dtype, dev, shape, qs = _first("q", q, (3, 4))
    if dtype not in _HALVES:
        raise SLHError("q must be bfloat16 or float16")
    n, Hq, d = shape[0], shape[-2], shape[-1]
    n_q = shape[1] if len(shape) == 4 else 1
    if out is None:
        out = _empty(shape, dtype, q.device, stream)
    os = _rows("out", out, dtype, dev, shape)
    if n_q > 1 and n > 1 and (qs[0] != n_q * qs[1] or os[0] != n_q * os[1]):
        raise SLHError("q and out: sequences must follow one another as their tokens do")
    at = 1 if n_q > 1 else 0                # the dimension whose stride is a token's
    kc = _plain("k_cache", k_cache, dtype, dev, 4)
    cache = k_cache.shape
    if cache[3] != d:
        raise SLHError("k_cache must have q's head size")
    vc = _plain("v_cache", v_cache, dtype, dev, cache)
    pages, Hkv, page, _ = cache
    if not isinstance(page_table, torch.Tensor) or page_table.dtype is not torch.int32 \
            or page_table.get_device() != dev or page_table.dim() != 2:
        raise SLHError(f"page_table must be an int32 tensor of two dimensions on device {dev}")
    rows, most = page_table.shape
    ld, unit = page_table.stride()
    if rows != n or (unit != 1 and most > 1):
        raise SLHError(f"page_table must have shape ({n}, *) and unit stride in the last dimension")
    if n < 2 or ld < most:
        if n > 1:
            raise SLHError("page_table: rows must not overlap")
        ld = most
    ln = _plain("lens", lens, torch.int32, dev, (n,))
    pre = None
    if prefix_len:
        if prefix_pages is None:
            raise SLHError("prefix_pages must be given with a prefix_len")
        pre = _plain("prefix_pages", prefix_pages, torch.int32, dev, 1)
        if prefix_len < 0 or prefix_pages.shape[0] * page < prefix_len:
            raise SLHError("prefix_pages hold fewer rows than prefix_len")
    lse = None if lse_out is None else _plain("lse_out", lse_out, torch.float32, dev, shape[:-1])
    need = _bytes("slh_attend_paged_workspace", dev, (n, n_q, Hq, Hkv, d, most * page, prefix_len))
    workspace, ws = _workspace(need, dev, workspace, q.device, stream)
    _call("slh_attend_paged", dev, stream,
          (q.data_ptr(), qs[at], qs[-2], kc, vc, _DTYPES[dtype], pages, page, n, n_q, Hq, Hkv, d,
           page_table.data_ptr(), ld, most, ln, pre, prefix_len, 1.0 / math.sqrt(d) if scale is None else scale,
           out.data_ptr(), os[at], os[-2], lse, ws, need))
    return out
