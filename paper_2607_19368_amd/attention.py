"""Python binding of the operators behind a compressed prompt (include/slh.h): argument
checks and marshalling, as in slh.py.  Every call goes to torch's current stream, or to the
`stream` given (a torch.cuda.Stream), and returns without waiting for it.
"""
import math

import torch

from . import slh as B
from .slh import SLHError

_DTYPES = {torch.bfloat16: B.SLH_BF16, torch.float16: B.SLH_F16, torch.float32: B.SLH_F32}
_HALVES = (torch.bfloat16, torch.float16)


def _fail(what, rc):
    raise SLHError(f"{what} failed ({rc}): " + {
        B.SLH_EINVAL: "a size, stride or alignment that the library does not take",
        B.SLH_EHIP: "a kernel launch failed"}.get(rc, ""))


def _stream(stream, device):
    return (torch.cuda.current_stream(device) if stream is None else stream).cuda_stream


def _rows(name, t, dims=3, like=None, shape=None):
    """t: a device tensor of rows ([token, head, element] at its end) with unit element stride; of
    the type and device of `like` and of `shape`, where given."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise SLHError(f"{name} must be a device tensor")
    if t.dim() != dims or (t.stride(-1) != 1 and t.numel() > 0):
        raise SLHError(f"{name} must have {dims} dimensions and unit stride in the last")
    if t.dtype not in _DTYPES:
        raise SLHError(f"{name}: unsupported type {t.dtype}")
    if like is not None and (t.dtype != like.dtype or t.device != like.device):
        raise SLHError(f"{name} must be {like.dtype} on {like.device}")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise SLHError(f"{name} must have shape {tuple(shape)}")


def _plain(name, t, dtype, device, shape):
    """t: a contiguous device tensor of `dtype` and `shape` (None: any length)."""
    if not isinstance(t, torch.Tensor) or t.dtype != dtype or t.device != device or not t.is_contiguous():
        raise SLHError(f"{name} must be a contiguous {dtype} tensor on {device}")
    if t.dim() != len(shape) or any(n is not None and n != m for n, m in zip(shape, t.shape)):
        raise SLHError(f"{name} must have shape ({', '.join('*' if n is None else str(n) for n in shape)})")


def _rotation(table, pos, T, device):
    """(table pointer, n_pos, rot_dim, pos pointer) of a rotation, or of none."""
    if table is None:
        return None, 0, 0, None
    _plain("table", table, torch.float32, device, (None, 2, None))
    if pos is None:
        raise SLHError("pos must be given with a table")
    _plain("pos", pos, torch.int32, device, (T,))
    return table.data_ptr(), table.shape[0], 2 * table.shape[2], pos.data_ptr()


def _weight(name, w, x):
    if w is None:
        return None
    _plain(name, w, x.dtype, x.device, (x.shape[-1],))
    return w.data_ptr()


def _address(t):
    return None if t is None else t.data_ptr()


def slh_rope_table(n_pos, rot_dim, base=10000.0, scaling=B.SLH_ROPE_PLAIN, factor=1.0, orig_len=0,
                   beta_fast=32.0, beta_slow=1.0, device="cuda", stream=None):
    """Table [n_pos, 2, rot_dim / 2] float32 of cosines and sines for slh_qk_norm_rope and
    slh_kv_append; `scaling` is one of SLH_ROPE_PLAIN, _LINEAR, _BASE and _BANDS."""
    if n_pos < 1 or rot_dim < 16 or rot_dim > 256 or rot_dim % 16:
        raise SLHError("n_pos must be positive and rot_dim a multiple of 16 from 16 to 256")
    table = torch.empty((n_pos, 2, rot_dim // 2), dtype=torch.float32, device=device)
    with torch.cuda.device(table.device):
        rc = B.load().slh_rope_table(table.data_ptr(), n_pos, rot_dim, float(base), int(scaling), float(factor),
                                     int(orig_len), float(beta_fast), float(beta_slow), _stream(stream, table.device))
    if rc != B.SLH_OK:
        _fail("slh_rope_table", rc)
    return table


def slh_qk_norm_rope(q, k=None, q_weight=None, k_weight=None, eps=1e-6, table=None, pos=None, interleaved=False,
                     q_out=None, k_out=None, stream=None):
    """Queries [T, Hq, d] and keys [T, Hk, d] (either may be None): RMS norm per head where a
    weight [d] is given, rotation by the table's rows `pos` [T] int32 where a table is.  Returns
    (q_out, k_out), which may be the inputs themselves."""
    x = q if q is not None else k
    if x is None:
        raise SLHError("q or k must be given")
    args = []
    shape = None
    outs = []
    for name, t, out in (("q", q, q_out), ("k", k, k_out)):
        if t is None:
            args += (None, 0, 0, 0, None, 0, 0)
            outs.append(None)
            continue
        _rows(name, t, 3, x)
        if shape is not None and (t.shape[0], t.shape[2]) != shape:
            raise SLHError("q and k must have the same tokens and head size")
        shape = (t.shape[0], t.shape[2])
        if out is None:
            out = torch.empty(t.shape, dtype=t.dtype, device=t.device)
        else:
            _rows(name + "_out", out, 3, t, t.shape)
        args += (t.data_ptr(), t.stride(0), t.stride(1), t.shape[1], out.data_ptr(), out.stride(0), out.stride(1))
        outs.append(out)
    T, d = shape
    tab, n_pos, rot, p = _rotation(table, pos, T, x.device)
    wq = _weight("q_weight", q_weight, x)
    wk = _weight("k_weight", k_weight, x)
    with torch.cuda.device(x.device):
        rc = B.load().slh_qk_norm_rope(*args, _DTYPES[x.dtype], T, d, wq, wk, float(eps), tab, n_pos, rot, p,
                                       int(interleaved), _stream(stream, x.device))
    if rc != B.SLH_OK:
        _fail("slh_qk_norm_rope", rc)
    return tuple(outs)


def slh_kv_append(k, v, k_cache, v_cache, slots, k_weight=None, eps=1e-6, table=None, pos=None, interleaved=False,
                  stream=None):
    """Writes k and v [T, H, d] into the caches [pages, H, page, d] at rows `slots` [T] int64
    (page * page size + row; negative: left out), the keys normed and rotated on the way as
    in slh_qk_norm_rope.  Returns the caches."""
    _rows("k", k)
    _rows("v", v, 3, k, k.shape)
    T, H, d = k.shape
    _plain("k_cache", k_cache, k.dtype, k.device, (None, H, None, d))
    _plain("v_cache", v_cache, k.dtype, k.device, k_cache.shape)
    _plain("slots", slots, torch.int64, k.device, (T,))
    tab, n_pos, rot, p = _rotation(table, pos, T, k.device)
    wk = _weight("k_weight", k_weight, k)
    with torch.cuda.device(k.device):
        rc = B.load().slh_kv_append(k.data_ptr(), k.stride(0), k.stride(1), v.data_ptr(), v.stride(0), v.stride(1),
                                    _DTYPES[k.dtype], T, H, d, wk, float(eps), tab, n_pos, rot, p, int(interleaved),
                                    k_cache.data_ptr(), v_cache.data_ptr(), k_cache.shape[0], k_cache.shape[2],
                                    slots.data_ptr(), _stream(stream, k.device))
    if rc != B.SLH_OK:
        _fail("slh_kv_append", rc)
    return k_cache, v_cache


def _workspace(workspace, need, device):
    """(tensor, pointer) of a workspace of `need` bytes: the given one, or a new one."""
    if need < 0:
        raise SLHError("sizes that the library does not take")
    if need == 0:
        return None, None
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=device)
    else:
        _plain("workspace", workspace, torch.uint8, device, (None,))
        if workspace.numel() < need:
            raise SLHError(f"workspace must hold {need} bytes")
    return workspace, workspace.data_ptr()


def slh_attend_workspace(Tq, Tk, B_, Hq, Hkv, d):
    """Bytes that slh_attend needs as workspace on the current device."""
    return int(B.load().slh_attend_workspace(Tq, Tk, B_, Hq, Hkv, d))


def slh_attend(q, k, v, cu_q, cu_k=None, scale=None, causal=True, out=None, lse_out=None, workspace=None,
               stream=None):
    """Attention of packed sequences: q [Tq, Hq, d], k and v [Tk, Hkv, d] (bf16 or fp16), sequence b
    at rows cu_q[b]..cu_q[b + 1] of q and cu_k[b]..cu_k[b + 1] of k and v (int32; cu_k None: as cu_q).
    causal: a sequence's last query sees all its keys, the one before it one fewer, and so on.
    scale: 1 / sqrt(d) by default.  lse_out: [Tq, Hq] float32.  Returns out."""
    _rows("q", q)
    _rows("k", k, 3, q)
    _rows("v", v, 3, q, k.shape)
    if q.dtype not in _HALVES:
        raise SLHError("q must be bfloat16 or float16")
    Tq, Hq, d = q.shape
    Tk, Hkv, dk = k.shape
    if dk != d:
        raise SLHError("q and k must have the same head size")
    if cu_k is None:
        cu_k = cu_q
    dev = q.device
    _plain("cu_q", cu_q, torch.int32, dev, (None,))
    _plain("cu_k", cu_k, torch.int32, dev, cu_q.shape)
    n = cu_q.shape[0] - 1
    if n < 0:
        raise SLHError("cu_q must have an entry more than there are sequences")
    if out is None:
        out = torch.empty((Tq, Hq, d), dtype=q.dtype, device=dev)
    else:
        _rows("out", out, 3, q, q.shape)
    if lse_out is not None:
        _plain("lse_out", lse_out, torch.float32, dev, (Tq, Hq))
    lib = B.load()
    with torch.cuda.device(dev):
        need = lib.slh_attend_workspace(Tq, Tk, n, Hq, Hkv, d)
        st = _stream(stream, dev)
        if stream is not None and workspace is None:
            with torch.cuda.stream(stream):
                workspace, ws = _workspace(None, need, dev)
        else:
            workspace, ws = _workspace(workspace, need, dev)
        rc = lib.slh_attend(q.data_ptr(), q.stride(0), q.stride(1), k.data_ptr(), k.stride(0), k.stride(1),
                            v.data_ptr(), v.stride(0), v.stride(1), _DTYPES[q.dtype], Tq, Tk, n, Hq, Hkv, d,
                            cu_q.data_ptr(), cu_k.data_ptr(), 1.0 / math.sqrt(d) if scale is None else scale,
                            int(causal), out.data_ptr(), out.stride(0), out.stride(1), _address(lse_out), ws, need,
                            st)
    if rc != B.SLH_OK:
        _fail("slh_attend", rc)
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
    _rows("q", q, q.dim() if isinstance(q, torch.Tensor) and q.dim() in (3, 4) else 4)
    if q.dtype not in _HALVES:
        raise SLHError("q must be bfloat16 or float16")
    dev = q.device
    if out is None:
        out = torch.empty(q.shape, dtype=q.dtype, device=dev)
    else:
        _rows("out", out, q.dim(), q, q.shape)
    n, Hq, d = q.shape[0], q.shape[-2], q.shape[-1]
    n_q = q.shape[1] if q.dim() == 4 else 1
    if n_q > 1 and n > 1:
        for name, t in (("q", q), ("out", out)):
            if t.stride(0) != n_q * t.stride(1):
                raise SLHError(f"{name}: sequences must follow one another as their tokens do")
    at = 1 if n_q > 1 else 0                # the dimension whose stride is a token's
    _plain("k_cache", k_cache, q.dtype, dev, (None, None, None, d))
    _plain("v_cache", v_cache, q.dtype, dev, k_cache.shape)
    pages, Hkv, page, _ = k_cache.shape
    if not isinstance(page_table, torch.Tensor) or page_table.dtype != torch.int32 or page_table.device != dev \
            or page_table.dim() != 2 or page_table.shape[0] != n or (page_table.shape[1] > 1 and page_table.stride(1) != 1):
        raise SLHError(f"page_table must be an int32 tensor ({n}, *) on {dev} with unit stride in the last dimension")
    most = page_table.shape[1]
    ld = page_table.stride(0) if n > 1 else max(most, 1)
    _plain("lens", lens, torch.int32, dev, (n,))
    prefix_len = int(prefix_len)
    if prefix_len:
        if prefix_pages is None:
            raise SLHError("prefix_pages must be given with a prefix_len")
        _plain("prefix_pages", prefix_pages, torch.int32, dev, (None,))
        if prefix_len < 0 or prefix_pages.shape[0] * page < prefix_len:
            raise SLHError("prefix_pages hold fewer rows than prefix_len")
    if lse_out is not None:
        _plain("lse_out", lse_out, torch.float32, dev, q.shape[:-1])
    lib = B.load()
    with torch.cuda.device(dev):
        need = lib.slh_attend_paged_workspace(n, n_q, Hq, Hkv, d, most * page, prefix_len)
        st = _stream(stream, dev)
        if stream is not None and workspace is None:
            with torch.cuda.stream(stream):
                workspace, ws = _workspace(None, need, dev)
        else:
            workspace, ws = _workspace(workspace, need, dev)
        rc = lib.slh_attend_paged(q.data_ptr(), q.stride(at), q.stride(-2), k_cache.data_ptr(), v_cache.data_ptr(),
                                  _DTYPES[q.dtype], pages, page, n, n_q, Hq, Hkv, d, page_table.data_ptr(), ld, most,
                                  lens.data_ptr(), _address(prefix_pages) if prefix_len else None, prefix_len,
                                  1.0 / math.sqrt(d) if scale is None else scale, out.data_ptr(), out.stride(at),
                                  out.stride(-2), _address(lse_out), ws, need, st)
    if rc != B.SLH_OK:
        _fail("slh_attend_paged", rc)
    return out
