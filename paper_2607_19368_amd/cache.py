"""Python binding of the operators of a smaller cache (include/slh.h): a paged cache held in 8 bits, the attention
weight that cached keys receive, and eviction by it.  Argument checks and marshalling, as in attention.py; calls go to
torch's current stream, or to the `stream` given, and return without waiting for it.

A cache in 8 bits is two tensors of codes [pages, H, page, d] (torch.float8_e4m3fn) and two of scales
[pages, H, page / block] (torch.float8_e8m0fnu: powers of two), one scale for each `block` rows of a
page and head; a code stands for code * scale.  page and block: powers of two, 16 <= block <= 256, block <= page.
"""
import math

import torch

from . import slh as B
from .attention import (_DTYPES, _HALVES, _bytes, _call, _empty, _first, _plain, _rotation, _rows, _workspace)
from .slh import SLHError

_CODE, _SCALE = torch.float8_e4m3fn, torch.float8_e8m0fnu


def _held(k_cache, v_cache, k_scale, v_scale, dev):
    """(codes' and scales' addresses, cache shape, block) of a cache in 8 bits; v_cache may be None."""
    kc = _plain("k_cache", k_cache, _CODE, dev, 4)
    shape = k_cache.shape
    ks = _plain("k_scale", k_scale, _SCALE, dev, 3)
    blocks = k_scale.shape
    if blocks[:2] != shape[:2] or blocks[2] < 1 or shape[2] % blocks[2]:
        raise SLHError("k_scale must have the cache's pages and heads and a whole number of rows a block")
    if v_cache is None:
        return (kc, ks), shape, shape[2] // blocks[2]
    vc = _plain("v_cache", v_cache, _CODE, dev, shape)
    vs = _plain("v_scale", v_scale, _SCALE, dev, blocks)
    return (kc, vc, ks, vs), shape, shape[2] // blocks[2]


def _pages(page_table, dev, n):
    """(address, row stride, width) of a page table of n sequences."""
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
    return page_table.data_ptr(), ld, most


def _lens(lens, dev):
    at = _plain("lens", lens, torch.int32, dev, 1)
    return at, lens.shape[0]


def slh_kv_append_e4m3(k, v, k_cache, v_cache, k_scale, v_scale, page_table, lens, cu=None, k_weight=None, eps=1e-6, table=None,
                       pos=None, interleaved=False, stream=None):
    """Writes k and v [T, H, d] (bf16, fp16 or fp32) into a cache in 8 bits, the keys normed and rotated on the way as in
    slh_qk_norm_rope.  Tokens cu[b]..cu[b + 1] (int32; None: T / B each) become the last rows of sequence b's
    lens[b] (int32, the new rows counted) in its pages page_table[b] (int32 [B, n]).  A block's scale is the smallest
    power of two whose 448-fold reaches its rows, and never falls while earlier rows of the sequence are in it: those
    are rescaled where it grows.  Returns the caches and scales."""
    dtype, dev, shape, ks = _first("k", k, (3,))
    vs = _rows("v", v, dtype, dev, shape)
    T, H, d = shape
    held, cache, block = _held(k_cache, v_cache, k_scale, v_scale, dev)
    if cache[1] != H or cache[3] != d:
        raise SLHError(f"k_cache must have shape (*, {H}, *, {d})")
    ln, n = _lens(lens, dev)
    pages, ld, most = _pages(page_table, dev, n)
    if cu is None:
        if T % n if n else T:
            raise SLHError("without cu, k must hold as many tokens of each sequence")
        cq = None
    else:
        cq = _plain("cu", cu, torch.int32, dev, (n + 1,))
    tab, n_pos, rot, p = _rotation(table, pos, T, dev)
    wk = None if k_weight is None else _plain("k_weight", k_weight, dtype, dev, (d,))
    _call("slh_kv_append_e4m3", dev, stream,
          (k.data_ptr(), ks[0], ks[1], v.data_ptr(), vs[0], vs[1], _DTYPES[dtype], T, n, H, d, wk, eps, tab, n_pos, rot, p,
           interleaved, *held, cache[0], cache[2], block, pages, ld, most, ln, cq))
    return k_cache, v_cache, k_scale, v_scale


def slh_attend_paged_e4m3_workspace(B_, n_q, Hq, Hkv, d, max_len, prefix_len):
    """Bytes that slh_attend_paged_e4m3 needs as workspace on the current device."""
    return int(B.load().slh_attend_paged_e4m3_workspace(B_, n_q, Hq, Hkv, d, max_len, prefix_len))


def slh_attend_paged_e4m3(q, k_cache, v_cache, k_scale, v_scale, page_table, lens, prefix_pages=None, prefix_len=0, scale=None,
                          out=None, lse_out=None, workspace=None, stream=None):
    """slh_attend_paged against a cache in 8 bits: the new tokens q [B, n_q, Hq, d] (or [B, Hq, d]: one each) of a
    batch, bf16 or fp16, behind a prefix that all sequences share.  Returns out."""
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
    held, cache, block = _held(k_cache, v_cache, k_scale, v_scale, dev)
    total, Hkv, page, width = cache
    if width != d:
        raise SLHError("k_cache must have q's head size")
    pages, ld, most = _pages(page_table, dev, n)
    ln = _plain("lens", lens, torch.int32, dev, (n,))
    pre = None
    if prefix_len:
        if prefix_pages is None:
            raise SLHError("prefix_pages must be given with a prefix_len")
        pre = _plain("prefix_pages", prefix_pages, torch.int32, dev, 1)
        if prefix_len < 0 or prefix_pages.shape[0] * page < prefix_len:
            raise SLHError("prefix_pages hold fewer rows than prefix_len")
    lse = None if lse_out is None else _plain("lse_out", lse_out, torch.float32, dev, shape[:-1])
    need = _bytes("slh_attend_paged_e4m3_workspace", dev, (n, n_q, Hq, Hkv, d, most * page, prefix_len))
    workspace, ws = _workspace(need, dev, workspace, q.device, stream)
    _call("slh_attend_paged_e4m3", dev, stream,
          (q.data_ptr(), qs[at], qs[-2], *held, _DTYPES[dtype], total, page, block, n, n_q, Hq, Hkv, d, pages, ld, most, ln, pre,
           prefix_len, 1.0 / math.sqrt(d) if scale is None else scale, out.data_ptr(), os[at], os[-2], lse, ws, need))
    return out


def slh_attend_weights_workspace(Tq, B_, Hq, Hkv, d, max_len):
    """Bytes that slh_attend_weights needs as workspace on the current device."""
    return int(B.load().slh_attend_weights_workspace(Tq, B_, Hq, Hkv, d, max_len))


def slh_attend_weights(q, k_cache, page_table, lens, lse, weights, cu_q=None, k_scale=None, scale=None, workspace=None, stream=None):
    """Adds to weights [B, Hkv, n * page] (float32) the attention weight exp(scale q_i . k_j - lse_i) that each cached row
    j < lens[b] of sequence b received from its queries, summed over them and over the query heads of its key/value head.
    q: [B, n_q, Hq, d], [B, Hq, d], or with cu_q (int32 [B + 1]) [Tq, Hq, d] packed; a sequence's last query sees all
    its rows, the one before it one fewer, and so on.  lse (float32, q's shape without d): what the attention call of
    these queries gave as lse_out.  k_cache: q's type, or 8 bits with k_scale.  Returns weights."""
    dtype, dev, shape, qs = _first("q", q, (3,) if cu_q is not None else (3, 4))
    if dtype not in _HALVES:
        raise SLHError("q must be bfloat16 or float16")
    ln, n = _lens(lens, dev)
    Hq, d = shape[-2], shape[-1]
    at = 0
    if cu_q is not None:
        cq, Tq = _plain("cu_q", cu_q, torch.int32, dev, (n + 1,)), shape[0]
    else:
        cq, n_q = None, shape[1] if len(shape) == 4 else 1
        Tq = n * n_q
        if shape[0] != n:
            raise SLHError("q must have as many sequences as lens")
        if n_q > 1 and n > 1 and qs[0] != n_q * qs[1]:
            raise SLHError("q: sequences must follow one another as their tokens do")
        at = 1 if n_q > 1 else 0
    if k_scale is None:
        kc = _plain("k_cache", k_cache, dtype, dev, 4)
        cache, block, ks = k_cache.shape, 0, None
    else:
        (kc, ks), cache, block = _held(k_cache, None, k_scale, None, dev)
    total, Hkv, page, width = cache
    if width != d:
        raise SLHError("k_cache must have q's head size")
    pages, ld, most = _pages(page_table, dev, n)
    ls = _plain("lse", lse, torch.float32, dev, shape[:-1])
    w = _plain("weights", weights, torch.float32, dev, (n, Hkv, most * page))
    need = _bytes("slh_attend_weights_workspace", dev, (Tq, n, Hq, Hkv, d, most * page))
    workspace, ws = _workspace(need, dev, workspace, q.device, stream)
    _call("slh_attend_weights", dev, stream,
          (q.data_ptr(), qs[at], qs[-2], kc, ks, _DTYPES[dtype], total, page, block, Tq, n, Hq, Hkv, d, pages, ld, most, ln, cq, ls,
           1.0 / math.sqrt(d) if scale is None else scale, w, ws, need))
    return weights


def slh_kv_evict_workspace(B_, H, d, dtype, budget, max_len):
    """Bytes that slh_kv_evict needs as workspace on the current device, for caches of the torch type `dtype` and tables of
    max_len rows a sequence."""
    return int(B.load().slh_kv_evict_workspace(B_, H, d, B.SLH_E4M3 if dtype is _CODE else _DTYPES[dtype], budget, max_len))


def slh_kv_evict(k_cache, v_cache, weights, page_table, lens, budget, first=0, last=0, k_scale=None, v_scale=None, weights_out=None,
                 lens_out=None, kept=None, workspace=None, stream=None):
    """Cuts each sequence of more than `budget` rows to that many, head by head: the first `first` and last `last` rows stay, and
    of the others those with the largest weights [B, H, n * page] (float32; equal ones: the first rows; NaN counts as
    the largest).  What stays moves in its order to the first rows of the sequence's pages, with its weights; rows
    behind are as they were, with weights of zero.  Caches [pages, H, page, d] of any element type, or in 8
    bits with k_scale and v_scale.  Returns (weights_out, lens_out, kept): kept [B, H, budget] int32 says which row
    each came from (-1: none); weights_out and lens_out may be weights and lens."""
    if not isinstance(k_cache, torch.Tensor) or not k_cache.is_cuda:
        raise SLHError("k_cache must be a device tensor")
    dtype, dev = k_cache.dtype, k_cache.get_device()
    ln, n = _lens(lens, dev)
    if k_scale is not None or v_scale is not None:
        held, cache, block = _held(k_cache, v_cache, k_scale, v_scale, dev)
        code = B.SLH_E4M3
    else:
        if dtype not in _DTYPES:
            raise SLHError(f"k_cache: unsupported type {dtype}")
        kc = _plain("k_cache", k_cache, dtype, dev, 4)
        cache, block, code = k_cache.shape, 0, _DTYPES[dtype]
        held = (kc, _plain("v_cache", v_cache, dtype, dev, cache), None, None)
    total, H, page, d = cache
    pages, ld, most = _pages(page_table, dev, n)
    shape = (n, H, most * page)
    w = _plain("weights", weights, torch.float32, dev, shape)
    if weights_out is None:
        weights_out = _empty(shape, torch.float32, k_cache.device, stream)
    if lens_out is None:
        lens_out = _empty((n,), torch.int32, k_cache.device, stream)
    if kept is None:
        kept = _empty((n, H, max(budget, 0)), torch.int32, k_cache.device, stream)
    wo = _plain("weights_out", weights_out, torch.float32, dev, shape)
    lo = _plain("lens_out", lens_out, torch.int32, dev, (n,))
    kp = _plain("kept", kept, torch.int32, dev, (n, H, budget))
    need = _bytes("slh_kv_evict_workspace", dev, (n, H, d, code, budget, most * page))
    workspace, ws = _workspace(need, dev, workspace, k_cache.device, stream)
    _call("slh_kv_evict", dev, stream,
          (*held, code, total, page, block, n, H, d, pages, ld, most, ln, lo, w, wo, budget, first, last, kp, ws, need))
    return weights_out, lens_out, kept
