"""Plain 64-bit forms of the attention operators, from their definitions, for tests."""
import math

import torch

# unit roundoff of the element types: half a unit in the last place of 8, 11 and 24 bits
U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}


def norm_rope(x, w, eps, table, pos, interleaved):
    """Rows x [T, H, d] normed and rotated, in 64 bits, and the magnitude that their errors go by."""
    y = x.double().clone()
    if w is not None:
        y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + eps) * w.double()
    size = y.abs()
    if table is not None:
        half = table.shape[2]
        c, s = (table[pos.long(), i].double()[:, None] for i in (0, 1))
        ia = torch.arange(half) * 2 if interleaved else torch.arange(half)
        ib = ia + 1 if interleaved else ia + half
        a, b = y[..., ia].clone(), y[..., ib].clone()
        y[..., ia], y[..., ib] = a * c - b * s, b * c + a * s
        both = a.abs() + b.abs()
        size[..., ia], size[..., ib] = both, both
    return y, size


def one_row(q, k, v, scale, dtype):
    """(o, tolerance, lse, its tolerance) of one query q [d] over the keys that it sees.

    Tolerance of an element of o, A = sum p |v| / sum p:  the output's rounding u |o|; the
    weights' rounding u A (and in fp16, whose smallest step is 2^-24, 2^-25 a weight of those at
    most 1, so 2^-25 n max |v| / sum p); errors of the scores, at most e, change each weight by a
    factor e^+-e, so o by at most 2 e A.  e: d fp32 additions of products, the scaled score's and
    the maximum's rounding, the exponential: (d + 8) 2^-24 (scale sum |q| |k| + 1) with the constant
    doubled; sums over n weights in fp32, n 2^-24 A at most, twice (numerator and denominator)."""
    d = q.shape[-1]
    if len(k) == 0:
        z = torch.zeros(d, dtype=torch.float64)
        return z, z, torch.tensor(-math.inf, dtype=torch.float64), 0.0
    s = (k @ q) * scale
    top = s.max()
    p = torch.exp(s - top)
    total = p.sum()
    o = (p @ v) / total
    A = (p @ v.abs()) / total
    u = U[dtype]
    e = 2 * (d + 8) * 2.0 ** -24 * (float(((k.abs() @ q.abs()) * scale).max()) + 1.0)
    tol = 1.02 * u * (o.abs() + A) + 2 * (e + len(k) * 2.0 ** -24) * A
    if dtype == torch.float16:
        tol = tol + 2.0 ** -25 * v.abs().sum(0) / total + 2.0 ** -25
    return o, tol, torch.log(total) + top, e + (len(k) + 8) * 2.0 ** -24 * (1 + float(abs(top)))


def attend(q, k, v, limit, scale):
    """Rows of q [n, Hq, d] over k, v [m, Hkv, d]; row i sees the first limit[i] keys."""
    n, Hq, d = q.shape
    g = Hq // k.shape[1]
    o, tol = torch.zeros((n, Hq, d), dtype=torch.float64), torch.zeros((n, Hq, d), dtype=torch.float64)
    lse, ltol = torch.zeros((n, Hq), dtype=torch.float64), torch.zeros((n, Hq), dtype=torch.float64)
    qd, kd, vd = q.double(), k.double(), v.double()
    for i in range(n):
        m = max(0, min(int(limit[i]), len(k)))
        for h in range(Hq):
            o[i, h], tol[i, h], lse[i, h], ltol[i, h] = one_row(qd[i, h], kd[:m, h // g], vd[:m, h // g], scale, q.dtype)
    return o, tol, lse, ltol
