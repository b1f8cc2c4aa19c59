"""Plain 64-bit forms of the operators of a smaller cache, from their definitions, for tests (on the CPU)."""
import math

import torch

CODE, SCALE = torch.float8_e4m3fn, torch.float8_e8m0fnu
MOST = {torch.float16: 8, torch.bfloat16: 120, torch.float32: 120}     # exponents of the largest powers in use


def power(top):
    """Exponent of the smallest power of two (from 2^-126) whose 448-fold reaches `top`."""
    x = -126
    while math.ldexp(448.0, x) < top:
        x += 1
    return x


def bytes_of(scales):
    return scales.view(torch.uint8).int()


def values(codes, scales):
    """What a cache stands for, [pages, H, page, d]."""
    p, H, ps, d = codes.shape
    n = scales.shape[2]
    two = torch.pow(torch.tensor(2.0, dtype=torch.float64), bytes_of(scales).double() - 127)
    return (codes.double().view(p, H, n, ps // n, d) * two[..., None, None]).view(p, H, ps, d)


def held(x, block):
    """x [pages, H, page, d] in 8 bits (codes, scales), by torch's own conversion."""
    p, H, ps, d = x.shape
    y = x.double().reshape(p, H, ps // block, block * d)
    top = y.abs().amax(-1)
    k = torch.tensor([power(float(t)) for t in top.flatten()]).view(top.shape)
    codes = (y * torch.pow(torch.tensor(2.0, dtype=torch.float64), -k.double())[..., None]).float().to(CODE)
    return codes.view(p, H, ps, d), (k + 127).to(torch.uint8).view(SCALE)


def half_step(y, k):
    """Half the distance between neighbouring codes around y, of a block with 2^k."""
    e = torch.floor(torch.log2((y.abs() * 2.0 ** -k).clamp(min=2.0 ** -6)))
    return torch.pow(torch.tensor(2.0, dtype=torch.float64), e - 4 + k)


def weights(q, k, lse, limit, scale):
    """w [Hkv, m] of rows q [n, Hq, d] over k [m, Hkv, d], lse [n, Hq]; row i sees the first limit[i] keys; and its tolerance.

    A weight is exp(x), x = scale s - lse: errors of s are those of d fp32 additions of products, 2 d 2^-24 scale sum |q| |k|;
    formed as 2^(s c - l) with c = scale log2(e) and l = lse log2(e) rounded, each by its constant's and its product's
    rounding, 2 2^-24 of |scale s| and of |lse|, and one more of x; the exponential 2^-23; a sum over n terms n 2^-24."""
    n, Hq, d = q.shape
    m, Hkv = k.shape[:2]
    g = Hq // Hkv
    w, tol = torch.zeros((Hkv, m), dtype=torch.float64), torch.zeros((Hkv, m), dtype=torch.float64)
    u = 2.0 ** -24
    for i in range(n):
        c = max(0, min(int(limit[i]), m))
        for h in range(Hq):
            if c == 0 or float(lse[i, h]) == -math.inf:
                continue
            kk, qq = k[:c, h // g].double(), q[i, h].double()
            s = kk @ qq * scale
            x = s - float(lse[i, h])
            p = torch.exp(x)
            e = 2 * d * u * (kk.abs() @ qq.abs()) * scale + 2 * u * (s.abs() + abs(float(lse[i, h]))) + 4 * u * x.abs() + 4 * u
            w[h // g, :c] += p
            tol[h // g, :c] += p * (e + n * g * u)
    return w, tol


def keep(w, n, budget, first, last):
    """Rows that stay of n with weights w, in order."""
    if n <= budget:
        return list(range(n))
    rank = sorted(range(first, n - last), key=lambda j: (-math.inf if math.isnan(w[j]) else -w[j], j))
    # NaN before every number, +inf included
    nan = [j for j in rank if math.isnan(w[j])]
    rank = nan + [j for j in rank if not math.isnan(w[j])]
    return sorted([*range(first), *rank[:budget - first - last], *range(n - last, n)])
