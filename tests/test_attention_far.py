"""Attention where scores are far from zero, up to fp32's end: slh_attend, slh_attend_paged and slh_attend_paged_e4m3."""
import math

import pytest
import torch

import cache_plain as CP
import paper_2607_19368_amd as P

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16


@pytest.mark.parametrize("dt,big_q,big_k,scale", [(BF, 2.0 ** 60, 1.5 * 2.0 ** 60, 0.3), (BF, 2.0 ** 60, -1.5 * 2.0 ** 60, 128.0), (BF, 2.0 ** 20, 1.5 * 2.0 ** 14, 0.3),
                                                  (BF, 2.0 ** 10, 1.5 * 2.0 ** 13, 0.69), (HF, 2.0 ** 14, 1.5 * 2.0 ** 14, 37.7),
                                                  (HF, -2.0 ** 14, 1.5 * 2.0 ** 14, 0.5), (HF, 2.0 ** 14, 1.75 * 2.0 ** 10, 0.5)])
@pytest.mark.parametrize("op,prefix", [("packed", 0), ("paged", 0), ("paged", 48), ("paged8", 0), ("paged8", 48)])
@pytest.mark.parametrize("d,n_q,Hq", [(64, 1, 3), (128, 3, 8), (80, 40, 1), (96, 130, 2), (128, 300, 7)])
def test_keys_that_take_all(dt, big_q, big_k, scale, op, prefix, d, n_q, Hq):
    """Two keys share all of a query's weight, or, for every other query, those with the opposite sign do: the mean of their values, and
    the score and ln 2 as lse."""
    g = torch.Generator()
    g.manual_seed(d + n_q)
    page, block = 16, 16
    m = -(-(prefix + 208 + n_q) // page) * page                      # keys, the prefix's first
    k = torch.randn(m, d, generator=g).clamp(-3, 3)
    k[:, 0] = 0
    pairs = ((3, 77), (52, 201))                                     # seen by all
    for (i, j), sign in zip(pairs, (1, -1)):
        k[[i, j]] = 0
        k[[i, j], 0] = sign * big_k
    v = torch.randn(m, d, generator=g)
    paged = [x.view(m // page, 1, page, d) for x in (k, v)]
    if op == "paged8":
        (kc, ks), (vc, vs) = (CP.held(x, block) for x in paged)
        k, v = CP.values(kc, ks).view(m, d), CP.values(vc, vs).view(m, d)
        assert float(k[3, 0]) == big_k and float(k[201, 0]) == -big_k
        cache = [kc.cuda(), vc.cuda(), ks.cuda(), vs.cuda()]
    else:
        cache = [x.to(dt).cuda() for x in paged]
        k, v = k.to(dt), v.to(dt)
    q = torch.randn(n_q, Hq, d, generator=g).to(dt)
    u = 1 - (torch.arange(n_q * Hq).view(n_q, Hq) % 100) / 256
    u = u * torch.where(torch.arange(Hq) % 2 == 1, -1, 1)            # heads of both signs in a block
    q[:, :, 0] = (big_q * u).to(dt)
    lse = torch.empty(n_q, Hq, device="cuda")
    if op == "packed":
        cu = [torch.tensor([0, n], dtype=torch.int32, device="cuda") for n in (n_q, m)]
        out = P.slh_attend(q.cuda(), k[:, None].cuda(), v[:, None].cuda(), *cu, scale=scale, lse_out=lse)
    else:
        call = P.slh_attend_paged_e4m3 if op == "paged8" else P.slh_attend_paged
        pages = torch.arange(m // page, dtype=torch.int32, device="cuda")
        out = call(q[None].cuda(), *cache, pages[None, prefix // page:].contiguous(), torch.tensor([m - prefix], dtype=torch.int32, device="cuda"),
                   pages[:prefix // page].clone(), prefix, scale=scale, lse_out=lse[None])[0]
    mean = torch.stack([(v[i].double() + v[j].double()) / 2 for i, j in pairs])
    positive = (u * big_q * big_k > 0)
    want = torch.where(positive[..., None], mean[0], mean[1])
    # the two weights are alike and powers of two, the rest 0: the output's rounding (subnormal fp16: 2^-25) beside fp32's
    off = (out.double().cpu() - want).abs()
    assert bool((off <= want.abs() * (torch.finfo(dt).eps / 2 + 2.0 ** -22) + 2.0 ** -25).all()), float(off.max())
    s = (big_q * big_k * u.double()).abs().float() * torch.tensor(scale, dtype=torch.float32)
    # the score, exact, times the scale, and ln 2 and a sum, each rounded once
    assert bool(((lse.cpu().double() - (s.double() + math.log(2))).abs() <= s.double() * 2.0 ** -22 + 2.0 ** -22).all())
