"""The operators of a smaller cache at the ends of what their contracts allow: powers of two that only a cache from elsewhere
holds."""
import pytest
import torch

import cache_plain as CP
import paper_2607_19368_amd as P

gpu = pytest.mark.gpu


def _gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


# ---------------------------------------------------------------- eviction
@gpu
@pytest.mark.parametrize("d", [64, 80, 96, 128])
@pytest.mark.parametrize("page,block", [(16, 16), (64, 32), (256, 256)])
@pytest.mark.parametrize("powers", [(248,), (254,), (1, 247, 250, 254), (253, 254), (1, 2, 9, 17), (1, 120, 127, 135, 247, 248)])
def test_evict_powers_of_both_ends(d, page, block, powers):
    """Blocks of every power from 2^-126 to 2^127 and every code: what stays keeps its values, exactly but for codes that become subnormal."""
    g = _gen(d + block + powers[-1])
    H, n, budget, first, last = 2, 590, 331, 3, 5
    width = -(-n // page)
    total = width + 1
    table = torch.randperm(total, generator=g).int()[:width][None]
    kc, vc = (torch.randint(0, 256, (total, H, page, d), generator=g).to(torch.uint8) for _ in range(2))
    for c in (kc, vc):
        c[:, 0] &= 0x8f                              # a head of small codes beside one of all, NaN among them
        c[:, 1, 1::2][c[:, 1, 1::2] & 0x7f == 0x7f] = 0x7e
        c[:, 1, ::16] = 0
    ks, vs = (torch.tensor(powers)[torch.randint(0, len(powers), (total, H, page // block), generator=g)].to(torch.uint8) for _ in range(2))
    w = torch.rand(1, H, width * page, generator=g)
    held = [x.clone().cuda() for x in (kc.view(CP.CODE), vc.view(CP.CODE), ks.view(CP.SCALE), vs.view(CP.SCALE))]
    P.slh_kv_evict(held[0], held[1], w.cuda(), table.cuda(), torch.tensor([n], dtype=torch.int32).cuda(), budget, first, last, held[2], held[3])
    for codes, scales, got, got_two in ((kc, ks, held[0], held[2]), (vc, vs, held[1], held[3])):
        val = CP.values(codes.view(CP.CODE), scales.view(CP.SCALE))
        for h in range(H):
            stay = CP.keep(w[0, h].tolist(), n, budget, first, last)
            for i0 in range(0, budget, block):
                y = torch.stack([val[int(table[0, j // page]), h, j % page] for j in stay[i0:i0 + block]])
                k = CP.power(float(y.nan_to_num(nan=0.0).abs().max()))
                p, at = int(table[0, i0 // page]), i0 % page
                assert int(got_two[p, h, at // block].cpu().view(torch.uint8)) == k + 127, (h, i0)
                want = (y * 2.0 ** -k).float().to(CP.CODE)          # to nearest even: exact where no code becomes subnormal
                have = got[p, h, at:at + len(y)].cpu()
                nan = torch.isnan(y)
                assert torch.equal(torch.isnan(have.float()), nan), (h, i0)
                assert torch.equal(have.view(torch.uint8)[~nan], want.view(torch.uint8)[~nan]), (h, i0)
