"""The operators of a smaller cache at the ends of what their contracts allow: powers of two that only a cache from elsewhere
holds, scores far from zero."""
import ctypes
import math
import os
import subprocess

import pytest
import torch

import cache_plain as CP
import paper_2607_19368_amd as P
from paper_2607_19368_amd import build as BUILD

gpu = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16


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


# ---------------------------------------------------------------- weights
def _far_case(d, dt, block, n, n_q, Hq, at, big_q, big_k, seed):
    """A cache of one sequence whose key `at` is (big_k, 0, ...), and queries (big_q u_i, ...) with u_i in eight bits."""
    g = _gen(seed)
    page = 32
    width = -(-n // page)
    x = torch.randn(width, 1, page, d, generator=g).clamp(-4, 4)
    x[at // page, 0, at % page] = 0
    x[at // page, 0, at % page, 0] = big_k
    q = torch.randn(1, n_q, Hq, d, generator=g).to(dt)
    u = 1 - (torch.arange(n_q * Hq).view(n_q, Hq) % 100) / 256
    q[0, :, :, 0] = (big_q * u).to(dt)
    assert bool((q[0, :, :, 0].double() == big_q * u.double()).all())
    if block:
        kc, ks = CP.held(x, block)
        k16 = None
        assert float(CP.values(kc, ks)[at // page, 0, at % page, 0]) == big_k
    else:
        kc, ks = x.to(dt), None
    return q.cuda(), kc.cuda(), None if ks is None else ks.cuda(), torch.arange(width, dtype=torch.int32).cuda()[None], torch.tensor([n], dtype=torch.int32).cuda(), u


@gpu
@pytest.mark.parametrize("dt,big_q,big_k,scale", [(BF, 2.0 ** 60, 1.5 * 2.0 ** 60, 128.0), (BF, 2.0 ** 60, 1.5 * 2.0 ** 60, 0.3), (BF, 2.0 ** 20, 1.5 * 2.0 ** 14, 0.3),
                                                  (BF, 2.0 ** 20, 2.0 ** 20, 1e26), (HF, 2.0 ** 14, 1.5 * 2.0 ** 14, 37.7), (HF, 2.0 ** 10, 1.75 * 2.0 ** 13, 0.7)])
@pytest.mark.parametrize("block", [0, 16])
@pytest.mark.parametrize("d,n_q", [(64, 2), (80, 3), (96, 130), (128, 2), (128, 150)])
def test_weights_of_a_key_that_takes_all(dt, big_q, big_k, scale, block, d, n_q):
    """Scores up to fp32's end, whatever the scale: the key that has all of a query's weight gets 1 from it, the others nothing."""
    n, Hq, at = 300, 2, 77
    q, kc, ks, table, lens, u = _far_case(d, dt, block, n, n_q, Hq, at, big_q, big_k, d + n_q)
    lse = torch.empty(1, n_q, Hq, device="cuda")
    if block:
        P.slh_attend_paged_e4m3(q, kc, torch.zeros_like(kc.view(torch.uint8)).view(CP.CODE), ks, ks, table, lens, scale=scale, lse_out=lse)
    else:
        P.slh_attend_paged(q, kc, torch.zeros_like(kc), table, lens, scale=scale, lse_out=lse)
    # one product, exact in fp32, times the scale in fp32
    s = (big_q * big_k * u.double()).float()
    assert torch.equal(lse[0].cpu(), s * torch.tensor(scale, dtype=torch.float32))
    w = torch.zeros(1, 1, table.shape[1] * 32, device="cuda")
    P.slh_attend_weights(q, kc, table, lens, lse, w, k_scale=ks, scale=scale)
    want = torch.zeros(w.shape)
    want[0, 0, at] = n_q * Hq
    assert torch.equal(w.cpu(), want)


@gpu
@pytest.mark.parametrize("scale", [1.0, 8.0, 2.0 ** -60])
@pytest.mark.parametrize("block", [0, 16])
@pytest.mark.parametrize("d,n_q", [(64, 2), (128, 17), (80, 140)])
def test_weights_of_large_and_ordinary_scores(scale, block, d, n_q):
    """Scores of 2560 and of 6400 in turn, by row: each within what fp32 holds of them; queries with an lse of either infinity give nothing."""
    g = _gen(n_q)
    n, Hq, page = 400, 2, 16
    x = torch.randn(n // page, 1, page, d, generator=g)
    x[..., 0] = 64
    if block:
        kc, ks = CP.held(x, block)
        k = CP.values(kc, ks)
    else:
        kc, ks = x.to(BF), None
        k = kc.double()
    k = k.transpose(1, 2).flatten(0, 1)
    q = torch.randn(n_q, Hq, d, generator=g)
    q[:, :, 0] = torch.where(torch.arange(n_q * Hq).view(n_q, Hq) % 3 == 0, 100, 40)
    q = (q / scale ** 0.5).to(BF)
    if scale == 2.0 ** -60:
        q = q * 2.0 ** 30
    s = torch.einsum("ihd,nd->ihn", q.double(), k[:, 0]) * scale
    limit = torch.arange(n_q) + n - n_q + 1
    s = s.masked_fill(torch.arange(n) >= limit[:, None, None], -math.inf)
    lse = torch.logsumexp(s, -1).float()
    lse[1::7] = -math.inf
    lse[0, 1] = math.inf
    w = torch.zeros(1, 1, n, device="cuda")
    P.slh_attend_weights(q[None].cuda(), kc.cuda(), torch.arange(n // page, dtype=torch.int32).cuda()[None], torch.tensor([n], dtype=torch.int32).cuda(),
                         lse[None].cuda(), w, k_scale=None if ks is None else ks.cuda(), scale=scale)
    gives = torch.where(torch.isinf(lse), torch.tensor(-math.inf), lse)
    want, tol = CP.weights(q, k, gives, limit, scale)
    tol += n_q * Hq * 2.0 ** -126                  # terms below the smallest normal number may be zeros
    assert bool(((w[0].double().cpu() - want).abs() <= tol).all()), float(((w[0].double().cpu() - want).abs() - tol).max())
    assert float(want.max()) > 0


@pytest.fixture(scope="module")
def wide(tmp_path_factory):
    out = os.path.join(str(tmp_path_factory.mktemp("weights")), "libweightsstub.so")
    cmd = [BUILD.HIPCC, "--offload-host-only", "-x", "hip", "-std=c++17", "-O1", "-shared", "-fPIC", "-Wl,-Bsymbolic", "-w",
           "-I", os.path.join(BUILD.ROOT, "include"), "-I", BUILD.CSRC, os.path.join(BUILD.ROOT, "tests", "weights_stub.cpp"), "-o", out]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    f = ctypes.CDLL(out).stub_weights_wide
    f.argtypes = [ctypes.c_int64] + 5 * [ctypes.c_int]
    return f


def test_tiles_of_any_cu_are_counted_in_bits_that_hold_them(wide):
    """cu_q lies in device memory: entries that do not ascend may give every other sequence all queries."""
    for B, Tq, g, rows, in ((1 << 16, 16384, 8, 16384), (64, 1 << 20, 8, 131072), (2, 1 << 27, 8, 1 << 16), (1, 140000, 1, 8190 * 65536), (23, 12007, 4, 1472),
                            (3, 192, 5, 9216), (1 << 20, 1 << 20, 1, 256), (4096, 4096, 7, 65536), (1024, 65536, 8, 131072), (1023, 65536, 8, 131072)):
        key_blocks = -(-rows // 256)
        most = B * -(-Tq * g // 128) * key_blocks
        assert wide(Tq, B, g, rows, 0, 64) == (most + 64 >= 1 << 31), (B, Tq, g, rows)
        if Tq % B == 0:
            assert wide(Tq, B, g, rows, 1, 64) == (B * -(-Tq // B * g // 128) * key_blocks + 64 >= 1 << 31), (B, Tq, g, rows)


@gpu
@pytest.mark.parametrize("block", [0, 16])
def test_weights_of_entries_that_do_not_ascend(block):
    """Sequences that share their queries, or have none: each as by itself."""
    g = _gen(8)
    page, d, T, Hq = 32, 64, 300, 2
    bounds = [0, 300, 0, 150, 100, 300, -7, 400, 20]
    lens = [300, 40, 513, 77, 200, 9, 1024, 33]
    n, width = len(lens), 32
    x = torch.randn(n * width, 1, page, d, generator=g)
    kc, ks = CP.held(x, block) if block else (x.to(BF), None)
    kc, ks = kc.cuda(), None if ks is None else ks.cuda()
    table = torch.randperm(n * width, generator=g).int().view(n, width).cuda()
    q = torch.randn(T, Hq, d, generator=g).to(BF).cuda()
    lse = torch.full((T, Hq), 6.0, device="cuda")
    w = torch.zeros(n, 1, width * page, device="cuda")
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    P.slh_attend_weights(q, kc, table, ints(lens), lse, w, cu_q=ints(bounds), k_scale=ks)
    for b in range(n):
        lo, hi = (min(max(v, 0), T) for v in bounds[b:b + 2])
        one = torch.zeros(1, 1, width * page, device="cuda")
        if lo < hi:
            P.slh_attend_weights(q[lo:hi].contiguous(), kc, table[b:b + 1], ints(lens[b:b + 1]), lse[lo:hi].contiguous(), one, cu_q=ints([0, hi - lo]), k_scale=ks)
        # the same positive terms, in another order
        assert bool(((w[b] - one[0]).abs() <= 2 * T * Hq * 2.0 ** -24 * one[0]).all()), b


@gpu
@pytest.mark.parametrize("block", [0, 32])
@pytest.mark.parametrize("share", [0.02, 0.5])
def test_weights_of_packed_prompts_with_large_scores_here_and_there(block, share):
    """Runs of several tiles and blocks of keys, in which some queries' scores are large: 64 runs a head take about seven tiles each."""
    g = torch.Generator(device="cuda")
    g.manual_seed(block + int(100 * share))
    d, page, Hkv, Hq, new, lens = 64, 64, 8, 32, [1500, 700, 1100], [1500, 760, 2000]
    pages = [-(-n // page) for n in lens]
    x = torch.randn(sum(pages), Hkv, page, d, generator=g, device="cuda")
    x[..., 0] = 64
    if block:
        kc, ks = CP.held(x.cpu(), block)
        k, kc, ks = CP.values(kc, ks).cuda(), kc.cuda(), ks.cuda()
    else:
        kc, ks = x.to(BF), None
        k = kc.double()
    table = torch.zeros(3, max(pages), dtype=torch.int32)
    cu, at = [0], 0
    for b, n in enumerate(pages):
        table[b, :n] = torch.arange(at, at + n)
        at += n
        cu.append(cu[-1] + new[b])
    q = torch.randn(cu[-1], Hq, d, generator=g, device="cuda")
    far = torch.rand(cu[-1], Hq, generator=g, device="cuda") < share
    q[..., 0] = torch.where(far, 100.0, 0.0)                             # scores of 6400 beside those of 0
    q = q.to(BF)
    lse = torch.empty(cu[-1], Hq, device="cuda")
    wants = []
    for b, (n, m) in enumerate(zip(new, lens)):
        kk = k[table[b, :pages[b]].long().cuda()].transpose(1, 2).flatten(0, 1)[:m]
        hide = torch.arange(m, device="cuda")[None] >= torch.arange(n, device="cuda")[:, None] + m - n + 1
        want, tol = (torch.zeros(Hkv, m, dtype=torch.float64, device="cuda") for _ in range(2))
        for h in range(Hq):
            qq, kh = q[cu[b]:cu[b + 1], h].double(), kk[:, h // 4]
            s = (qq @ kh.t().contiguous()).masked_fill(hide, -math.inf)
            ll = torch.logsumexp(s, -1).float()
            lse[cu[b]:cu[b + 1], h] = ll
            ll = ll.double()[:, None]
            p = torch.exp(s - ll)
            s = s.masked_fill(hide, 0.0)
            # the error of a weight as in cache_plain.weights; terms below the smallest normal number may be zeros
            u = 2.0 ** -24
            e = 2 * d * u * (qq.abs() @ kh.abs().t().contiguous()) + 2 * u * (s.abs() + ll.abs()) + 4 * u * (s - ll).abs() + 4 * u
            want[h // 4] += p.sum(0)
            tol[h // 4] += (p * (e + n * 4 * u)).sum(0) + n * 2.0 ** -126
        wants.append((want, tol))
    w = torch.zeros(3, Hkv, max(pages) * page, device="cuda")
    P.slh_attend_weights(q, kc, table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), lse, w, cu_q=torch.tensor(cu, dtype=torch.int32).cuda(),
                         k_scale=ks, scale=1.0)
    for b, (want, tol) in enumerate(wants):
        got = w[b, :, :lens[b]].double()
        assert bool(((got - want).abs() <= tol).all()), (b, float(((got - want).abs() - tol).max()))
        assert not bool(w[b, :, lens[b]:].any())
