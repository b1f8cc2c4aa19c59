"""Each way in which slh_attend_paged_e4m3 goes about a call: blocks of 16, 32 and 128 rows, keys split or not, a prefix in front
of each sequence's own keys, in parts of its own, in one launch with them or in another.  The shapes say which (checked
without a GPU, for all head sizes, against the plans of a card of 256 compute units); values are compared with the
definition in 64 bits (the tolerances of attention_plain.py)."""
import math

import pytest
import torch

import attention_plain as AP
import cache_plain as CP
import cache_plan
import paper_2607_19368_amd as P
from test_attention_paths import close, close_lse, rows_of

gpu = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16
SIZES = [64, 80, 96, 128]

# (sequences, new tokens, query heads, key/value heads, page size, pages a sequence, prefix): the launches (kernel, rows of
# a block), whether partial results are joined, whether the prefix is read in front of each sequence's own keys
PATHS = {
    (1, 1, 4, 4, 16, 1, 0): ([("rows", 16)], False, False),
    (1, 1, 4, 4, 16, 1, 77): ([("rows", 16)], False, True),
    (1, 1, 4, 4, 64, 50, 0): ([("rows", 16)], True, False),
    (64, 3, 28, 4, 16, 1, 0): ([("rows", 32)], False, False),
    (64, 3, 28, 4, 16, 1, 77): ([("rows", 32)], False, True),
    (1, 16, 40, 8, 64, 50, 0): ([("rows", 32)], True, False),
    (64, 5, 28, 4, 16, 1, 0): ([("tiles", 128)], False, False),
    (1, 24, 40, 8, 64, 512, 77): ([("tiles", 128)], True, False),
    (8, 5, 40, 8, 16, 24, 5000): ([("both", 16)], True, False),
    (8, 40, 28, 4, 16, 24, 5000): ([("both", 32)], True, False),
    (2, 16, 28, 4, 64, 512, 2001): ([("rows", 16), ("tiles", 128)], True, False),
    (1, 24, 40, 8, 64, 512, 5000): ([("rows", 32), ("tiles", 128)], True, False),
}


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    return cache_plan.build(tmp_path_factory.mktemp("cache"))


@pytest.mark.parametrize("shape", PATHS)
def test_shapes_take_their_paths(plans, shape):
    for d in SIZES:
        done = plans.paged(*shape[:4], d, *shape[4:])
        kernels = [x for x in done if x[0] != "join"]
        assert ([x[:2] for x in kernels], len(done) > len(kernels), bool(kernels[0][6])) == PATHS[shape], d


def test_a_long_prefix_is_read_once_whatever_the_tables_width(plans):
    for Hq, Hkv in ((28, 4), (32, 8)):
        for n in (64, 128):
            for width in (704, 4096, 32768):
                first = plans.paged(n, 1, Hq, Hkv, 128, 64, width // 64, 32768)[0]
                assert first[6] == 0 and first[4] > 0, (Hq, n, width)


def _held(x, block):
    """Codes and scales of x [pages, H, page, d] on the card."""
    p, H, ps, d = x.shape
    y = x.reshape(p, H, ps // block, block * d)
    k = torch.ceil(torch.log2(y.abs().amax(-1) / 448)).clamp(min=-126)
    return ((y * torch.exp2(-k)[..., None]).clamp(-448, 448).to(CP.CODE).view(p, H, ps, d), (k + 127).to(torch.uint8).view(CP.SCALE))


def _own(x, pages, n):
    ps = x.shape[2]
    return x[pages[:-(-n // ps)].long()].transpose(1, 2).flatten(0, 1)[:n]


def _call(shape, d, dt, block, seed, lens=None):
    n, n_q, Hq, Hkv, page, width, prefix = shape
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    n_pre = -(-prefix // page)
    total = n_pre + n * width
    order = torch.randperm(total, generator=g, device="cuda").int()
    (kc, ks), (vc, vs) = (_held(torch.randn(total, Hkv, page, d, generator=g, device="cuda"), block) for _ in range(2))
    table = order[n_pre:].view(n, width)
    if lens is None:
        lens = torch.randint(0, width * page + 1, (n,), generator=g, device="cuda").int()
        lens[0] = width * page
        if n > 2:
            lens[1], lens[2] = 0, max(1, n_q - 1)
    q = torch.randn(n, n_q, Hq, d, generator=g, device="cuda").to(dt)
    return q, kc, vc, ks, vs, table, lens, order[:n_pre].clone(), prefix


@gpu
@pytest.mark.parametrize("dt", [BF, HF])
@pytest.mark.parametrize("shape", PATHS)
def test_paged(shape, dt):
    for d, big in zip(SIZES if shape[0] * shape[1] * shape[2] < 3000 else [64, 128], (False, True, False, True)):
        args = _call(shape, d, dt, min(shape[4], 64) if big else 16, d)
        q, kc, vc, ks, vs, table, lens, pre, prefix = args
        n, n_q, Hq = q.shape[:3]
        lse = torch.empty(n, n_q, Hq, device="cuda")
        out = P.slh_attend_paged_e4m3(*args, lse_out=lse)
        k, v = ((x.double().unflatten(2, (s.shape[2], -1)) * s.double()[..., None, None]).flatten(2, 3) for x, s in ((kc, ks), (vc, vs)))
        kp, vp = (_own(x, pre, prefix) for x in (k, v))
        for b in sorted({0, 1, 2, n // 2, n - 1} & set(range(n))):
            m = int(lens[b])
            kk, vv = (torch.cat([f, _own(x, table[b], m)]) for f, x in ((kp, k), (vp, v)))
            limit = [prefix + max(0, m - n_q + i + 1) for i in range(n_q)]
            o, tol, e, etol = rows_of(q[b], kk, vv, limit, 1 / math.sqrt(d))
            close(out[b], o, tol, f"{d}, sequence {b}")
            close_lse(lse[b], e, etol, f"{d}, sequence {b}")
        assert all(torch.equal(P.slh_attend_paged_e4m3(*args), out) for _ in range(3))


@gpu
@pytest.mark.parametrize("shape", [s for s in PATHS if s[1] > 2])
def test_codes_that_a_row_does_not_see(shape):
    """NaN codes of a sequence's last row reach its last token alone."""
    d, (n, n_q, Hq, Hkv, page, width, prefix) = 128, shape
    lens = torch.full((n,), width * page - 3, dtype=torch.int32, device="cuda")
    q, kc, vc, ks, vs, table, lens, pre, prefix = _call(shape, d, BF, 16, 1, lens)
    clean = P.slh_attend_paged_e4m3(q, kc, vc, ks, vs, table, lens, pre, prefix)
    m = int(lens[0]) - 1
    page_ = table[:, m // page].long()
    for cache in (kc, vc):
        was = cache.view(torch.uint8)[page_, :, m % page].clone()
        cache.view(torch.uint8)[page_, :, m % page, 3:7] = 0x7f
        got = P.slh_attend_paged_e4m3(q, kc, vc, ks, vs, table, lens, pre, prefix)
        assert torch.equal(got[:, :-1], clean[:, :-1])
        bad = torch.isnan(got[:, -1])
        assert bool(bad[..., 3:7].all()) and bool(bad.all() if cache is kc else not bad[..., 7:].any())
        cache.view(torch.uint8)[page_, :, m % page] = was
