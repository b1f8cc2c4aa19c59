"""The operators of a smaller cache (slh_kv_append_e4m3, slh_attend_paged_e4m3, slh_attend_weights, slh_kv_evict) against
their definitions in 64 bits."""
import math

import pytest
import torch

import attention_plain as AP
import cache_plain as CP
import paper_2607_19368_amd as P

pytestmark = pytest.mark.gpu
BF, HF, FF = torch.bfloat16, torch.float16, torch.float32
SIZES = [64, 80, 96, 128]


def _gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def _table(used, total, g, spare=1):
    """Page table of sequences with `used` pages each, in any order among `total`; entries behind are out of range."""
    order = torch.randperm(total, generator=g).int()
    table = torch.full((len(used), max([*used, 0]) + spare), 2 ** 30, dtype=torch.int32)
    at = 0
    for b, n in enumerate(used):
        table[b, :n] = order[at:at + n]
        at += n
    return table, order[at:]


def _cache(total, H, page, d, block, g, spread=1.0):
    x = [torch.randn(total, H, page, d, generator=g) * spread for _ in range(2)]
    (kc, ks), (vc, vs) = (CP.held(t, block) for t in x)
    return kc, vc, ks, vs


def _rows(x, pages, n):
    """The first n rows of a sequence, [n, H, d], of x [pages, H, page, d]."""
    per = x.shape[2]
    return x[pages[:-(-n // per)].long()].transpose(1, 2).flatten(0, 1)[:n] if n else x[:0].transpose(1, 2).flatten(0, 1)


# ---------------------------------------------------------------- the card's conversions
def test_every_code_and_power():
    """Codes through attention: one key a sequence with weight 1 gives its value back, for every code and for powers of both ends."""
    d, block = 64, 16
    codes = torch.arange(256, dtype=torch.uint8).view(4, 64)
    for dt, powers in ((BF, (-100, -7, -1, 0, 3, 100)), (HF, (-5, 0, 7, 9))):       # 2^9: past fp16, infinite
        for x in powers:
            kc = torch.zeros(4, 1, 16, d, dtype=torch.uint8).view(CP.CODE).cuda()
            vc = torch.zeros(4, 1, 16, d, dtype=torch.uint8)
            vc[:, 0, 0] = codes
            vc = vc.view(CP.CODE)
            s = torch.full((4, 1, 1), 127 + x, dtype=torch.uint8).view(CP.SCALE)
            q = torch.ones(4, 1, d, dtype=dt).cuda()
            out = P.slh_attend_paged_e4m3(q, kc, vc.cuda(), s.cuda(), s.cuda(), torch.arange(4, dtype=torch.int32).cuda()[:, None],
                                          torch.ones(4, dtype=torch.int32).cuda())
            want = (codes.view(CP.CODE).double() * 2.0 ** x).to(dt)
            assert torch.equal(out[:, 0].cpu().nan_to_num(nan=0.5), want.nan_to_num(nan=0.5)), (dt, x)


@pytest.mark.parametrize("dt,x", [(HF, 8), (HF, 9), (HF, 14), (HF, 23), (HF, 24), (HF, 30), (BF, 120), (BF, 121), (BF, 127)])
@pytest.mark.parametrize("d", [64, 80, 96, 128])
@pytest.mark.parametrize("n_q", [1, 3, 40])
def test_values_past_the_type(dt, x, d, n_q):
    """Infinite values: those that a query sees make its outputs infinite, those behind them (and NaN there) nothing."""
    page, n = 32, 16 + n_q + 5
    kc = torch.zeros(2, 1, page, d, dtype=torch.uint8)
    vc = torch.zeros(2, 1, page, d, dtype=torch.uint8)
    rows = vc.view(2 * page, d)
    codes = torch.arange(256, dtype=torch.uint8)
    rows[n - n_q] = codes[(torch.arange(d) * 3 + 64) % 256]                     # seen by all; the columns' codes differ
    rows[n - 1] = codes[(torch.arange(d) * 7 + 5) % 256]                        # seen by the last query
    rows[n:] = codes[(torch.arange(d) * 5 + 1) % 256]                           # unwritten rows, some of them NaN
    two = torch.full((2, 1, page // 16), 127 + x, dtype=torch.uint8)
    held = [kc.view(CP.CODE).cuda(), vc.view(CP.CODE).cuda(), torch.full_like(two, 127).view(CP.SCALE).cuda(), two.view(CP.SCALE).cuda()]
    q = torch.ones(1, n_q, 1, d, dtype=dt).cuda()
    out = P.slh_attend_paged_e4m3(q, *held, torch.tensor([[0, 1]], dtype=torch.int32).cuda(), torch.tensor([n], dtype=torch.int32).cuda())[0, :, 0]
    v = (rows.view(CP.CODE).double() * 2.0 ** x).to(dt).double()                # keys are zeros: every row that is seen has the same weight
    for i in range(n_q):
        want = v[:n - n_q + 1 + i].mean(0)
        got, most = out[i].cpu().double(), v[:n - n_q + 1 + i].nan_to_num(0, 0, 0).abs().mean(0)
        odd = ~torch.isfinite(want)
        # the largest weight is 1 before the sums are divided, here every one: finite fp32 sums are those below 2^128, in any
        # order if those of the magnitudes are
        whole = most * (n - n_q + 1 + i) < 2.0 ** 128 * (1 - 2.0 ** -16)
        assert torch.equal(got[odd].nan_to_num(nan=0.5), want[odd].nan_to_num(nan=0.5)), i
        # weights to half a step, the sum of n terms in fp32, the output to half a step (subnormal fp16: 2^-25)
        tol = most[~odd] * (torch.finfo(dt).eps + (n + 8) * 2.0 ** -23) + 2.0 ** -25
        assert bool(((got[~odd] - want[~odd]).abs() <= tol)[whole[~odd]].all()), i


# ---------------------------------------------------------------- append
def _append_case(new, lens, H, d, dt, page, block, seed, norm=False, rot=0, inter=False, spread=1.0, even=False, x=None):
    """Runs slh_kv_append_e4m3 and checks every code and scale of the cache."""
    g = _gen(seed)
    B, T = len(new), sum(new)
    used = [-(-n // page) for n in lens]
    total = sum(used) + 2
    table, _ = _table(used, total, g)
    kc, vc, ks, vs = _cache(total, H, page, d, block, g)
    kv = (torch.randn(T, 2 * H + 1, d + 8, generator=g) * spread).to(dt) if x is None else x
    w = (1 + 0.3 * torch.randn(d, generator=g)).to(dt) if norm else None
    tab = P.slh_rope_table(3 * T + 1, rot) if rot else None
    pos = torch.randint(0, 3 * T + 1, (T,), generator=g).int() if rot else None
    cu = torch.tensor([0, *new]).cumsum(0).int()
    dev = [t.cuda() for t in (kc, vc, ks, vs)]
    kvd = kv.cuda()
    P.slh_kv_append_e4m3(kvd[:, :H, :d], kvd[:, H:2 * H, :d], *dev, table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda(),
                         None if even else cu.cuda(), None if w is None else w.cuda(), 1e-6, tab, None if pos is None else pos.cuda(), inter)
    got = [t.cpu() for t in dev]
    key, size = AP.norm_rope(kv[:, :H, :d], w, 1e-6, None if tab is None else tab.cpu(), pos, inter)
    # fp32 arithmetic of norm and rotation (as for slh_qk_norm_rope); without them the values are the inputs
    err = (d / 2 + 10) * 2.0 ** -24 * size if norm or rot else torch.zeros_like(key)
    for rows, e, was, two, out, out2 in ((key, err, kc, ks, got[0], got[2]),
                                         (kv[:, H:2 * H, :d].double(), torch.zeros_like(key), vc, vs, got[1], got[3])):
        bytes_, codes = CP.bytes_of(two).clone(), was.view(torch.uint8).clone()
        got_bytes, got_codes = CP.bytes_of(out2), out.view(torch.uint8)
        for b in range(B):
            begin = lens[b] - new[b]
            for lo in range(max(0, begin) // block * block, lens[b] if new[b] else 0, block):
                fresh = [r for r in range(max(lo, begin), min(lo + block, lens[b]))]
                page_, at = int(table[b, lo // page]), lo % page
                for h in range(H):
                    r = rows[[int(cu[b + 1]) - lens[b] + i for i in fresh], h]
                    re = e[[int(cu[b + 1]) - lens[b] + i for i in fresh], h]
                    fin = torch.isfinite(r)
                    top = float(r[fin].abs().max()) if bool(fin.any()) else 0.0
                    old = int(bytes_[page_, h, at // block]) - 127
                    # the power goes by the computed maximum, which may lie `re` to either side
                    near = float(re.max())
                    k = [min(max(CP.power(t), -126), CP.MOST[dt]) for t in (max(0.0, top - near), top, top + near)]
                    k = {max(x, old) for x in k} if lo < begin else set(k)
                    now = int(got_bytes[page_, h, at // block]) - 127
                    assert now in k, (b, lo, h, now, k)
                    bytes_[page_, h, at // block] = now + 127
                    if lo < begin:                      # earlier rows: rescaled codes
                        part = was[page_, h, at:at + begin - lo]
                        codes[page_, h, at:at + begin - lo] = (part.float() * 2.0 ** (old - now)).to(CP.CODE).view(torch.uint8)
                    c = out[page_, h, at + fresh[0] - lo:at + fresh[-1] + 1 - lo].double()
                    limit = 240.0 if now == CP.MOST[dt] else 448.0
                    y = r.clamp(-limit * 2.0 ** now, limit * 2.0 ** now)
                    assert torch.equal(torch.isnan(c), ~fin)
                    off = (c * 2.0 ** now - y).abs()[fin]
                    assert bool((off <= (CP.half_step(y, now) + re)[fin]).all()), (b, lo, h, float((off - (CP.half_step(y, now) + re)[fin]).max()))
                    if not (norm or rot):               # exact inputs: nearest even, as torch rounds
                        want = (y * 2.0 ** -now).float().to(CP.CODE)
                        assert torch.equal(c[fin], want.double()[fin])
                    codes[page_, h, at + fresh[0] - lo:at + fresh[-1] + 1 - lo] = got_codes[page_, h, at + fresh[0] - lo:at + fresh[-1] + 1 - lo]
        assert torch.equal(got_codes, codes) and torch.equal(got_bytes, bytes_)      # nothing else changed
    return got


@pytest.mark.parametrize("dt", [BF, HF, FF])
@pytest.mark.parametrize("d", SIZES)
@pytest.mark.parametrize("page,block", [(16, 16), (64, 32), (64, 64), (256, 256), (128, 128)])
def test_append_blocks(dt, d, page, block):
    new, lens = [1, 0, 17, 65, 3, 300], [1, 40, 17, 97, 130, 301]
    _append_case(new, lens, 2, d, dt, page, block, d + block)


@pytest.mark.parametrize("d,rot,inter,norm", [(128, 128, False, True), (128, 64, True, True), (80, 32, False, False), (96, 96, True, True),
                                              (64, 16, False, True), (64, 0, False, True)])
@pytest.mark.parametrize("dt", [BF, FF])
def test_append_normed_and_rotated(d, rot, inter, norm, dt):
    _append_case([5, 33, 1], [12, 33, 64], 3, d, dt, 32, 16, rot + d, norm=norm, rot=rot, inter=inter)


@pytest.mark.parametrize("spread", [1e-3, 0.2, 30.0, 6000.0])
@pytest.mark.parametrize("block", [16, 64])
def test_append_where_blocks_grow(spread, block):
    """One new row after another: much smaller and much larger than the earlier rows, which become subnormal or zero."""
    _append_case([1, 2, 1, 16], [17, 24, 64, 75], 1, 64, HF if spread < 5000 else BF, 64, block, 3, spread=spread)
    _append_case([1, 1, 1], [16, 33, 9], 5, 128, BF, 64, block, 4, spread=spread, even=True)


@pytest.mark.parametrize("dt", [BF, HF, FF])
def test_append_extremes(dt):
    """The type's largest and smallest values, zeros, infinities and NaN."""
    top = torch.finfo(dt).max
    x = torch.randn(40, 3, 72, generator=_gen(1)).to(dt)
    x[0:16, 0] = 0
    x[3, 1, 5], x[17, 0, 3], x[18, 0, 4] = top, -top, top / 2
    x[20, 1, 7], x[21, 1, 8], x[22, 0, 9] = math.inf, -math.inf, math.nan
    x[32:, 0] = torch.finfo(dt).tiny
    got = _append_case([40], [40], 1, 64, dt, 64, 16, 1, x=x)
    back = CP.values(got[0], got[2])
    assert bool((back[~torch.isnan(back)].abs() <= top).all())
    x[22, 0, :] = math.nan                                    # whole rows that are not finite
    x[16:32, 1, :] = math.inf
    _append_case([40], [40], 1, 64, dt, 64, 16, 2, x=x)


def test_append_tokens_that_have_no_row():
    """More tokens than rows, lengths past the table, pages outside the cache, sequences without tokens, batches of none."""
    g = _gen(5)
    k, v = (torch.randn(40, 2, 64, generator=g).to(BF).cuda() for _ in range(2))
    kc, vc, ks, vs = _cache(5, 2, 16, 64, 16, g)

    def call(table, lens, cu):
        dev = [t.cuda() for t in (kc, vc, ks, vs)]
        P.slh_kv_append_e4m3(k, v, *dev, torch.tensor(table, dtype=torch.int32).cuda(), torch.tensor(lens, dtype=torch.int32).cuda(),
                             torch.tensor(cu, dtype=torch.int32).cuda())
        return [t.cpu() for t in dev]

    same = lambda a, b: all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(a, b))
    # the last three of forty tokens
    got = call([[3]], [3], [0, 40])
    want = [t.clone() for t in (kc, vc, ks, vs)]
    for c, s, x in ((0, 2, k), (1, 3, v)):
        codes, two = CP.held(torch.cat([x[37:].cpu().float(), torch.zeros(13, 2, 64)]).transpose(0, 1)[None], 16)
        want[c][3, :, :3], want[s][3] = codes[0, :, :3], two[0]
    assert same(got, want)
    # lengths past the table are its size; a negative one is none
    assert same(call([[3, 1]], [1000], [0, 5]), call([[3, 1]], [32], [0, 5]))
    assert same(call([[3], [4]], [-7, 0], [0, 4, 40]), (kc, vc, ks, vs))
    # pages outside the cache: those rows are left out, the others not
    a, b = call([[3, 99]], [32], [0, 32]), call([[3, 1]], [32], [0, 32])
    assert torch.equal(a[0][3].view(torch.uint8), b[0][3].view(torch.uint8)) and torch.equal(a[2][3].view(torch.uint8), b[2][3].view(torch.uint8))
    a[0][3], a[1][3], a[2][3], a[3][3] = kc[3], vc[3], ks[3], vs[3]
    assert same(a, (kc, vc, ks, vs))
    assert same(call([[-1], [5]], [16, 16], [0, 16, 32]), (kc, vc, ks, vs))
    # cu outside [0, T]
    assert same(call([[3, 1, 0]], [48], [-5, 400]), call([[3, 1, 0]], [48], [0, 40]))
    assert same(call([[3]], [4], [7, 3]), (kc, vc, ks, vs))


def test_append_many_sequences():
    """More sequences than a wave counts at a time, some without tokens."""
    new = [(7 * b) % 4 for b in range(150)]
    lens = [n + (5 * b) % 23 for b, n in enumerate(new)]
    _append_case(new, lens, 1, 64, BF, 16, 16, 9)


# ---------------------------------------------------------------- attention
def _paged_case(B, n_q, Hq, Hkv, d, dt, page, block, prefix, lens, seed, spread=1.0, scale=None):
    """Rows past a length hold NaN codes."""
    g = _gen(seed)
    used = [-(-n // page) for n in lens]
    n_pre = -(-prefix // page)
    total = n_pre + sum(used) + 2
    table, left = _table(used, total, g)
    pre = left[:n_pre].clone()
    kc, vc, ks, vs = _cache(total, Hkv, page, d, block, g, spread)
    bad = torch.ones(total, page, dtype=torch.bool)
    for pages, n in [(pre, prefix)] + [(table[b], lens[b]) for b in range(B)]:
        for i in range(-(-n // page)):
            bad[int(pages[i]), :n - i * page] = False
    for c in (kc, vc):
        c.view(torch.uint8).transpose(1, 2)[bad] = 0xff
    for s in (ks, vs):                              # and blocks without rows any power
        whole = bad.view(total, page // block, block).all(-1)
        s.view(torch.uint8).transpose(1, 2)[whole] = 255
    q = torch.randn(B, n_q, Hq, d, generator=g).to(dt)
    lse = torch.full((B, n_q, Hq), 7.0).cuda()
    scale = 1 / math.sqrt(d) if scale is None else scale
    out = P.slh_attend_paged_e4m3(q.cuda(), kc.cuda(), vc.cuda(), ks.cuda(), vs.cuda(), table.cuda(),
                                  torch.tensor(lens, dtype=torch.int32).cuda(), pre.cuda(), prefix, scale=scale, lse_out=lse)
    k, v = CP.values(kc, ks), CP.values(vc, vs)
    for b in range(B):
        kk, vv = (torch.cat([_rows(x, pre, prefix), _rows(x, table[b], lens[b])]) for x in (k, v))
        limit = [prefix + max(0, lens[b] - n_q + i + 1) for i in range(n_q)]
        o, tol, e, etol = AP.attend(q[b], kk, vv, limit, scale)
        got = out[b].double().cpu()
        assert bool(torch.isfinite(got).all()), b
        assert bool(((got - o).abs() <= tol).all()), (b, float(((got - o).abs() - tol).max()))
        got, empty = lse[b].double().cpu(), e == -math.inf
        assert torch.equal(got[empty], e[empty]) and bool(((got - e).abs() <= etol)[~empty].all()), b


@pytest.mark.parametrize("dt", [BF, HF])
@pytest.mark.parametrize("d", SIZES)
@pytest.mark.parametrize("n_q", [1, 3])
def test_paged_types_and_heads(dt, d, n_q):
    _paged_case(3, n_q, 14, 2, d, dt, 16, 16, 37, [n_q, 50, 129], d + n_q)


@pytest.mark.parametrize("page,block", [(16, 16), (32, 16), (32, 32), (64, 64), (256, 32), (256, 256)])
@pytest.mark.parametrize("prefix", [0, 1, 64, 300])
def test_paged_pages_and_prefixes(page, block, prefix):
    _paged_case(4, 2, 4, 1, 64, BF, page, block, prefix, [2, 31, 64, 65], page + prefix)


@pytest.mark.parametrize("prefix", [0, 40])
def test_paged_rows_without_own_keys(prefix):
    _paged_case(4, 3, 4, 2, 128, BF, 16, 16, prefix, [0, 1, 2, 3], prefix)


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (7, 1), (28, 4), (40, 8), (6, 6), (33, 1)])
def test_paged_head_groups(Hq, Hkv):
    _paged_case(2, 1, Hq, Hkv, 128, BF, 16, 16, 20, [19, 90], Hq)


@pytest.mark.parametrize("B,n_q,Hq,Hkv,prefix,lens", [
    (1, 1, 4, 2, 0, [3001]), (1, 2, 28, 4, 2001, [3]), (2, 5, 8, 1, 500, [900, 40]), (40, 1, 8, 1, 600, None), (70, 2, 4, 2, 0, None),
    (3, 9, 16, 2, 700, [9, 30, 300])])
def test_paged_batches_and_splits(B, n_q, Hq, Hkv, prefix, lens):
    lens = [n_q + (7 * b) % 90 for b in range(B)] if lens is None else lens
    _paged_case(B, n_q, Hq, Hkv, 64, BF, 64, 16, prefix, lens, B + n_q)


@pytest.mark.parametrize("dt", [BF, HF])
def test_paged_large_scores_and_scale(dt):
    _paged_case(2, 2, 4, 2, 64, dt, 16, 16, 33, [40, 90], 7, scale=8.0)
    _paged_case(2, 2, 4, 2, 64, BF, 16, 16, 33, [40, 90], 8, spread=2.0 ** 40, scale=2.0 ** -40)


@pytest.mark.parametrize("dt", [BF, HF])
@pytest.mark.parametrize("d", SIZES)
def test_paged_values_that_a_row_does_not_see(dt, d):
    """A NaN code of a later token leaves the rows before it alone, and reaches the element of those that see it."""
    g = _gen(3)
    n_q, n, page = 40, 75, 32
    table = torch.arange(3, dtype=torch.int32)[None]
    kc, vc, ks, vs = _cache(3, 2, page, d, 16, g)
    q = torch.randn(1, n_q, 4, d, generator=g).to(dt).cuda()
    lens = torch.tensor([n], dtype=torch.int32).cuda()

    def call(k, v):
        return P.slh_attend_paged_e4m3(q, k.cuda(), v.cuda(), ks.cuda(), vs.cuda(), table.cuda(), lens)[0].cpu()

    clean = call(kc, vc)
    for at, e in ((50, 5), (63, d - 1), (64, 17), (74, 0), (36, 62)):
        sees = torch.arange(n_q) + n - n_q >= at
        v2 = vc.clone()
        v2.view(torch.uint8)[at // page, 1, at % page, e] = 0x7f
        got = call(kc, v2)
        want = clean.clone()
        want[sees, 2:, e] = math.nan
        assert torch.equal(got.nan_to_num(nan=99.0), want.nan_to_num(nan=99.0)), (at, e)
        k2 = kc.clone()
        k2.view(torch.uint8)[at // page, 1, at % page, e] = 0xff
        got = call(k2, vc)
        want = clean.clone()
        want[sees, 2:] = math.nan
        assert torch.equal(got.nan_to_num(nan=99.0), want.nan_to_num(nan=99.0)), (at, e)


# ---------------------------------------------------------------- weights
def _weights_case(new, lens, Hq, Hkv, d, dt, page, block, seed, even=False, scale=None, bad_lse=False, elsewhere=False):
    """Queries that are parts of wider rows; rows past a length hold NaN."""
    g = _gen(seed)
    B, T = len(new), sum(new)
    used = [-(-n // page) for n in lens]
    total = sum(used) + 1
    table, _ = _table(used, total, g)
    bad = torch.ones(total, page, dtype=torch.bool)
    for b, n in enumerate(lens):
        for i in range(used[b]):
            bad[int(table[b, i]), :n - i * page] = False
    x = torch.randn(total, Hkv, page, d, generator=g)
    if block:
        kc, ks = CP.held(x, block)
        k = CP.values(kc, ks)
        kc.view(torch.uint8).transpose(1, 2)[bad] = 0x7f
    else:
        kc, ks = x.to(dt), None
        k = kc.double()
        kc.transpose(1, 2)[bad] = math.nan
    qw = torch.randn(T, Hq + 1, d + 8, generator=g).to(dt)
    q = qw[:, 1:, :d]
    cu = torch.tensor([0, *new]).cumsum(0).int()
    scale = 1 / math.sqrt(d) if scale is None else scale
    lse = torch.full((T, Hq), -math.inf)
    for b in range(B):
        rows = slice(int(cu[b]), int(cu[b + 1]))
        limit = [lens[b] - new[b] + i + 1 for i in range(new[b])]
        for i, lim in enumerate(limit):
            for h in range(Hq):
                if lim > 0:
                    s = _rows(k, table[b], lens[b])[:lim, h // (Hq // Hkv)] @ q[rows][i, h].double() * scale
                    lse[rows.start + i, h] = torch.logsumexp(s, 0) + 0.3          # as behind a prefix
    if elsewhere:                                  # rows that see none of these keys have others
        lse[lse == -math.inf] = 0.3
    if bad_lse:
        lse[::3] = -math.inf
    w = torch.rand(B, Hkv, table.shape[1] * page, generator=g)
    qd = qw.cuda()[:, 1:, :d]
    if even:
        qd = qd.unflatten(0, (B, -1))
    got = w.cuda()
    P.slh_attend_weights(qd, kc.cuda(), table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda(),
                         (lse.view(B, -1, Hq) if even else lse).cuda(), got, cu_q=None if even else cu.cuda(),
                         k_scale=None if ks is None else ks.cuda(), scale=scale)
    got = got.double().cpu()
    for b in range(B):
        rows = slice(int(cu[b]), int(cu[b + 1]))
        limit = [lens[b] - new[b] + i + 1 for i in range(new[b])]
        add, tol = CP.weights(q[rows], _rows(k, table[b], lens[b]), lse[rows], limit, scale)
        want = w[b].double().clone()
        assert torch.equal(got[b, :, lens[b]:], want[:, lens[b]:])
        want[:, :lens[b]] += add
        off = (got[b, :, :lens[b]] - want[:, :lens[b]]).abs() - tol - 2.0 ** -24 * want[:, :lens[b]].abs()
        assert not off.numel() or float(off.max()) <= 0, (b, float(off.max()))


@pytest.mark.parametrize("dt", [BF, HF])
@pytest.mark.parametrize("d", SIZES)
@pytest.mark.parametrize("block", [0, 16, 32])
def test_weights_types_and_heads(dt, d, block):
    _weights_case([1, 0, 5, 2, 40], [1, 9, 5, 130, 70], 6, 2, d, dt, 32, block, d + block)


@pytest.mark.parametrize("page", [1, 4, 16, 128])
def test_weights_pages(page):
    _weights_case([1, 1, 1], [17, 1, 150], 7, 1, 64, BF, page, 0, page, even=True)


@pytest.mark.parametrize("new,lens,Hq,Hkv", [
    ([1], [1], 1, 1), ([3], [2], 4, 2), ([2, 5], [0, 3], 4, 2), ([33], [33], 5, 1), ([64], [200], 8, 1), ([17, 90], [17, 90], 2, 2),
    ([1] * 70, [1 + (11 * b) % 60 for b in range(70)], 3, 1), ([129], [257], 7, 1)])
def test_weights_lengths(new, lens, Hq, Hkv):
    """Queries of one token and of many, in front of which rows lie or not, some that see nothing."""
    _weights_case(new, lens, Hq, Hkv, 64, BF, 16, 0, len(new) + Hq)
    _weights_case(new, lens, Hq, Hkv, 64, HF, 16, 16, len(new) + Hq)


@pytest.mark.parametrize("new,lens,Hq", [([60], [30], 1), ([64], [1], 1), ([100], [3], 1), ([20], [11], 5), ([300, 200], [100, 0], 3), ([129], [128], 1), ([500], [257], 2)])
@pytest.mark.parametrize("block", [0, 16])
def test_weights_of_more_queries_than_rows(new, lens, Hq, block):
    """The first queries see nothing; tiles that hold such rows beside others."""
    for elsewhere in (False, True):
        _weights_case(new, lens, Hq, 1, 64, BF, 16, block, new[0] + Hq, elsewhere=elsewhere)


@pytest.mark.parametrize("byte", [253, 254])
def test_append_beside_rows_of_the_largest_powers(byte):
    """A block whose earlier row has a power that append itself does not give: it stays, and the codes are its."""
    kc, vc = (torch.zeros(1, 1, 16, 64, dtype=torch.uint8).view(CP.CODE).cuda() for _ in range(2))
    ks, vs = (torch.full((1, 1, 1), byte, dtype=torch.uint8).view(CP.SCALE).cuda() for _ in range(2))
    kc.view(torch.uint8)[0, 0, 0] = 0x38                                        # 1
    x = (torch.linspace(-1, 1, 64) * 3e38).to(BF)[None, None]
    P.slh_kv_append_e4m3(x.cuda(), x.cuda(), kc, vc, ks, vs, torch.zeros(1, 1, dtype=torch.int32).cuda(), torch.tensor([2], dtype=torch.int32).cuda())
    want = (x.double() * 2.0 ** (127 - byte)).float().to(CP.CODE)[0, 0]         # exact in fp32: at most 4, at least 2^-133 of 8 bits
    for cache, two in ((kc, ks), (vc, vs)):
        assert CP.bytes_of(two).item() == byte
        assert torch.equal(cache[0, 0, 1].cpu().view(torch.uint8), want.view(torch.uint8))
    assert bool((kc.view(torch.uint8)[0, 0, 0] == 0x38).all()) and not bool(kc.view(torch.uint8)[0, 0, 2:].any())


@pytest.mark.parametrize("n_q,Hq,Hkv", [(12, 8, 1), (13, 8, 1), (33, 2, 2), (96, 1, 1), (97, 1, 1)])
@pytest.mark.parametrize("block", [0, 16])
def test_weights_of_even_batches(n_q, Hq, Hkv, block):
    """Rows of a sequence about 96, where the kernel changes."""
    _weights_case([n_q] * 3, [n_q, n_q + 200, 5 * n_q + 1], Hq, Hkv, 64, BF, 16, block, n_q, even=True)


def test_weights_of_queries_that_attend_to_nothing():
    _weights_case([9, 4], [20, 4], 4, 2, 64, BF, 16, 0, 1, bad_lse=True)


def test_weights_add_up_to_the_queries():
    """With the lse of slh_attend_paged_e4m3, a prefix's share apart, the weights of a query sum to one."""
    g = _gen(2)
    B, n_q, Hq, Hkv, d = 5, 3, 8, 2, 128
    lens = [3, 40, 77, 128, 19]
    table, _ = _table([4] * B, 4 * B + 1, g, 0)
    kc, vc, ks, vs = (t.cuda() for t in _cache(4 * B + 1, Hkv, 32, d, 32, g))
    q = torch.randn(B, n_q, Hq, d, generator=g).to(BF).cuda()
    ln, lse = torch.tensor(lens, dtype=torch.int32).cuda(), torch.empty(B, n_q, Hq).cuda()
    P.slh_attend_paged_e4m3(q, kc, vc, ks, vs, table.cuda(), ln, lse_out=lse)
    w = torch.zeros(B, Hkv, 128).cuda()
    P.slh_attend_weights(q, kc, table.cuda(), ln, lse, w, k_scale=ks)
    assert bool(((w.double().sum(-1) - n_q * Hq / Hkv).abs() < 1e-4).all())


# ---------------------------------------------------------------- eviction
def _evict_case(lens, budget, first, last, H, d, dt, page, block, seed, w=None, place=False):
    g = _gen(seed)
    B = len(lens)
    used = [-(-n // page) for n in lens]
    total = sum(used) + 2
    table, _ = _table(used, total, g)
    if block:
        kc, vc, ks, vs = _cache(total, H, page, d, block, g)
        for t in (kc, vc):                         # outlying rows, so that powers differ and codes become subnormal
            t.view(torch.uint8)[:, :, ::5] = 0x01
        ks.view(torch.uint8).add_(torch.randint(-12, 12, ks.shape, generator=g).to(torch.uint8))
    else:
        kc, vc = (torch.randn(total, H, page, d, generator=g).to(dt) for _ in range(2))
        ks = vs = None
    rows = table.shape[1] * page
    if w is None:
        w = torch.randint(0, 40, (B, H, rows), generator=g).float() / 8          # many ties
    dev = [None if t is None else t.cuda() for t in (kc, vc, ks, vs)]
    wd, ld = w.cuda(), torch.tensor(lens, dtype=torch.int32).cuda()
    wo, lo, kept = P.slh_kv_evict(dev[0], dev[1], wd, table.cuda(), ld, budget, first, last, dev[2], dev[3],
                                  weights_out=wd if place else None, lens_out=ld if place else None)
    if place:
        assert wo is wd and lo is ld
    else:
        assert torch.equal(wd.cpu().nan_to_num(nan=5.5), w.nan_to_num(nan=5.5)) and ld.tolist() == lens
    assert lo.tolist() == [min(n, budget) for n in lens]
    wo, kept = wo.cpu(), kept.cpu()
    want = [None if t is None else t.clone() for t in (kc, vc, ks, vs)]
    for b, n in enumerate(lens):
        for h in range(H):
            stay = CP.keep(w[b, h].tolist(), n, budget, first, last)
            assert kept[b, h].tolist() == stay + [-1] * (budget - len(stay)), (b, h)
            assert torch.equal(wo[b, h, :len(stay)].nan_to_num(nan=5.5), w[b, h, stay].nan_to_num(nan=5.5))
            assert not bool(wo[b, h, len(stay):].any())
            if n <= budget:
                continue
            for x in range(2):
                old, new = (kc, vc)[x], want[x]
                if not block:
                    for i, j in enumerate(stay):
                        new[int(table[b, i // page]), h, i % page] = old[int(table[b, j // page]), h, j % page]
                    continue
                two = CP.bytes_of((ks, vs)[x])
                val = CP.values(old, (ks, vs)[x])
                for i0 in range(0, budget, block):
                    part = [val[int(table[b, j // page]), h, j % page] for j in stay[i0:i0 + block]]
                    y = torch.stack(part)
                    k = max(CP.power(float(y.abs().max())), -126)
                    p, at = int(table[b, i0 // page]), i0 % page
                    want[2 + x].view(torch.uint8)[p, h, at // block] = k + 127
                    new[p, h, at:at + len(part)] = (y * 2.0 ** -k).float().to(CP.CODE)
                del two
    for t, u in zip(dev, want):
        if t is not None:
            view = torch.uint8 if block else {BF: torch.int16, HF: torch.int16, FF: torch.int32}[dt]
            assert torch.equal(t.cpu().view(view), u.view(view))


@pytest.mark.parametrize("dt,d", [(BF, 128), (HF, 80), (FF, 64), (BF, 8), (FF, 256), (BF, 96)])
@pytest.mark.parametrize("place", [False, True])
def test_evict_types(dt, d, place):
    _evict_case([100, 33, 7, 0, 64], 33, 2, 5, 2, d, dt, 16, 0, d, place=place)


@pytest.mark.parametrize("page,block", [(16, 16), (64, 32), (256, 256), (128, 64)])
@pytest.mark.parametrize("d", SIZES)
def test_evict_blocks(page, block, d):
    _evict_case([100, 41, 7, 0, 300], 41, 2, 5, 2, d, BF, page, block, d + page, place=bool(d & 16))


@pytest.mark.parametrize("budget,first,last", [(1, 0, 0), (1, 1, 0), (1, 0, 1), (20, 20, 0), (20, 0, 20), (20, 7, 13), (599, 0, 1), (600, 4, 4), (3000, 0, 0)])
def test_evict_budgets(budget, first, last):
    _evict_case([600, 20, 19, 21, 1], budget, first, last, 1, 64, BF, 64, 0, budget)
    _evict_case([600, 20, 19, 21, 1], budget, first, last, 1, 64, BF, 64, 16, budget)


@pytest.mark.parametrize("n,budget", [(33000, 1500), (60011, 32900), (8193, 8192)])
def test_evict_long_in_place(n, budget):
    """More rows than are held at once, their weights moved in place."""
    _evict_case([n, 17, budget + 1], budget, 3, 11, 1, 64, BF, 64, 0, n, place=True)


@pytest.mark.parametrize("block", [0, 64])
@pytest.mark.parametrize("n,budget", [(1024, 1023), (1025, 512), (3000, 700), (5003, 1), (25000, 3001), (24576, 24575), (60011, 1300)])
def test_evict_long(n, budget, block):
    """Chunks of the pass over the weights and of the move, and their ends."""
    _evict_case([n, 17], budget, 0, 0, 2, 64, BF, 64, block, n)


def _few(n, seed):
    """Weights of a sequence of n rows: few of them equal (spread), all of one upper part, NaN, all zeros."""
    g = _gen(seed)
    w = torch.stack([torch.randn(n, generator=g), 1 + torch.rand(n, generator=g) * 2.0 ** -6,
                     torch.where(torch.rand(n, generator=g) < 0.3, float("nan"), 2.0), torch.zeros(n)])
    return w[:, None].contiguous()


@pytest.mark.parametrize("n,budget,first,last", [(16385, 16384, 0, 0), (16448, 2000, 4, 700), (20000, 37, 20, 17), (40000, 33000, 0, 9), (49157, 12301, 4, 256),
                                                 (140003, 900, 10, 50), (140003, 60000, 50000, 3)])
@pytest.mark.parametrize("place", [False, True])
def test_evict_by_runs(n, budget, first, last, place):
    """Few long sequences: several blocks pick of each; runs that end inside one another's waves, rows kept at both ends."""
    page = 64
    w = torch.zeros(4, 1, (-(-n // page) + 1) * page)
    w[:, :, :n] = _few(n, n)
    _evict_case([n, n - 1, budget + 1, budget], budget, first, last, 1, 8, BF, page, 0, n, w=w, place=place)


@pytest.mark.parametrize("n", [16390, 33000])
def test_evict_many_long_tables(n):
    """More sequences than compute units: a block each, which holds 32768 rows of weights or fewer than the sequence has."""
    _evict_case([n, n - 77] + [31, 1, 0] * 90, 30, 1, 3, 1, 8, BF, 64, 0, n, place=True)


@pytest.mark.parametrize("n", [17000, 70000])
def test_evict_runs_of_a_long_run(n):
    """Two blocks a sequence, with rows behind those that they hold."""
    _evict_case([n, 2 * n + 1000] + [600, 40] * 58, 500, 1, 3, 1, 8, BF, 64, 0, n)


def test_evict_weights_of_all_kinds():
    """Infinities, NaN of both signs, zeros of both signs, negative ones, the smallest and largest numbers."""
    kinds = torch.tensor([math.inf, -math.inf, math.nan, -math.nan, 0.0, -0.0, -1.0, 1.0, 1e-45, -1e-45, 3.4e38, -3.4e38, 1.0000001])
    for seed in range(6):
        w = kinds[torch.randint(0, len(kinds), (2, 3, 192), generator=_gen(seed))]
        _evict_case([90, 128], [1, 20, 45, 60, 80, 89][seed], 0, 0, 3, 64, BF, 64, 0, seed, w=w, place=seed % 2 == 1)
    for x in (0.0, math.nan, math.inf, 2.5):                 # all equal: the first rows
        _evict_case([90, 128], 50, 1, 3, 2, 64, BF, 64, 16, 3, w=torch.full((2, 2, 192), x))
