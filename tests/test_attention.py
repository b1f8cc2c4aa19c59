"""The operators behind a compressed prompt against their definitions in 64 bits
(attention_plain.py, where the tolerances are derived), at the sizes, masks, strides and
values where they can go wrong."""
import math

import pytest
import torch

import attention_plain as AP
import paper_2607_19368_amd as P
from paper_2607_19368_amd import slh as B

gpu = pytest.mark.gpu
BF, HF, F32 = torch.bfloat16, torch.float16, torch.float32


def _gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def _close(got, want, tol, what=""):
    got = got.double().cpu()
    assert got.shape == want.shape
    if not got.numel():
        return
    assert bool(torch.isfinite(got).all()), f"{what}: not finite"
    over = ((got - want).abs() - tol).max()
    assert float(over) <= 0.0, f"{what}: {float(over):.3g} past the tolerance"


# ---------------------------------------------------------------- rotation table
def _freqs(rot, base, scaling, factor, orig, fast, slow):
    out = []
    for i in range(rot // 2):
        b = base * factor ** (rot / (rot - 2)) if scaling == B.SLH_ROPE_BASE else base
        f = b ** (-2 * i / rot)
        if scaling == B.SLH_ROPE_LINEAR:
            f /= factor
        if scaling == B.SLH_ROPE_BANDS:
            turns = orig * f / (2 * math.pi)
            mix = min(1.0, max(0.0, (turns - slow) / (fast - slow)))
            f = f / factor * (1 - mix) + f * mix
        out.append(f)
    return out


@gpu
@pytest.mark.parametrize("rot,n_pos,scaling,factor", [
    (128, 1000, B.SLH_ROPE_PLAIN, 1.0), (64, 517, B.SLH_ROPE_LINEAR, 4.0), (16, 1, B.SLH_ROPE_BASE, 8.0),
    (80, 4099, B.SLH_ROPE_BANDS, 8.0), (256, 70001, B.SLH_ROPE_BANDS, 4.0)])
def test_rope_table(rot, n_pos, scaling, factor):
    got = P.slh_rope_table(n_pos, rot, 10000.0, scaling, factor, 2048, 32.0, 1.0).cpu().double()
    f = torch.tensor(_freqs(rot, 10000.0, scaling, factor, 2048, 32.0, 1.0), dtype=torch.float64)
    a = torch.arange(n_pos, dtype=torch.float64)[:, None] * f
    s = 0.1 * math.log(factor) + 1 if scaling == B.SLH_ROPE_BANDS else 1.0
    want = torch.stack([s * a.cos(), s * a.sin()], 1)
    # the rounding to 32 bits, and the frequency's last bit times the position
    assert float((got - want).abs().max()) <= s * (2.0 ** -24 + n_pos * 2.0 ** -51)


# ---------------------------------------------------------------- norms and rotation
@gpu
@pytest.mark.parametrize("dt", [BF, HF, F32])
@pytest.mark.parametrize("T,Hq,Hk,d,rot,inter,norm", [
    (1, 1, 1, 64, 64, False, True), (37, 7, 1, 128, 128, False, True), (61, 4, 4, 80, 32, True, False),
    (5, 12, 3, 96, 96, True, True), (33, 3, 5, 72, 48, False, True), (130, 2, 2, 256, 256, False, True),
    (9, 5, 0, 8, 0, False, True), (17, 0, 3, 24, 16, True, False), (11, 2, 1, 128, 0, False, True)])
def test_qk_norm_rope(T, Hq, Hk, d, rot, inter, norm, dt):
    g = _gen(T + d)
    qkv = (torch.randn(T, Hq + 2 * Hk + 1, d, generator=g) * 2).to(dt)
    w = [(1 + torch.randn(d, generator=g) * 0.3).to(dt) if norm else None for _ in range(2)]
    table = P.slh_rope_table(4 * T + 3, rot) if rot else None
    pos = torch.randint(0, 4 * T + 3, (T,), generator=g).int() if rot else None
    dev = qkv.cuda()
    q, k = dev[:, :Hq] if Hq else None, dev[:, Hq:Hq + Hk] if Hk else None
    wd = [None if x is None else x.cuda() for x in w]
    out = P.slh_qk_norm_rope(q, k, wd[0] if Hq else None, wd[1] if Hk else None, 1e-5, table,
                             None if pos is None else pos.cuda(), inter)
    u = AP.U[dt]
    for got, x, wt in ((out[0], qkv[:, :Hq], w[0]), (out[1], qkv[:, Hq:Hq + Hk], w[1])):
        if got is None:
            continue
        want, size = AP.norm_rope(x, wt, 1e-5, None if table is None else table.cpu(), pos, inter)
        # one rounding to the type (fp16: or half its smallest step), and in 32 bits the sum of d
        # squares (half of its error after the root), the root, division and five products
        tol = u * want.abs() + (d / 2 + 10) * 2.0 ** -24 * size + (2.0 ** -25 if dt == HF else 0.0)
        _close(got, want, 1.01 * tol)
    # in place on the projection's own rows: the same bits, and the values beside them untouched
    here = dev.clone()
    P.slh_qk_norm_rope(here[:, :Hq] if Hq else None, here[:, Hq:Hq + Hk] if Hk else None, wd[0] if Hq else None,
                       wd[1] if Hk else None, 1e-5, table, None if pos is None else pos.cuda(), inter,
                       q_out=here[:, :Hq] if Hq else None, k_out=here[:, Hq:Hq + Hk] if Hk else None)
    if Hq:
        assert torch.equal(here[:, :Hq], out[0])
    if Hk:
        assert torch.equal(here[:, Hq:Hq + Hk], out[1])
    assert torch.equal(here[:, Hq + Hk:], dev[:, Hq + Hk:])


@gpu
def test_positions_outside_the_table_give_nan():
    x = torch.randn(4, 2, 64).cuda()
    table = P.slh_rope_table(10, 32)
    pos = torch.tensor([9, 10, -1, 0], dtype=torch.int32).cuda()
    y, _ = P.slh_qk_norm_rope(x, table=table, pos=pos)
    bad = torch.isnan(y).cpu()
    assert bool(bad[1:3, :, :32].all()) and not bool(bad[1:3, :, 32:].any()) and not bool(bad[[0, 3]].any())


@gpu
def test_norm_of_zero_rows_and_of_no_tokens():
    x = torch.zeros(3, 2, 128, dtype=BF).cuda()
    w = torch.ones(128, dtype=BF).cuda()
    y, _ = P.slh_qk_norm_rope(x, q_weight=w)
    assert not bool(y.any())
    assert P.slh_qk_norm_rope(x[:0], q_weight=w)[0].shape == (0, 2, 128)
    table, none = P.slh_rope_table(4, 64), torch.empty(0, dtype=torch.int32).cuda()
    assert P.slh_qk_norm_rope(x[:0], x[:0], w, w, table=table, pos=none)[1].shape == (0, 2, 128)
    kc = torch.zeros(1, 2, 16, 128, dtype=BF).cuda()
    P.slh_kv_append(x[:0], x[:0], kc, kc.clone(), none.long(), table=table, pos=none)
    cu = torch.tensor([0], dtype=torch.int32).cuda()
    assert P.slh_attend(x[:0], x[:0], x[:0], cu).shape == (0, 2, 128)
    assert P.slh_attend_paged(x[:0], kc, kc, none.view(0, 1), none).shape == (0, 2, 128)


# ---------------------------------------------------------------- cache append
@gpu
@pytest.mark.parametrize("dt", [BF, HF, F32])
@pytest.mark.parametrize("T,H,d,page,rot,norm", [(1, 1, 64, 1, 0, False), (53, 4, 128, 16, 128, True),
                                                 (40, 8, 80, 64, 32, False), (129, 3, 96, 8, 96, True)])
def test_kv_append(T, H, d, page, rot, norm, dt):
    g = _gen(T)
    pages = T // page + 5
    kv = torch.randn(T, 2 * H, d, generator=g).to(dt)
    kc, vc = (torch.randn(pages, H, page, d, generator=g).to(dt) for _ in range(2))
    slots = torch.randperm(pages * page, generator=g)[:T]
    slots[T // 2] = -1                            # padding, and a slot past the cache: left out
    if T > 8:
        slots[3] = pages * page
    w = (1 + torch.randn(d, generator=g) * 0.3).to(dt) if norm else None
    table = P.slh_rope_table(3 * T, rot) if rot else None
    pos = torch.randint(0, 3 * T, (T,), generator=g).int() if rot else None
    kd, vd, dev = kc.cuda(), vc.cuda(), kv.cuda()
    P.slh_kv_append(dev[:, :H], dev[:, H:], kd, vd, slots.cuda(), None if w is None else w.cuda(), 1e-6, table,
                    None if pos is None else pos.cuda())
    want, size = AP.norm_rope(kv[:, :H], w, 1e-6, None if table is None else table.cpu(), pos, False)
    tol = 1.01 * (AP.U[dt] * want.abs() + (d / 2 + 10) * 2.0 ** -24 * size) + (2.0 ** -25 if dt == HF else 0.0)
    kd, vd = kd.cpu(), vd.cpu()
    for t in range(T):
        s = int(slots[t])
        if 0 <= s < pages * page:
            _close(kd[s // page, :, s % page], want[t], tol[t])
            assert torch.equal(vd[s // page, :, s % page], kv[t, H:])
            kd[s // page, :, s % page], vd[s // page, :, s % page] = kc[s // page, :, s % page], vc[s // page, :, s % page]
    assert torch.equal(kd, kc) and torch.equal(vd, vc)          # nothing else changed


# ---------------------------------------------------------------- packed attention
def _attend_case(lq, lk, Hq, Hkv, d, dt, causal, seed, spoil=False, scale=None):
    """Runs slh_attend on q, k, v that are parts of wider rows, and checks out and lse."""
    g = _gen(seed)
    cq, ck = (torch.tensor([0] + x).cumsum(0).int() for x in (lq, lk))
    Tq, Tk = int(cq[-1]), int(ck[-1])
    qw = torch.randn(Tq, Hq + 1, d + 8, generator=g).to(dt)
    kw = torch.randn(Tk, 2 * Hkv, d, generator=g).to(dt)
    q, k, v = qw[:, 1:, :d], kw[:, :Hkv], kw[:, Hkv:]
    scale_ = 1 / math.sqrt(d) if scale is None else scale
    qd, kd = qw.cuda(), kw.cuda()
    out = torch.full((Tq, Hq, d), 7.0, dtype=dt).cuda()
    lse = torch.full((Tq, Hq), 7.0).cuda()
    P.slh_attend(qd[:, 1:, :d], kd[:, :Hkv], kd[:, Hkv:], cq.cuda(), ck.cuda(), scale=scale, causal=causal, out=out,
                 lse_out=lse)
    for b in range(len(lq)):
        limit = [lk[b] - lq[b] + i + 1 if causal else lk[b] for i in range(lq[b])]
        rq, rk = slice(int(cq[b]), int(cq[b + 1])), slice(int(ck[b]), int(ck[b + 1]))
        o, tol, e, etol = AP.attend(q[rq], k[rk], v[rk], limit, scale_)
        _close(out[rq], o, tol, f"sequence {b}")
        got = lse[rq].double().cpu()
        empty = e == -math.inf
        assert torch.equal(got[empty], e[empty])
        assert bool(((got - e).abs() <= etol)[~empty].all())


@gpu
@pytest.mark.parametrize("d", [64, 80, 96, 128])
@pytest.mark.parametrize("dt", [BF, HF])
@pytest.mark.parametrize("causal", [True, False])
def test_attend_packed(d, dt, causal):
    lq = [1, 0, 63, 64, 65, 33, 5, 3]
    lk = [1, 7, 63, 64, 65, 200, 2, 0]            # equal, none, a context before, fewer keys than queries, no keys
    _attend_case(lq, lk, 4, 2, d, dt, causal, d)


@gpu
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (7, 1), (28, 4), (40, 8), (6, 6)])
def test_attend_heads(Hq, Hkv):
    _attend_case([70, 19], [70, 90], Hq, Hkv, 128, BF, True, Hq)


@gpu
@pytest.mark.parametrize("n", [1, 2, 31, 32, 127, 128, 129, 257, 511])
def test_attend_lengths(n):
    _attend_case([n], [n], 2, 1, 64, BF, True, n)


@gpu
@pytest.mark.parametrize("lq,lk", [(1, 5000), (3, 4097), (40, 3001)])
def test_attend_few_queries_many_keys(lq, lk):
    _attend_case([lq, lq], [lk, 17 + lq], 5, 1, 128, BF, True, lk)


@gpu
@pytest.mark.parametrize("lk", [30, 6000])          # in one piece, and with the keys split
def test_attend_rows_of_no_sequence_and_wider_outputs(lk):
    """Rows in front of the first sequence and behind the last are not written, nor what lies beside out."""
    g = _gen(lk)
    q = torch.randn(20, 4, 64, generator=g).to(BF)
    k, v = (torch.randn(lk + 9, 2, 64, generator=g).to(BF) for _ in range(2))
    wide, lse = torch.full((20, 5, 72), 7.0, dtype=BF).cuda(), torch.full((20, 4), 7.0).cuda()
    cq, ck = torch.tensor([3, 5, 16], dtype=torch.int32), torch.tensor([4, 4 + lk // 3, 4 + lk], dtype=torch.int32)
    P.slh_attend(q.cuda(), k.cuda(), v.cuda(), cq.cuda(), ck.cuda(), out=wide[:, 1:, :64], lse_out=lse)
    for b in (0, 1):
        rq, rk = slice(int(cq[b]), int(cq[b + 1])), slice(int(ck[b]), int(ck[b + 1]))
        n, m = rq.stop - rq.start, rk.stop - rk.start
        o, tol, e, etol = AP.attend(q[rq], k[rk], v[rk], [m - n + i + 1 for i in range(n)], 1 / 8)
        _close(wide[rq, 1:, :64], o, tol)
        assert bool(((lse[rq].double().cpu() - e).abs() <= etol).all())
    wide[3:16, 1:, :64] = 7.0
    lse[3:16] = 7.0
    assert bool((wide == 7.0).all()) and bool((lse == 7.0).all())


@gpu
def test_attend_large_scores_and_scale():
    """Scores of several hundred: the running maximum moves by more than fp16 or exp can hold."""
    _attend_case([90], [90], 2, 1, 64, HF, True, 5, scale=8.0)
    _attend_case([90], [90], 2, 1, 64, BF, False, 6, scale=30.0)


@gpu
@pytest.mark.parametrize("dt", [BF, HF])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_attend_values_that_a_row_does_not_see(dt, bad):
    """Keys and values of later tokens, infinite or NaN, leave the rows before them alone; the
    rows that see them show what their definition gives: a NaN key makes the row NaN, an
    infinite value its element infinite."""
    g = _gen(3)
    n, at, d = 150, 75, 64
    q, k, v = (torch.randn(n, 1, d, generator=g).to(dt) for _ in range(3))
    cu = torch.tensor([0, n], dtype=torch.int32).cuda()
    clean = P.slh_attend(q.cuda(), k.cuda(), v.cuda(), cu).cpu()
    v2 = v.clone()
    v2[at, 0, 5] = bad
    got = P.slh_attend(q.cuda(), k.cuda(), v2.cuda(), cu).cpu()
    assert torch.equal(got[:at], clean[:at])
    other = [e for e in range(d) if e != 5]
    assert torch.equal(got[:, 0, other], clean[:, 0, other])
    assert torch.equal(torch.nan_to_num(got[at:, 0, 5], nan=9.0), torch.full((n - at,), 9.0 if math.isnan(bad) else bad).to(dt).nan_to_num(nan=9.0))
    k2 = k.clone()
    k2[at] = math.nan
    got = P.slh_attend(q.cuda(), k2.cuda(), v.cuda(), cu).cpu()
    assert torch.equal(got[:at], clean[:at]) and bool(torch.isnan(got[at:]).all())


@gpu
def test_attend_lowest_and_equal_scores():
    """Keys that give the type's lowest and highest values: a row of equal scores is a mean."""
    n, d = 70, 64
    q = torch.ones(n, 1, d, dtype=BF)
    v = torch.randn(n, 1, d, generator=_gen(1)).to(BF)
    cu = torch.tensor([0, n], dtype=torch.int32).cuda()
    for x in (torch.finfo(BF).min / 64, torch.finfo(BF).max / 64, 0.0):
        k = torch.full((n, 1, d), x, dtype=BF)
        out = P.slh_attend(q.cuda(), k.cuda(), v.cuda(), cu, scale=1.0)
        mean = v.double().cumsum(0) / torch.arange(1, n + 1)[:, None, None]
        A = v.double().abs().cumsum(0) / torch.arange(1, n + 1)[:, None, None]
        _close(out, mean, 1.02 * 2.0 ** -8 * (mean.abs() + A) + n * 2.0 ** -23 * A)


@gpu
@pytest.mark.parametrize("dt", [BF, HF])
@pytest.mark.parametrize("d", [64, 80, 96, 128])
def test_attend_again_gives_the_same_bits(dt, d):
    """Few rows and many, masked and whole steps: a result read before its product is done, or a
    buffer refilled while it is read, would differ from run to run."""
    g = _gen(d)
    for lq, lk, Hq, Hkv in (([65, 33, 7], [65, 200, 90], 4, 2), ([1300, 900], [1300, 2100], 28, 4)):
        cq, ck = (torch.tensor([0] + x, dtype=torch.int32).cumsum(0).int().cuda() for x in (lq, lk))
        q, k, v = (torch.randn(n, h, d, generator=g).to(dt).cuda() for n, h in ((sum(lq), Hq), (sum(lk), Hkv), (sum(lk), Hkv)))
        want = P.slh_attend(q, k, v, cq, ck)
        assert all(torch.equal(P.slh_attend(q, k, v, cq, ck), want) for _ in range(4))


@gpu
@pytest.mark.parametrize("dt", [BF, HF])
@pytest.mark.parametrize("d", [64, 80, 96, 128])
def test_paged_again_gives_the_same_bits(dt, d):
    g = _gen(d)
    for B_, n_q, Hq, Hkv, prefix in ((3, 1, 14, 2, 90), (3, 3, 14, 2, 90), (40, 3, 14, 2, 2000), (40, 1, 14, 2, 2000), (5, 5, 28, 1, 300)):
        pages = -(-prefix // 16)
        kc, vc = (torch.randn(pages + B_ * 9, Hkv, 16, d, generator=g).to(dt).cuda() for _ in range(2))
        table = (pages + torch.arange(B_ * 9, dtype=torch.int32)).view(B_, 9).cuda()
        lens = torch.randint(n_q, 145, (B_,), generator=g).int().cuda()
        q = torch.randn(B_, n_q, Hq, d, generator=g).to(dt).cuda()
        pre = torch.arange(pages, dtype=torch.int32).cuda()
        want = P.slh_attend_paged(q, kc, vc, table, lens, pre, prefix)
        assert all(torch.equal(P.slh_attend_paged(q, kc, vc, table, lens, pre, prefix), want) for _ in range(4))


@gpu
def test_attend_on_another_stream_and_in_a_graph():
    g = _gen(8)
    n = 200
    q, k, v = (torch.randn(n, h, 128, generator=g).to(BF).cuda() for h in (4, 2, 2))
    cu = torch.tensor([0, 77, n], dtype=torch.int32).cuda()
    want = P.slh_attend(q, k, v, cu)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    out = torch.empty_like(q)
    P.slh_attend(q, k, v, cu, out=out, stream=s)
    s.synchronize()
    assert torch.equal(out, want)
    graph, out = torch.cuda.CUDAGraph(), torch.empty_like(q)
    ws = torch.empty(max(1, P.slh_attend_workspace(n, n, 2, 4, 2, 128)), dtype=torch.uint8, device="cuda")
    with torch.cuda.graph(graph):
        P.slh_attend(q, k, v, cu, out=out, workspace=ws)
    for i in range(4):
        q.copy_(torch.randn(n, 4, 128, generator=g).to(BF))
        ws.fill_(255 - i)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, P.slh_attend(q, k, v, cu))


# ---------------------------------------------------------------- paged attention
def _paged_case(B_, n_q, Hq, Hkv, d, dt, page, prefix, lens, seed, spoil=math.nan):
    """Pages in random order; rows past a length hold `spoil`."""
    g = _gen(seed)
    own = [-(-n // page) for n in lens]
    n_pre = -(-prefix // page)
    most = max(own + [1]) + 1
    total = n_pre + sum(own) + 3
    kc, vc = (torch.full((total, Hkv, page, d), spoil).to(dt) for _ in range(2))
    order = torch.randperm(total, generator=g).int()
    table = torch.full((B_, most), 2 ** 30, dtype=torch.int32)      # entries that no length reaches
    at = n_pre
    for b in range(B_):
        table[b, :own[b]] = order[at:at + own[b]]
        at += own[b]
    pre = order[:n_pre].clone()

    def fill(pages, n):
        k, v = (torch.randn(n, Hkv, d, generator=g).to(dt) for _ in range(2))
        for j in range(n):
            kc[int(pages[j // page]), :, j % page], vc[int(pages[j // page]), :, j % page] = k[j], v[j]
        return k, v

    shared = fill(pre, prefix)
    mine = [fill(table[b], lens[b]) for b in range(B_)]
    q = torch.randn(B_, n_q, Hq, d, generator=g).to(dt)
    lse = torch.full((B_, n_q, Hq), 7.0).cuda()
    out = P.slh_attend_paged(q.cuda(), kc.cuda(), vc.cuda(), table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda(),
                             pre.cuda(), prefix, lse_out=lse)
    for b in range(B_):
        k, v = (torch.cat([shared[i], mine[b][i]]) for i in (0, 1))
        limit = [prefix + max(0, lens[b] - n_q + i + 1) for i in range(n_q)]
        o, tol, e, etol = AP.attend(q[b], k, v, limit, 1 / math.sqrt(d))
        _close(out[b], o, tol, f"sequence {b}")
        got, empty = lse[b].double().cpu(), e == -math.inf
        assert torch.equal(got[empty], e[empty]) and bool(((got - e).abs() <= etol)[~empty].all())


@gpu
@pytest.mark.parametrize("dt", [BF, HF])
@pytest.mark.parametrize("d", [64, 80, 96, 128])
@pytest.mark.parametrize("n_q", [1, 3])
def test_paged_types_and_heads(dt, d, n_q):
    _paged_case(3, n_q, 14, 2, d, dt, 16, 37, [n_q, 50, 129], d + n_q)


@gpu
@pytest.mark.parametrize("page", [1, 8, 32, 256])
@pytest.mark.parametrize("prefix", [0, 1, 64, 300])
def test_paged_pages_and_prefixes(page, prefix):
    _paged_case(4, 2, 4, 1, 64, BF, page, prefix, [2, 31, 64, 65], page + prefix)


@gpu
@pytest.mark.parametrize("prefix", [0, 40])
def test_paged_rows_without_own_keys(prefix):
    """Lengths of zero and of fewer rows than new tokens: those tokens see the prefix or nothing."""
    _paged_case(4, 3, 4, 2, 128, BF, 16, prefix, [0, 1, 2, 3], prefix)


@gpu
@pytest.mark.parametrize("B_,n_q,Hq,Hkv", [(1, 1, 1, 1), (1, 1, 28, 4), (2, 9, 8, 2), (33, 1, 8, 1), (70, 2, 4, 2), (300, 1, 2, 1)])
def test_paged_batches(B_, n_q, Hq, Hkv):
    lens = [n_q + (7 * b) % 90 for b in range(B_)]
    _paged_case(B_, n_q, Hq, Hkv, 64, BF, 16, 150, lens, B_)


@gpu
def test_paged_long():
    _paged_case(2, 1, 8, 2, 128, BF, 64, 5000, [9000, 1], 4)
    _paged_case(1, 2, 4, 4, 128, HF, 32, 0, [20011], 5)


@gpu
@pytest.mark.parametrize("B_,prefix", [(3, 700), (40, 3000)])      # one launch of rows; tiles and rows
def test_paged_strided_queries_and_outputs(B_, prefix):
    g = _gen(B_)
    page, Hkv, d, n_q = 16, 2, 96, 2
    n = -(-prefix // page)
    kc, vc = (torch.randn(n + B_ * 3, Hkv, page, d, generator=g).to(HF) for _ in range(2))
    wide = torch.randn(B_ * n_q, 9, d, generator=g).to(HF)
    out = torch.full((B_ * n_q, 9, d), 7.0, dtype=HF).cuda()
    table = torch.empty(B_, 5, dtype=torch.int32)
    table[:, :3] = n + torch.arange(B_ * 3).view(B_, 3)
    lens = torch.randint(2, 49, (B_,), generator=g).int()
    P.slh_attend_paged(wide.cuda().view(B_, n_q, 9, d)[:, :, 1:], kc.cuda(), vc.cuda(), table.cuda()[:, :3], lens.cuda(),
                       torch.arange(n, dtype=torch.int32).cuda(), prefix, out=out.view(B_, n_q, 9, d)[:, :, 1:])
    flat = [t.permute(0, 2, 1, 3).reshape(-1, Hkv, d) for t in (kc, vc)]
    for b in range(0, B_, 7):
        at = (n + 3 * b) * page
        k, v = (torch.cat([t[:prefix], t[at:at + int(lens[b])]]) for t in flat)
        o, tol, _, _ = AP.attend(wide[b * n_q:(b + 1) * n_q, 1:], k, v, [prefix + int(lens[b]) - n_q + i + 1 for i in range(n_q)], d ** -0.5)
        _close(out[b * n_q:(b + 1) * n_q, 1:], o, tol)
    assert bool((out[:, 0] == 7.0).all())


@gpu
@pytest.mark.parametrize("bad", [math.inf, math.nan])
def test_paged_tokens_that_a_new_token_does_not_see(bad):
    """The last new token's own value is infinite or NaN: the tokens before it do not change."""
    g = _gen(2)
    kc, vc = (torch.randn(8, 1, 16, 64, generator=g).to(BF).cuda() for _ in range(2))
    table = torch.arange(8, dtype=torch.int32).cuda()[None]
    lens = torch.tensor([100], dtype=torch.int32).cuda()
    q = torch.randn(1, 3, 2, 64, generator=g).to(BF).cuda()
    clean = P.slh_attend_paged(q, kc, vc, table, lens).cpu()
    vc[99 // 16, 0, 99 % 16] = bad
    got = P.slh_attend_paged(q, kc, vc, table, lens).cpu()
    assert torch.equal(got[:, :2], clean[:, :2]) and not bool(torch.isfinite(got[:, 2]).any())


@gpu
def test_caches_past_32_bits():
    """Rows whose offsets pass 2^32 elements, written and read back."""
    H, page, d = 8, 64, 128
    pages = 2 ** 32 // (H * page * d) + 3
    kc, vc = (torch.empty((pages, H, page, d), dtype=BF, device="cuda") for _ in range(2))
    g = _gen(9)
    n = 70
    k, v = (torch.randn(n, H, d, generator=g).to(BF) for _ in range(2))
    ids = torch.tensor([pages - 1, pages - 2], dtype=torch.int32)
    j = torch.arange(n)
    slots = ids.long()[j // page] * page + j % page
    P.slh_kv_append(k.cuda(), v.cuda(), kc, vc, slots.cuda())
    q = torch.randn(1, 1, 16, d, generator=g).to(BF)
    for kw in ({}, {"prefix_pages": ids.cuda(), "prefix_len": n}):
        lens = torch.tensor([0 if kw else n], dtype=torch.int32).cuda()
        out = P.slh_attend_paged(q.cuda(), kc, vc, ids.cuda()[None], lens, **kw)
        o, tol, _, _ = AP.attend(q[0], k, v, [n], 1 / math.sqrt(d))
        _close(out[0], o, tol)
    big = torch.empty((2 ** 32 // (H * d) + 100, H, d), dtype=BF, device="cuda")   # packed rows past 2^32 elements
    big[-n:] = k.cuda()
    cu = torch.tensor([len(big) - n, len(big)], dtype=torch.int32).cuda()
    big2 = torch.empty_like(big)
    big2[-n:] = v.cuda()
    qs = torch.randn(n, H, d, generator=g).to(BF)
    out = P.slh_attend(qs.cuda(), big, big2, torch.tensor([0, n], dtype=torch.int32).cuda(), cu)
    o, tol, _, _ = AP.attend(qs, k, v, [i + 1 for i in range(n)], 1 / math.sqrt(d))
    _close(out, o, tol)


@gpu
def test_paged_in_a_graph():
    g = _gen(12)
    kc, vc = (torch.randn(40, 2, 16, 128, generator=g).to(BF).cuda() for _ in range(2))
    table = torch.arange(40, dtype=torch.int32).cuda().view(2, 20)
    lens = torch.tensor([200, 13], dtype=torch.int32).cuda()
    pre = torch.arange(7, dtype=torch.int32).cuda()
    q = torch.randn(2, 1, 8, 128, generator=g).to(BF).cuda()
    out = torch.empty_like(q)
    ws = torch.empty(max(1, P.slh_attend_paged_workspace(2, 1, 8, 2, 128, 320, 100)), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        P.slh_attend_paged(q, kc, vc, table, lens, pre, 100, out=out, workspace=ws)
    for i in range(4):
        lens.copy_(torch.tensor([20 + 90 * i, 320 - 80 * i], dtype=torch.int32))
        q.copy_(torch.randn(2, 1, 8, 128, generator=g).to(BF))
        ws.fill_(255 - i)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, P.slh_attend_paged(q, kc, vc, table, lens, pre, 100))


# ---------------------------------------------------------------- blocks of 64 rows, joins of many splits
@gpu
@pytest.mark.parametrize("d", [64, 80, 96, 128])
@pytest.mark.parametrize("dt", [BF, HF])
def test_attend_prompts_between_few_and_many_rows(d, dt):
    """Sizes between the kernels of few rows and of many: whole and ragged blocks, more keys than queries,
    sequences of one token and of none."""
    _attend_case([561], [561], 32, 4, d, dt, True, d)
    _attend_case([257, 1, 0, 302], [257, 1, 3, 365], 32, 4, d, dt, True, d + 1)
    _attend_case([190, 330], [201, 63], 32, 4, d, dt, False, d + 2)


@gpu
@pytest.mark.parametrize("lq,lk", [([60], [4001]), ([129, 31], [1500, 2000])])
def test_attend_some_queries_many_keys(lq, lk):
    _attend_case(lq, lk, 28, 4, 128, BF, True, len(lq))


@gpu
@pytest.mark.parametrize("dt", [BF, HF])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("at", [300, 351])         # in the first and the second half of a tile's keys
def test_attend_values_not_seen_in_blocks_of_64_rows(dt, bad, at):
    g = _gen(4)
    n, d, Hq, Hkv = 560, 64, 32, 4
    q, k, v = (torch.randn(n, h, d, generator=g).to(dt) for h in (Hq, Hkv, Hkv))
    cu = torch.tensor([0, n], dtype=torch.int32).cuda()
    clean = P.slh_attend(q.cuda(), k.cuda(), v.cuda(), cu).cpu()
    v2 = v.clone()
    v2[at, 2, 5] = bad
    got = P.slh_attend(q.cuda(), k.cuda(), v2.cuda(), cu).cpu()
    want = clean.clone()
    want[at:, 16:24, 5] = bad
    assert torch.equal(got.nan_to_num(nan=9.0), want.nan_to_num(nan=9.0))
    k2 = k.clone()
    k2[at, 2] = math.nan
    got = P.slh_attend(q.cuda(), k2.cuda(), v.cuda(), cu).cpu()
    want = clean.clone()
    want[at:, 16:24] = math.nan
    assert torch.equal(got.nan_to_num(nan=9.0), want.nan_to_num(nan=9.0))


@gpu
@pytest.mark.parametrize("dt", [BF, HF])
@pytest.mark.parametrize("d", [64, 80, 96, 128])
def test_attend_blocks_of_64_rows_again_give_the_same_bits(dt, d):
    g = _gen(d + 7)
    cu = torch.tensor([0, 560, 1100], dtype=torch.int32).cuda()
    q, k, v = (torch.randn(1100, h, d, generator=g).to(dt).cuda() for h in (28, 4, 4))
    want = P.slh_attend(q, k, v, cu)
    assert all(torch.equal(P.slh_attend(q, k, v, cu), want) for _ in range(4))


@gpu
@pytest.mark.parametrize("d", [64, 80, 128])
@pytest.mark.parametrize("dt", [BF, HF])
def test_paged_many_splits_of_few_rows(d, dt):
    _paged_case(1, 1, 7, 1, d, dt, 64, 2000, [3001], d)
    _paged_case(2, 1, 4, 2, d, dt, 16, 0, [4100, 1], d + 1)


@gpu
@pytest.mark.parametrize("dt", [BF, HF])
@pytest.mark.parametrize("d", [64, 80, 96, 128])
def test_paged_prefixes_read_by_each_sequence_and_by_all(d, dt):
    """A short prefix stands in front of every sequence's own keys, a long one has blocks of its own: ends inside
    a step and a page, sequences without own keys, several new tokens."""
    _paged_case(24, 1, 8, 2, d, dt, 16, 131, [b % 9 + (b > 2) * 11 for b in range(24)], d)
    _paged_case(3, 5, 6, 3, d, dt, 4, 77, [64, 3, 0], d + 1)
    _paged_case(2, 3, 14, 2, d, dt, 32, 1501, [3, 20], d + 2)
    _paged_case(40, 3, 8, 1, d, dt, 64, 3001, [3 + b for b in range(40)], d + 3)


@gpu
@pytest.mark.parametrize("d,dt", [(64, HF), (128, BF)])
def test_paged_many_rows_against_a_long_prefix(d, dt):
    """The prefix in tiles of many rows, the own keys by few."""
    _paged_case(128, 2, 28, 1, d, dt, 32, 3001, [2 + (5 * b) % 31 for b in range(128)], d)


# ---------------------------------------------------------------- refusals
def test_library_refuses_before_any_gpu_work():
    lib = B.load()
    p = 4096                                      # an aligned address that nothing reads
    rope = dict(q=p, q_st=128, q_sh=64, Hq=2, qo=p, qo_st=128, qo_sh=64, k=None, k_st=0, k_sh=0, Hk=0, ko=None, ko_st=0,
                ko_sh=0, dt=0, T=3, d=64, wq=None, wk=None, eps=1e-6, table=None, n_pos=0, rot=0, pos=None, inter=0, st=None)
    bad = [dict(q=p + 2), dict(q=None), dict(q_st=12), dict(q_sh=-64), dict(dt=3), dict(T=-1), dict(d=12), dict(d=264), dict(d=0),
           dict(eps=-1.0), dict(eps=math.nan), dict(rot=16), dict(table=p, rot=24, n_pos=9, pos=p), dict(Hq=0), dict(Hq=-1),
           dict(table=p, rot=128, n_pos=9, pos=p), dict(table=p, rot=64, n_pos=0, pos=p), dict(table=p, rot=64, n_pos=9),
           dict(T=2 ** 27), dict(wq=p + 4), dict(qo=None)]
    for b in bad:
        assert lib.slh_qk_norm_rope(*{**rope, **b}.values()) == B.SLH_EINVAL, b
    app = dict(k=p, k_st=128, k_sh=64, v=p, v_st=128, v_sh=64, dt=0, T=3, H=2, d=64, wk=None, eps=1e-6, table=None, n_pos=0, rot=0,
               pos=None, inter=0, kc=p, vc=p, pages=4, page=16, slots=p, st=None)
    for b in [dict(page=24), dict(page=0), dict(page=1 << 17), dict(pages=-1), dict(slots=None), dict(kc=None), dict(vc=p + 8),
              dict(H=0), dict(v_sh=4), dict(d=60), dict(dt=-1)]:
        assert lib.slh_kv_append(*{**app, **b}.values()) == B.SLH_EINVAL, b
    att = dict(q=p, q_st=128, q_sh=64, k=p, k_st=64, k_sh=64, v=p, v_st=64, v_sh=64, dt=0, Tq=3, Tk=3, B=1, Hq=2, Hkv=1, d=64, cq=p,
               ck=p, scale=0.1, causal=1, out=p, o_st=128, o_sh=64, lse=None, ws=None, n=0, st=None)
    for b in [dict(dt=1), dict(d=72), dict(d=256), dict(Hq=3, Hkv=2), dict(Hkv=0), dict(scale=0.0), dict(scale=-1.0),
              dict(scale=math.inf), dict(scale=math.nan), dict(cq=None), dict(ck=None), dict(q=p + 8), dict(v_st=4), dict(out=None),
              dict(B=-1), dict(Tk=-1), dict(k=None), dict(Tq=2 ** 31)]:
        assert lib.slh_attend(*{**att, **b}.values()) == B.SLH_EINVAL, b
    pag = dict(q=p, q_st=128, q_sh=64, kc=p, vc=p, dt=0, pages=4, page=16, B=2, n_q=1, Hq=2, Hkv=1, d=64, table=p, ld=3, most=3, lens=p,
               pre=None, plen=0, scale=0.1, out=p, o_st=128, o_sh=64, lse=None, ws=None, n=0, st=None)
    for b in [dict(dt=1), dict(page=20), dict(pages=0), dict(ld=2), dict(lens=None), dict(table=None), dict(plen=5), dict(plen=-1),
              dict(n_q=-1), dict(kc=None), dict(d=48), dict(scale=0.0), dict(most=-1), dict(q=None)]:
        assert lib.slh_attend_paged(*{**pag, **b}.values()) == B.SLH_EINVAL, b
    table = dict(t=p, n=4, rot=64, base=1e4, scaling=0, factor=1.0, orig=0, fast=32.0, slow=1.0, st=None)
    for b in [dict(t=None), dict(n=0), dict(rot=24), dict(rot=272), dict(base=1.0), dict(scaling=4), dict(scaling=1, factor=0.5),
              dict(scaling=3, factor=2.0, orig=0), dict(scaling=3, factor=2.0, orig=9, fast=1.0), dict(base=math.nan)]:
        assert lib.slh_rope_table(*{**table, **b}.values()) == B.SLH_EINVAL, b


def test_library_refuses_past_its_limits():
    lib = B.load()
    p = 4096                                      # an aligned address that nothing reads
    att = dict(q=p, q_st=128, q_sh=64, k=p, k_st=64, k_sh=64, v=p, v_st=64, v_sh=64, dt=0, Tq=3, Tk=3, B=1, Hq=2, Hkv=1, d=64, cq=p,
               ck=p, scale=0.1, causal=1, out=p, o_st=128, o_sh=64, lse=None, ws=None, n=0, st=None)
    for b in [dict(scale=1e300), dict(scale=1e38), dict(scale=1e-40), dict(k_st=2 ** 24 + 8), dict(v_st=2 ** 25), dict(q_st=2 ** 24 + 8),
              dict(Hq=2048), dict(B=2 ** 20 + 1), dict(B=2 ** 20, Hkv=16, Hq=16),
              dict(Tq=2 ** 20, Tk=2 ** 20, B=2 ** 18, Hkv=64, Hq=64)]:
        assert lib.slh_attend(*{**att, **b}.values()) == B.SLH_EINVAL, b
    need = lib.slh_attend_workspace(3, 4096, 1, 2, 1, 64, 1)
    assert need > 0
    for b in [dict(ws=None, n=need), dict(ws=p, n=need - 1), dict(ws=p + 8, n=need)]:
        assert lib.slh_attend(*{**att, "Tk": 4096, **b}.values()) == B.SLH_EINVAL, b
    pag = dict(q=p, q_st=128, q_sh=64, kc=p, vc=p, dt=0, pages=4, page=16, B=2, n_q=1, Hq=2, Hkv=1, d=64, table=p, ld=3, most=3, lens=p,
               pre=None, plen=0, scale=0.1, out=p, o_st=128, o_sh=64, lse=None, ws=None, n=0, st=None)
    for b in [dict(pages=2 ** 27), dict(pages=2 ** 31), dict(page=1 << 17), dict(scale=1e38), dict(most=2 ** 26, ld=2 ** 26),
              dict(B=2 ** 20, Hq=16, Hkv=16), dict(pre=p, plen=2 ** 30), dict(B=1, most=2000, ld=2000, pages=2000)]:
        assert lib.slh_attend_paged(*{**pag, **b}.values()) == B.SLH_EINVAL, b


def test_host_tensors_are_refused():
    x = torch.zeros(2, 2, 64, dtype=BF)
    cu = torch.tensor([0, 2], dtype=torch.int32)
    for call in (lambda: P.slh_qk_norm_rope(x), lambda: P.slh_attend(x, x, x, cu),
                 lambda: P.slh_kv_append(x, x, x[None], x[None], cu.long()),
                 lambda: P.slh_attend_paged(x, x[None], x[None], cu[None], cu)):
        with pytest.raises(P.SLHError):
            call()


@gpu
def test_binding_refusals():
    x = torch.zeros(4, 2, 64, dtype=BF).cuda()
    cu = torch.tensor([0, 4], dtype=torch.int32).cuda()
    kc = torch.zeros(2, 2, 16, 64, dtype=BF).cuda()
    pt, lens = torch.zeros(4, 1, dtype=torch.int32).cuda(), torch.ones(4, dtype=torch.int32).cuda()
    table, pos = P.slh_rope_table(8, 64), torch.zeros(4, dtype=torch.int32).cuda()
    calls = [
        lambda: P.slh_qk_norm_rope(x, x[:3]), lambda: P.slh_qk_norm_rope(x, x.half()), lambda: P.slh_qk_norm_rope(x, table=table),
        lambda: P.slh_qk_norm_rope(x, table=table, pos=pos.long()), lambda: P.slh_qk_norm_rope(x, table=table, pos=pos[:3]),
        lambda: P.slh_qk_norm_rope(x, q_weight=torch.ones(64).cuda()), lambda: P.slh_qk_norm_rope(x.transpose(1, 2)),
        lambda: P.slh_qk_norm_rope(x, q_out=x[:3]), lambda: P.slh_qk_norm_rope(None), lambda: P.slh_qk_norm_rope(x[:, :, 4:]),
        lambda: P.slh_kv_append(x, x, kc, kc[:1], pos.long()), lambda: P.slh_kv_append(x, x, kc, kc, pos),
        lambda: P.slh_kv_append(x, x[:, :1], kc, kc, pos.long()), lambda: P.slh_kv_append(x, x, kc.half(), kc.half(), pos.long()),
        lambda: P.slh_attend(x, x, x, cu.long()), lambda: P.slh_attend(x.float(), x.float(), x.float(), cu),
        lambda: P.slh_attend(x, x, x[:3], cu), lambda: P.slh_attend(x, x, x, cu, out=x[:3]),
        lambda: P.slh_attend(x, x, x, cu, scale=0.0), lambda: P.slh_attend(x, x, x, cu, lse_out=torch.zeros(4, 3).cuda()),
        lambda: P.slh_attend(x, x, x, cu, cu[:1]), lambda: P.slh_attend_paged(x, kc, kc, pt[:3], lens),
        lambda: P.slh_attend_paged(x, kc, kc, pt, lens.long()), lambda: P.slh_attend_paged(x, kc, kc, pt, lens, prefix_len=3),
        lambda: P.slh_attend_paged(x, kc, kc, pt, lens, pt[:1, 0].contiguous(), 17),
        lambda: P.slh_attend_paged(x.view(2, 2, 2, 64).transpose(0, 1), kc, kc, pt[:2], lens[:2]),
    ]
    for i, call in enumerate(calls):
        with pytest.raises(P.SLHError):
            call()
            print("not refused:", i)
