"""Each way in which slh_attend and slh_attend_paged go about a call: blocks of 16, 32, 64 and 128 rows, keys split or
not, a prefix in front of each sequence's own keys, in parts of its own, in one launch with them or in another.
The shapes say which (checked without a GPU, for all head sizes, against the plans of a card of 256 compute
units); values are compared with the definition in 64 bits (the tolerances of attention_plain.py)."""
import math
import random

import pytest
import torch

import attend_plan
import attention_plain as AP
import paper_2607_19368_amd as P

gpu = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16
SIZES = [64, 80, 96, 128]

# (queries, keys, sequences, query heads, key/value heads): kernel, rows of a block, whether the keys are split
PACKED = {
    (89, 160, 3, 14, 2): ("rows", 16, False),
    (7, 5003, 3, 5, 1): ("rows", 16, True),
    (560, 560, 64, 14, 1): ("rows", 32, False),
    (20, 12020, 4, 28, 4): ("rows", 32, True),
    (560, 626, 4, 32, 4): ("tiles", 64, False),
    (130, 5230, 3, 16, 1): ("tiles", 64, True),
    (2200, 3400, 3, 28, 4): ("tiles", 128, False),
    (130, 27130, 9, 28, 4): ("tiles", 128, True),
}
# (sequences, new tokens, query heads, key/value heads, page size, pages a sequence, prefix): the launches (kernel, rows of
# a block), whether partial results are joined, whether the prefix is read in front of each sequence's own keys
PAGED = {
    (3, 2, 14, 2, 16, 9, 0): ([("rows", 16)], False, False),
    (3, 2, 14, 2, 4, 36, 0): ([("rows", 16)], False, False),
    (2, 1, 4, 2, 64, 60, 0): ([("rows", 16)], True, False),
    (24, 1, 8, 2, 16, 2, 131): ([("rows", 16)], False, True),
    (24, 1, 8, 2, 2, 16, 131): ([("rows", 16)], False, True),
    (1, 1, 4, 4, 64, 1, 2001): ([("rows", 16)], True, False),
    (1, 3, 4, 4, 16, 2000, 77): ([("rows", 16)], True, False),
    (128, 2, 28, 1, 16, 1, 0): ([("rows", 32)], False, False),
    (24, 5, 64, 8, 16, 1, 77): ([("rows", 32)], False, True),
    (1, 5, 28, 4, 64, 512, 0): ([("rows", 32)], True, False),
    (1, 5, 28, 4, 16, 2048, 77): ([("rows", 32)], True, False),
    (8, 5, 40, 8, 16, 6, 5000): ([("both", 16)], True, False),
    (1, 40, 40, 8, 64, 1, 5000): ([("both", 16)], True, False),
    (2, 16, 64, 8, 64, 50, 5000): ([("both", 32)], True, False),
    (64, 5, 28, 4, 16, 1, 0): ([("tiles", 128)], False, False),
    (2, 5, 28, 4, 64, 512, 0): ([("tiles", 128)], True, False),
    (2, 5, 28, 4, 16, 2048, 0): ([("tiles", 128)], True, False),
    (8, 5, 28, 4, 128, 24, 500): ([("tiles", 128)], True, False),
    (2, 5, 28, 4, 4, 8192, 77): ([("tiles", 128)], True, False),
    (2, 5, 28, 4, 16, 2048, 5000): ([("rows", 16), ("tiles", 128)], True, False),
    (1, 16, 64, 8, 64, 512, 2001): ([("rows", 32), ("tiles", 128)], True, False),
}


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    return attend_plan.build(tmp_path_factory.mktemp("attend"))


@pytest.mark.parametrize("shape", PACKED)
def test_packed_shapes_take_their_paths(plans, shape):
    for d in SIZES:
        for causal in (True, False):
            first, *rest = plans.packed(*shape, d, causal)
            assert (first[0], first[2], bool(rest)) == PACKED[shape], (d, causal)


@pytest.mark.parametrize("shape", PAGED)
def test_paged_shapes_take_their_paths(plans, shape):
    for d in SIZES:
        done = plans.paged(*shape[:4], d, *shape[4:])
        kernels = [x for x in done if x[0] != "join"]
        assert ([(x[0], x[2]) for x in kernels], len(done) > len(kernels), bool(kernels[0][7])) == PAGED[shape], d


def test_a_long_prefix_is_read_once_whatever_the_tables_width(plans):
    """Tables are as wide as the longest sequence may become; what a call reads goes by the lengths."""
    for Hq, Hkv in ((28, 4), (32, 8), (40, 8)):
        for n in (64, 128, 256):
            for prefix in (8000, 32768):
                for page in (16, 64):
                    want = plans.paged(n, 1, Hq, Hkv, 128, page, 704 // page, prefix)
                    assert want[0][7] == 0 and want[0][5] > 0
                    for width in (1408, 4096, 8192, 32768, 131072):
                        got = plans.paged(n, 1, Hq, Hkv, 128, page, width // page, prefix)
                        assert got[0][7] == 0 and got[0][5] > 0, (Hq, n, prefix, width)
                        assert got == want or Hkv != 4, (n, prefix, width)
    # a short one is not worth a second launch
    for n, prefix, own in ((8, 512, 112), (64, 512, 64), (4, 300, 304), (32, 300, 704), (256, 64, 32)):
        assert plans.paged(n, 1, 28, 4, 128, 16, own // 16, prefix)[0][7] == 1, (n, prefix, own)


# ---------------------------------------------------------------- the definition, on the card in 64 bits
def rows_of(q, k, v, limit, scale):
    """(o, tolerance, lse, its tolerance) of rows q [n, Hq, d] over k, v [m, Hkv, d]; row i sees limit[i] keys.
    The formulas of AP.one_row, all rows of a head at once."""
    n, Hq, d = q.shape
    g = Hq // k.shape[1]
    m = len(k)
    limit = torch.as_tensor(list(limit), device=q.device).clamp(0, m)
    o, tol = (torch.zeros((n, Hq, d), dtype=torch.float64, device=q.device) for _ in range(2))
    lse, ltol = (torch.zeros((n, Hq), dtype=torch.float64, device=q.device) for _ in range(2))
    seen = torch.arange(m, device=q.device)[None] < limit[:, None]
    none = limit == 0
    lse[none] = -math.inf
    for h in range(Hq) if m else ():
        qh, kh, vh = q[:, h].double(), k[:, h // g].double(), v[:, h // g].double()
        s = (qh @ kh.t().contiguous() * scale).masked_fill(~seen, -math.inf)
        top = s.amax(-1, keepdim=True)
        p = torch.exp(s - top).masked_fill(~seen, 0.0)
        total = p.sum(-1, keepdim=True)
        x, A = p @ vh / total, p @ vh.abs() / total
        size = (qh.abs() @ kh.abs().t().contiguous() * scale).masked_fill(~seen, 0.0).amax(-1, keepdim=True)
        e = 2 * (d + 8) * 2.0 ** -24 * (size + 1)
        t = 1.02 * AP.U[q.dtype] * (x.abs() + A) + 2 * (e + limit[:, None] * 2.0 ** -24) * A
        if q.dtype == HF:
            t = t + 2.0 ** -25 * (seen.double() @ vh.abs()) / total + 2.0 ** -25
        o[:, h], tol[:, h] = x.masked_fill(none[:, None], 0.0), t.masked_fill(none[:, None], 0.0)
        lse[:, h] = (total.log() + top)[:, 0].masked_fill(none, -math.inf)
        ltol[:, h] = e[:, 0] + (limit + 8) * 2.0 ** -24 * (1 + top[:, 0].abs())
    return o, tol, lse, ltol


def close(got, want, tol, what):
    assert bool(torch.isfinite(got).all()), f"{what}: not finite"
    over = float(((got.double() - want).abs() - tol).max()) if got.numel() else 0.0
    assert over <= 0.0, f"{what}: {over:.3g} past the tolerance"


def close_lse(got, want, tol, what):
    none = want == -math.inf
    assert torch.equal(got.double()[none], want[none]), what
    assert bool(((got.double() - want).abs() <= tol)[~none].all()), what


def lengths(Tq, Tk, n, seed):
    """Queries and keys of n sequences, ragged; of three or more, one has no queries and one no keys; some have fewer
    keys than queries."""
    r = random.Random(seed)

    def share(total, empty):
        w = [0.0 if i == empty else r.uniform(0.2, 1.0) for i in range(n)]
        out = [int(total * x / sum(w)) for x in w]
        out[0] += total - sum(out)
        return out

    return share(Tq, 1 if n > 2 else None), share(Tk, 2 if n > 2 else None)


class Packed:
    """Inputs of a packed shape, parts of wider rows."""

    def __init__(self, shape, d, dt, causal):
        self.Tq, self.Tk, self.n, self.Hq, self.Hkv = shape
        self.d, self.causal, self.scale = d, causal, None
        g = torch.Generator(device="cuda")
        g.manual_seed(d + self.Tq)
        self.lq, self.lk = lengths(self.Tq, self.Tk, self.n, d)
        self.q = torch.randn(self.Tq, self.Hq + 1, d + 8, generator=g, device="cuda").to(dt)[:, 1:, :d]
        kv = torch.randn(self.Tk, 2 * self.Hkv, d, generator=g, device="cuda").to(dt)
        self.k, self.v = kv[:, :self.Hkv], kv[:, self.Hkv:]
        self.cq, self.ck = (torch.tensor([0] + x, device="cuda").cumsum(0).int() for x in (self.lq, self.lk))

    def run(self, k=None, v=None):
        """Output and lse; every row belongs to a sequence."""
        out = torch.full((self.Tq, self.Hq, self.d), 7.0, dtype=self.q.dtype, device="cuda")
        lse = torch.full((self.Tq, self.Hq), 7.0, device="cuda")
        P.slh_attend(self.q, self.k if k is None else k, self.v if v is None else v, self.cq, self.ck, scale=self.scale,
                     causal=self.causal, out=out, lse_out=lse)
        return out, lse

    def sequences(self):
        """(rows, keys, limits) of each sequence."""
        iq = ik = 0
        for nq, nk in zip(self.lq, self.lk):
            yield slice(iq, iq + nq), slice(ik, ik + nk), [nk - nq + i + 1 if self.causal else nk for i in range(nq)]
            iq, ik = iq + nq, ik + nk


@gpu
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dt", [BF, HF])
@pytest.mark.parametrize("d", SIZES)
@pytest.mark.parametrize("shape", PACKED)
def test_packed_paths(shape, d, dt, causal):
    c = Packed(shape, d, dt, causal)
    out, lse = c.run()
    for b, (rq, rk, limit) in enumerate(c.sequences()):
        o, tol, e, etol = rows_of(c.q[rq], c.k[rk], c.v[rk], limit, d ** -0.5)
        close(out[rq], o, tol, f"sequence {b}")
        close_lse(lse[rq], e, etol, f"sequence {b}")


@gpu
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("dt", [BF, HF])
@pytest.mark.parametrize("d", [80, 128])
@pytest.mark.parametrize("shape", PACKED)
def test_packed_paths_unseen_values(shape, d, dt, bad):
    """A late key's value is infinite or NaN in one element, or the whole key is NaN: rows that do not see it are as
    without, rows that do show it."""
    c = Packed(shape, d, dt, True)
    clean, _ = c.run()
    rq, rk, limit = max(c.sequences(), key=lambda s: min(s[0].stop - s[0].start, s[1].stop - s[1].start))
    at = rk.stop - min(max(1, len(limit) // 2), rk.stop - rk.start)      # the middle of the queries sees it first
    from_row = rq.start + next(i for i, n in enumerate(limit) if n > at - rk.start)
    head = c.Hkv - 1
    heads = slice(head * c.Hq // c.Hkv, c.Hq)
    v = c.v.clone()
    v[at, head, 5] = bad
    want = clean.clone()
    want[from_row:rq.stop, heads, 5] = bad
    assert torch.equal(c.run(v=v)[0].nan_to_num(nan=9.0), want.nan_to_num(nan=9.0))
    k = c.k.clone()
    k[at, head] = math.nan
    got = c.run(k=k)[0]
    assert bool(torch.isnan(got[from_row:rq.stop, heads]).all())
    # when a row's running maximum moves, those of the rows beside it in a wave do: not the same bits
    o, tol, _, _ = rows_of(c.q[rq.start:from_row, heads], c.k[rk, head:], c.v[rk, head:], limit[:from_row - rq.start], d ** -0.5)
    close(got[rq.start:from_row, heads], o, tol, "rows that do not see the key")
    got[rq, heads] = clean[rq, heads]
    assert torch.equal(got, clean)


class Paged:
    """Inputs of a paged shape: pages in random order, rows that no length reaches hold NaN."""

    def __init__(self, shape, d, dt):
        self.n, self.n_q, self.Hq, self.Hkv, page, width, self.prefix = shape
        self.d, self.page, self.scale = d, page, None
        g = torch.Generator(device="cuda")
        g.manual_seed(d + self.prefix)
        r = random.Random(d)
        most = min(width * page, 700)
        self.lens = [r.randint(0, most) for _ in range(self.n)]
        self.lens[0] = min(width * page, 3007)
        if self.n > 2:
            self.lens[1:3] = 0, min(most, self.n_q)
        used, n_pre = [-(-x // page) for x in self.lens], -(-self.prefix // page)
        total = n_pre + sum(used) + 3
        order = torch.randperm(total, generator=g, device="cuda").int()
        self.pre = order[:n_pre].clone()
        self.table = torch.full((self.n, width), 2 ** 30, dtype=torch.int32, device="cuda")
        at = n_pre
        for b, x in enumerate(used):
            self.table[b, :x] = order[at:at + x]
            at += x
        self.kc, self.vc = (torch.randn(total, self.Hkv, page, d, generator=g, device="cuda").to(dt) for _ in range(2))
        for cache in (self.kc, self.vc):
            if self.prefix % page:
                cache[self.pre[-1], :, self.prefix % page:] = math.nan
            for b, x in enumerate(self.lens):
                if x % page:
                    cache[self.table[b, x // page], :, x % page:] = math.nan
            cache[order[-3:].long()] = math.nan
        self.q = torch.randn(self.n, self.n_q, self.Hq, d, generator=g, device="cuda").to(dt)
        self.len_ = torch.tensor(self.lens, dtype=torch.int32, device="cuda")

    def run(self):
        lse = torch.full(self.q.shape[:3], 7.0, device="cuda")
        out = torch.full_like(self.q, 7.0)
        P.slh_attend_paged(self.q, self.kc, self.vc, self.table, self.len_, self.pre, self.prefix, scale=self.scale, out=out,
                           lse_out=lse)
        return out, lse

    def keys(self, b):
        """All keys and values of sequence b, the prefix first, and its tokens' limits."""
        pages = torch.cat([self.pre, self.table[b, :-(-self.lens[b] // self.page)]]).long()
        k, v = (t[pages].permute(0, 2, 1, 3).reshape(-1, self.Hkv, self.d) for t in (self.kc, self.vc))
        n_pre = len(self.pre) * self.page
        keep = [torch.cat([t[:self.prefix], t[n_pre:n_pre + self.lens[b]]]) for t in (k, v)]
        return *keep, [self.prefix + max(0, self.lens[b] - self.n_q + i + 1) for i in range(self.n_q)]


@gpu
@pytest.mark.parametrize("dt", [BF, HF])
@pytest.mark.parametrize("d", SIZES)
@pytest.mark.parametrize("shape", PAGED)
def test_paged_paths(shape, d, dt):
    c = Paged(shape, d, dt)
    out, lse = c.run()
    for b in range(c.n) if c.n <= 8 else list(range(5)) + [c.n // 2, c.n - 1]:
        k, v, limit = c.keys(b)
        o, tol, e, etol = rows_of(c.q[b], k, v, limit, d ** -0.5)
        close(out[b], o, tol, f"sequence {b}")
        close_lse(lse[b], e, etol, f"sequence {b}")


@gpu
@pytest.mark.parametrize("bad", [math.inf, math.nan])
@pytest.mark.parametrize("dt", [BF, HF])
@pytest.mark.parametrize("d", [80, 128])
@pytest.mark.parametrize("shape", [s for s in PAGED if s[1] > 1])
def test_paged_paths_unseen_values(shape, d, dt, bad):
    """The first sequence's last token has an infinite or NaN value: only that token shows it."""
    c = Paged(shape, d, dt)
    clean, _ = c.run()
    j = c.lens[0] - 1
    c.vc[c.table[0, j // c.page], c.Hkv - 1, j % c.page, 5] = bad
    want = clean.clone()
    want[0, -1, (c.Hkv - 1) * c.Hq // c.Hkv:, 5] = bad
    assert torch.equal(c.run()[0].nan_to_num(nan=9.0), want.nan_to_num(nan=9.0))


# ---------------------------------------------------------------- partial results: graphs, streams, dirty memory
def _splits(pre, own):
    """Packed (lengths of keys) and paged (lengths) calls whose keys are split, more and less full."""
    return [(pre, own), (0, 1), (pre // 3, own // 2), (pre, 0), (5, own)]


@gpu
@pytest.mark.parametrize("lq,heads,d", [(20, (4, 2), 64), (130, (16, 1), 128)])          # joined by four waves, by one
def test_packed_splits_in_a_graph_and_on_another_stream(lq, heads, d):
    """Partial results in memory that holds NaN before each replay, with splits that are empty in some: the eager
    call's bits."""
    Hq, Hkv = heads
    most = 6000
    need = P.slh_attend_workspace(lq, most, 2, Hq, Hkv, d)
    assert need > 0
    g = torch.Generator(device="cuda")
    g.manual_seed(lq)
    q = torch.randn(lq, Hq, d, generator=g, device="cuda").to(BF)
    k, v = (torch.randn(most, Hkv, d, generator=g, device="cuda").to(BF) for _ in range(2))
    cq = torch.tensor([0, lq // 2, lq], dtype=torch.int32, device="cuda")
    ck = torch.tensor([0, 2500, most], dtype=torch.int32, device="cuda")
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    out, lse = torch.empty_like(q), torch.empty(lq, Hq, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        P.slh_attend(q, k, v, cq, ck, out=out, lse_out=lse, workspace=ws)
    side = torch.cuda.Stream()
    for a, b in _splits(2500, 3500):
        ck.copy_(torch.tensor([0, a, a + b], dtype=torch.int32))
        q.copy_(torch.randn(lq, Hq, d, generator=g, device="cuda"))
        want_lse = torch.empty_like(lse)
        want = P.slh_attend(q, k, v, cq, ck, lse_out=want_lse)
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, want_lse)
        for rows, keys in ((slice(0, lq // 2), slice(0, a)), (slice(lq // 2, lq), slice(a, a + b))):
            n, m = rows.stop - rows.start, keys.stop - keys.start
            o, tol, e, etol = rows_of(q[rows], k[keys], v[keys], [m - n + i + 1 for i in range(n)], d ** -0.5)
            close(out[rows], o, tol, f"{a} and {b} keys")
            close_lse(lse[rows], e, etol, f"{a} and {b} keys")
        ws.fill_(255)
        out.fill_(7.0)
        side.wait_stream(torch.cuda.current_stream())
        P.slh_attend(q, k, v, cq, ck, out=out, workspace=ws, stream=side)
        side.synchronize()
        assert torch.equal(out, want)


@gpu
@pytest.mark.parametrize("n,heads,prefix", [(2, (8, 2), 3000), (40, (28, 4), 3000), (128, (28, 1), 9000)])
def test_paged_splits_in_a_graph_and_on_another_stream(n, heads, prefix):
    """As above behind a prefix, whose parts are rows or tiles, with own lengths that change."""
    (Hq, Hkv), d, page, width = heads, 128, 16, 40
    need = P.slh_attend_paged_workspace(n, 1, Hq, Hkv, d, width * page, prefix)
    assert need > 0
    g = torch.Generator(device="cuda")
    g.manual_seed(n)
    n_pre = -(-prefix // page)
    kc, vc = (torch.randn(n_pre + n * width, Hkv, page, d, generator=g, device="cuda").to(BF) for _ in range(2))
    pre = torch.arange(n_pre, dtype=torch.int32, device="cuda")
    table = (n_pre + torch.arange(n * width, dtype=torch.int32, device="cuda")).view(n, width)
    lens = torch.full((n,), width * page, dtype=torch.int32, device="cuda")
    q = torch.randn(n, 1, Hq, d, generator=g, device="cuda").to(BF)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    out, lse = torch.empty_like(q), torch.empty(n, 1, Hq, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        P.slh_attend_paged(q, kc, vc, table, lens, pre, prefix, out=out, lse_out=lse, workspace=ws)
    side = torch.cuda.Stream()
    for a, b in _splits(width * page, width * page - 3):
        lens.copy_(torch.tensor([a if i % 2 else b for i in range(n)], dtype=torch.int32))
        q.copy_(torch.randn(n, 1, Hq, d, generator=g, device="cuda"))
        want_lse = torch.empty_like(lse)
        want = P.slh_attend_paged(q, kc, vc, table, lens, pre, prefix, lse_out=want_lse)
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, want_lse)
        for i in (0, 1):
            own = a if i % 2 else b
            at = (n_pre + i * width) * page
            kk, vv = (torch.cat([t[:prefix], t[at:at + own]]) for t in (x.permute(0, 2, 1, 3).reshape(-1, Hkv, d) for x in (kc, vc)))
            o, tol, e, etol = rows_of(q[i], kk, vv, [prefix + own], d ** -0.5)
            close(out[i], o, tol, f"{own} own keys")
            close_lse(lse[i], e, etol, f"{own} own keys")
        ws.fill_(255)
        out.fill_(7.0)
        side.wait_stream(torch.cuda.current_stream())
        P.slh_attend_paged(q, kc, vc, table, lens, pre, prefix, out=out, workspace=ws, stream=side)
        side.synchronize()
        assert torch.equal(out, want)


# ---------------------------------------------------------------- keys that are seen and weigh nothing
def _broken_key(k, head):
    """The element of every key of a head that makes its score with a query of ones there -inf."""
    k = k.clone()
    k[:, head, 3] = -math.inf
    return k


@gpu
@pytest.mark.parametrize("dt", [BF, HF])
@pytest.mark.parametrize("shape", PACKED)
def test_packed_rows_whose_keys_all_score_minus_infinity(shape, dt):
    """0 / 0 by the definition, so NaN, with lse -inf: not the zeros of a row that sees no key, which stay.  With one
    finite score among them such keys weigh nothing."""
    c = Packed(shape, 64, dt, True)
    c.q[:, :, 3] = 1.0
    head = c.Hkv - 1
    heads = slice(head * c.Hq // c.Hkv, c.Hq)
    want, want_lse = c.run()
    k = _broken_key(c.k, head)
    got, lse = c.run(k=k)
    for rq, rk, limit in c.sequences():
        blind = sum(x <= 0 for x in limit)
        assert not bool(got[rq.start:rq.start + blind].any())
        assert bool(torch.isnan(got[rq.start + blind:rq.stop, heads]).all())
        assert bool((lse[rq, heads] == -math.inf).all())
        got[rq, heads], lse[rq, heads] = want[rq, heads], want_lse[rq, heads]
    assert torch.equal(got, want) and torch.equal(lse, want_lse)
    rq, rk, limit = max(c.sequences(), key=lambda s: min(s[0].stop - s[0].start, s[1].stop - s[1].start))
    k[rk.start, head] = c.k[rk.start, head]                       # the one key of finite score
    got, lse = c.run(k=k)
    blind = sum(x <= 0 for x in limit)
    assert not bool(got[rq.start:rq.start + blind, heads].any())
    assert torch.equal(got[rq.start + blind:rq.stop, heads], c.v[rk.start, head].expand(len(limit) - blind, heads.stop - heads.start, 64))
    s = c.q[rq, heads].double() @ c.k[rk.start, head].double() / 8
    e = 2 * (64 + 8) * 2.0 ** -24 * (c.q[rq, heads].double().abs() @ c.k[rk.start, head].double().abs() / 8 + 1) + 9 * 2.0 ** -24 * (1 + s.abs())
    assert bool(((lse[rq, heads].double() - s).abs() <= e)[blind:].all())


@gpu
@pytest.mark.parametrize("dt", [BF, HF])
@pytest.mark.parametrize("shape", PAGED)
def test_paged_rows_whose_keys_all_score_minus_infinity(shape, dt):
    c = Paged(shape, 64, dt)
    c.q[..., 3] = 1.0
    head = c.Hkv - 1
    heads = slice(head * c.Hq // c.Hkv, c.Hq)
    want, want_lse = c.run()
    c.kc[:, head, :, 3] = -math.inf
    got, lse = c.run()
    limit = torch.tensor([[c.prefix + max(0, x - c.n_q + i + 1) for i in range(c.n_q)] for x in c.lens], device="cuda")
    broken = got[:, :, heads]
    assert bool(torch.isnan(broken[limit > 0]).all()) and not bool(broken[limit == 0].any())
    assert bool((lse[:, :, heads] == -math.inf).all())
    got[:, :, heads], lse[:, :, heads] = want[:, :, heads], want_lse[:, :, heads]
    assert torch.equal(got, want) and torch.equal(lse, want_lse)


# ---------------------------------------------------------------- light weights
LIGHT = 17.5                                      # exp(-17.5) = 2^-25.2


def light(d, keys):
    """Output of a row that sees `keys` of keys whose every 16th, the first among them, has the score 0 and the value
    0, the others the score -LIGHT and the value 1024; and its tolerance.

    A light weight is less than half the smallest step of fp16, 2^-24: it has to be raised before it is rounded.
    Raised by 2^7 its rounding is 2^-32 of a heavy one at most.  Besides, u of the output for its own rounding and u for
    the weights' where they are normal, half the smallest step of the output, and 2 (e + keys 2^-24) of the
    output for fp32 sums and scores that are off by e = 2 (d + 8) 2^-24 (LIGHT + 1)."""
    heavy = -(-keys // 16)
    w = (keys - heavy) * math.exp(-LIGHT)
    o = 1024 * w / (heavy + w)
    e = 2 * (d + 8) * 2.0 ** -24 * (LIGHT + 1)
    return o, 1.02 * (2 * 2.0 ** -11 * o + 1024 * 2.0 ** -32 * (keys - heavy) / heavy) + 2 * (e + keys * 2.0 ** -24) * o + 2.0 ** -25


def light_rows(n, d):
    """n keys and values as above."""
    k, v = torch.zeros(n, d, dtype=HF, device="cuda"), torch.full((n, d), 1024.0, dtype=HF, device="cuda")
    k[:, 0] = -LIGHT
    k[::16], v[::16] = 0.0, 0.0
    return k, v


def close_light(got, limit, d, what):
    for i, n in enumerate(limit):
        o, tol = light(d, n) if n > 0 else (0.0, 0.0)
        over = float((got[i].double() - o).abs().max())
        assert over <= tol, f"{what}, row {i} of {n} keys: {over:.3g} > {tol:.3g} of {o:.3g}"


@gpu
@pytest.mark.parametrize("d", SIZES)
@pytest.mark.parametrize("shape", PACKED)
def test_packed_light_weights_count_in_fp16(shape, d):
    c = Packed(shape, d, HF, True)
    c.scale = 1.0
    c.q.zero_()
    c.q[..., 0] = 1.0
    for _, rk, _ in c.sequences():
        c.k[rk], c.v[rk] = (x[:, None] for x in light_rows(rk.stop - rk.start, d))
    got, lse = c.run()
    for b, (rq, rk, limit) in enumerate(c.sequences()):
        some = list(range(0, len(limit), max(1, len(limit) // 40))) + [len(limit) - 1] * (len(limit) > 0)
        close_light(got[rq][some], [limit[i] for i in some], d, f"sequence {b}")
        for i in some:
            if limit[i] > 0:
                heavy = -(-limit[i] // 16)
                want = math.log(heavy + (limit[i] - heavy) * math.exp(-LIGHT))
                assert float((lse[rq][i].double() - want).abs().max()) <= 2 * (d + 8) * 2.0 ** -24 * (LIGHT + 1) + (limit[i] + 8) * 2.0 ** -24 * (1 + want)


@gpu
@pytest.mark.parametrize("d", SIZES)
@pytest.mark.parametrize("shape", PAGED)
def test_paged_light_weights_count_in_fp16(shape, d):
    c = Paged(shape, d, HF)
    c.scale = 1.0
    c.q.zero_()
    c.q[..., 0] = 1.0
    c.lens[:] = [x // 16 * 16 for x in c.lens]    # ratios as of whole sixteens, behind a prefix of whole sixteens
    c.prefix = c.prefix // 16 * 16
    c.len_.copy_(torch.tensor(c.lens))
    for pages, n in [(c.pre, c.prefix)] + [(c.table[b], c.lens[b]) for b in range(c.n)]:
        k, v = light_rows(n, d)
        at = torch.arange(n, device="cuda")
        c.kc[pages[at // c.page].long(), :, at % c.page], c.vc[pages[at // c.page].long(), :, at % c.page] = k[:, None], v[:, None]
    got, _ = c.run()
    for b in range(min(c.n, 5)):
        close_light(got[b], [c.prefix + max(0, c.lens[b] - c.n_q + i + 1) for i in range(c.n_q)], d, f"sequence {b}")
