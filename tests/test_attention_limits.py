"""The operators behind a compressed prompt at the limits that the library states (include/slh.h)."""
import pytest
import torch

import paper_2607_19368_amd as P
from paper_2607_19368_amd import slh as B
from test_attention_paths import close, rows_of

gpu = pytest.mark.gpu


def test_tables_past_a_launch_are_refused():
    """A launch has fewer than 2^32 threads, each of one cosine and sine."""
    lib = B.load()
    p = 4096                                      # an aligned address that nothing reads
    for n, rot in ((2 ** 26, 128), (2 ** 31, 256), (2 ** 29, 16), (2 ** 29 - 1, 16), ((2 ** 32 - 256) // 40 + 1, 80)):
        assert lib.slh_rope_table(p, n, rot, 1e4, 0, 1.0, 0, 32.0, 1.0, None) == B.SLH_EINVAL, (n, rot)


@gpu
def test_a_table_at_the_limit():
    n, rot = 2 ** 29 - 32, 16
    table = P.slh_rope_table(n, rot)
    f = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    for p in (0, 1, n // 2, n - 1):
        a = p * f
        assert float((table[p].cpu().double() - torch.stack([a.cos(), a.sin()])).abs().max()) <= 2.0 ** -24 + n * 2.0 ** -51, p


@gpu
def test_partial_results_of_more_rows_than_a_launch_has_threads_for():
    """2^26 rows, a wave each, are 2^32 threads."""
    n, Hq, d, page, prefix = 2 ** 16, 1024, 64, 16, 600
    assert P.slh_attend_paged_workspace(n, 1, Hq, 1, d, page, prefix) >= 2 * n * Hq * (4 * d + 8)
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    n_pre = -(-prefix // page)
    kc, vc = (torch.randn(n_pre + n, 1, page, d, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    q = torch.randn(1, 1024, d, generator=g, device="cuda").to(torch.bfloat16).repeat(n, 1, 1)
    table = (n_pre + torch.arange(n, dtype=torch.int32, device="cuda"))[:, None]
    lens = (torch.arange(n, dtype=torch.int32, device="cuda") % page) + 1
    pre = torch.arange(n_pre, dtype=torch.int32, device="cuda")
    lse = torch.full((n, Hq), 7.0, device="cuda")
    out = P.slh_attend_paged(q, kc, vc, table, lens, pre, prefix, lse_out=lse)
    shared = [x[:n_pre, 0].reshape(-1, 1, d)[:prefix] for x in (kc, vc)]
    for b in (0, 1, n // 2 - 1, n // 2, n // 2 + 1, n - 2, n - 1):
        k, v = (torch.cat([s, x[n_pre + b, 0, :int(lens[b]), None]]) for s, x in zip(shared, (kc, vc)))
        o, tol, e, etol = rows_of(q[b:b + 1], k, v, [len(k)], d ** -0.5)
        close(out[b:b + 1], o, tol, f"sequence {b}")
        assert bool(((lse[b:b + 1].double() - e).abs() <= etol).all())


# ---------------------------------------------------------------- what lies in device memory
@gpu
@pytest.mark.parametrize("lk", [60, 5000])         # in one piece, and with the keys split
def test_sequence_bounds_outside_the_tensors_are_taken_as_the_nearest(lk):
    g = torch.Generator(device="cuda")
    g.manual_seed(lk)
    q, k, v = (torch.randn(n, h, 64, generator=g, device="cuda").to(torch.bfloat16) for n, h in ((20, 4), (lk, 2), (lk, 2)))

    def run(cq, ck):
        out, lse = torch.full_like(q, 7.0), torch.full((20, 4), 7.0, device="cuda")
        P.slh_attend(q, k, v, *(torch.tensor(x, dtype=torch.int32, device="cuda") for x in (cq, ck)), out=out, lse_out=lse)
        return out, lse

    low, high = -2 ** 31, 2 ** 31 - 1
    for cq, ck in (([low, 7, high], [-1, 31, lk + 1]), ([-3, 20, 21], [low, lk + 9, high]), ([0, 9, 20], [low, low, high])):
        near = [[min(max(x, 0), n) for x in c] for c, n in ((cq, 20), (ck, lk))]
        for a, b in zip(run(cq, ck), run(*near)):
            assert torch.equal(a, b)


@gpu
@pytest.mark.parametrize("n,n_q,prefix", [(3, 1, 40), (3, 2, 0), (3, 2, 3000), (40, 3, 3000)])
def test_lengths_and_pages_outside_the_cache(n, n_q, prefix):
    """Lengths are taken as the nearest that the table has room for; a page that is none spoils its own sequence alone; a
    table without columns is one of lengths 0."""
    g = torch.Generator(device="cuda")
    g.manual_seed(n + prefix)
    page, width, Hq, Hkv, d = 16, 5, 28, 4, 64
    n_pre = -(-prefix // page)
    kc, vc = (torch.randn(n_pre + n * width, Hkv, page, d, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    pre = torch.arange(n_pre, dtype=torch.int32, device="cuda")
    table = (n_pre + torch.arange(n * width, dtype=torch.int32, device="cuda")).view(n, width)
    q = torch.randn(n, n_q, Hq, d, generator=g, device="cuda").to(torch.bfloat16)

    def run(lens, table=table):
        lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
        return P.slh_attend_paged(q, kc, vc, table, lens, pre, prefix)

    most = page * width
    lens = [(17 * b) % most for b in range(n)]
    assert torch.equal(run([2 ** 31 - 1, -2 ** 31, -1] + lens[3:]), run([most, 0, 0] + lens[3:]))
    want = run(lens)
    for wrong in (-1, -2 ** 31, 2 ** 31 - 1, len(kc)):
        spoiled = table.clone()
        spoiled[1, 0] = wrong
        got = run(lens, spoiled)
        assert torch.equal(got[0], want[0]) and torch.equal(got[2:], want[2:])
    got = run([0] * n, table[:, :0])
    for b in range(0, n, 7):
        o, tol, _, _ = rows_of(q[b], *(x[:n_pre].permute(0, 2, 1, 3).reshape(-1, Hkv, d)[:prefix] for x in (kc, vc)), [prefix] * n_q, d ** -0.5)
        close(got[b], o, tol, f"sequence {b}")
