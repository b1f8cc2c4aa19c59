"""The attention layer behind a compressed prompt with a smaller cache (examples/answer_layer.py: run_small): what it gives against
the definition in 64 bits, on the keys and values that its cache holds at each step."""
import os
import sys

import pytest
import torch

import attention_plain as AP
import cache_plain as CP
import paper_2607_19368_amd as P
import parity as PR
from workloads import make_inputs

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import answer_layer as AL  # noqa: E402

pytestmark = pytest.mark.gpu


def test_answers_from_a_small_cache(monkeypatch):
    inp = make_inputs("tiny")
    wl = inp.workload
    n_seq, n, budget, own_budget = 3, 21, 24, 6
    layer = AL.Layer(wl.D, 4, 2, n_pos=wl.N + n)
    ctx = P.slh_create(wl.N, wl.D, wl.m, wl.r, wl.bits, 0)
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    asked = torch.randn((n_seq, n, wl.D), generator=g, device="cuda")
    seen, evicted = [], []
    attend, evict = P.slh_attend_paged_e4m3, P.slh_kv_evict

    def watch(q, kc, vc, ks, vs, table, lens, pages, M, **kw):
        out = attend(q, kc, vc, ks, vs, table, lens, pages, M, **kw)
        seen.append([x.cpu() for x in (q, CP.values(kc.cpu(), ks.cpu()), CP.values(vc.cpu(), vs.cpu()), table, lens, pages, out)] + [M])
        return out

    def watch_evict(kc, vc, weights, table, lens, keep, first, last, *rest, **kw):
        had = weights.cpu().clone(), lens.tolist()
        got = evict(kc, vc, weights, table, lens, keep, first, last, *rest, **kw)
        evicted.append((*had, keep, first, last, got[2].cpu()))
        return got

    monkeypatch.setattr(P, "slh_attend_paged_e4m3", watch)
    monkeypatch.setattr(P, "slh_kv_evict", watch_evict)
    E, pos, M, out, steps = AL.run_small(PR.to_device_x(inp), ctx, wl.n_it, layer, asked, budget, own_budget)
    assert len(E) > budget == M and out.shape == (len(E), 4, 128) and steps.shape == (n_seq, n, 4, 128)
    for q, K, V, table, lens, pages, got, m in seen:
        for b in range(n_seq):
            kk, vv = (torch.cat([x[pages.long()].transpose(1, 2).flatten(0, 1)[:m],
                                 x[table[b].long()].transpose(1, 2).flatten(0, 1)[:int(lens[b])]]) for x in (K, V))
            o, tol, _, _ = AP.attend(q[b:b + 1], kk, vv, [len(kk)], 128 ** -0.5)
            assert bool(((got[b].double() - o[0]).abs() <= tol[0]).all())
    # the document once, the questions' own tokens at the steps that fill their room
    assert [x[2] for x in evicted] == [budget] + [own_budget] * ((n - own_budget) // own_budget)
    for w, lens, keep, first, last, kept in evicted:
        for b, m in enumerate(lens):
            for h in range(2):
                assert kept[b, h].tolist() == CP.keep(w[b, h].tolist(), m, keep, first, last)


def test_a_budget_for_everything_evicts_nothing():
    inp = make_inputs("tiny")
    wl = inp.workload
    layer = AL.Layer(wl.D, 4, 2, n_pos=wl.N + 9)
    ctx = P.slh_create(wl.N, wl.D, wl.m, wl.r, wl.bits, 0)
    asked = torch.randn((2, 9, wl.D), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    X = PR.to_device_x(inp)
    E, pos, out, steps = AL.run(X, ctx, wl.n_it, layer, asked)
    E8, pos8, M, out8, steps8 = AL.run_small(X, ctx, wl.n_it, layer, asked, 10 ** 6, 10 ** 6)
    assert torch.equal(E, E8) and torch.equal(pos, pos8) and M == len(E) and torch.equal(out, out8)
    assert steps8.shape == steps.shape and bool(torch.isfinite(steps8).all())


def test_answers_in_8_bits_are_those_in_16(monkeypatch):
    """Without eviction both caches hold the same rows in the same places, up to the codes' rounding, and the answers in 8 bits are
    the definition's on what is held, at every step."""
    inp = make_inputs("tiny")
    wl = inp.workload
    n_seq, n, Hkv = 2, 19, 2
    layer = AL.Layer(wl.D, 4, Hkv, n_pos=wl.N + n)
    ctx = P.slh_create(wl.N, wl.D, wl.m, wl.r, wl.bits, 0)
    asked = torch.randn((n_seq, n, wl.D), generator=torch.Generator(device="cuda").manual_seed(5), device="cuda")
    X = PR.to_device_x(inp)
    seen = {"slh_attend_paged": [], "slh_attend_paged_e4m3": []}

    def watch(name):
        real = getattr(P, name)

        def call(q, *args, **kw):
            out = real(q, *args, **kw)
            *cache, table, lens, pages, M = args
            seen[name].append((q.cpu(), [c.cpu() for c in cache], table.cpu(), lens.tolist(), pages.cpu(), M, out.cpu()))
            return out
        monkeypatch.setattr(P, name, call)

    for name in seen:
        watch(name)
    monkeypatch.setattr(P, "slh_kv_evict", lambda *a, **kw: pytest.fail("a budget for everything evicts nothing"))
    AL.run(X, ctx, wl.n_it, layer, asked)
    _, _, M, _, steps = AL.run_small(X, ctx, wl.n_it, layer, asked, 10 ** 6, 10 ** 6)
    both = list(zip(*seen.values()))
    assert len(both) == n
    for t, (a, b) in enumerate(both):
        assert torch.equal(a[0], b[0]) and torch.equal(a[2], b[2]) and a[3] == b[3] == [t + 1] * n_seq
        assert torch.equal(a[4], b[4]) and a[5] == b[5] == M
        kc, vc, ks, vs = b[1]
        held = CP.values(kc, ks), CP.values(vc, vs)
        for x16, x8, two in zip(a[1], held, (ks, vs)):
            power = torch.pow(2.0, CP.bytes_of(two).double() - 127).repeat_interleave(kc.shape[2] // two.shape[2], -1)[..., None]
            # the 16-bit row is within 2^-8 of the exact one, which the code was within 2^-4 of, or, as a subnormal one, within 2^-10 of the power;
            # rescaled as its block grew, within twice that
            off = (x8 - x16.double()).abs() - x16.double().abs() * (2.0 ** -4 + 2.0 ** -8) * (1 + 2.0 ** -7) - 2.0 ** -9 * power
            for pages, rows in [(b[4], M)] + [(b[2][s], t + 1) for s in range(n_seq)]:
                at = off[pages.long()].transpose(1, 2).flatten(0, 1)[:rows]
                assert float(at.max()) <= 0, t
        for s in range(n_seq):
            kk, vv = (torch.cat([x[b[4].long()].transpose(1, 2).flatten(0, 1)[:M], x[b[2][s].long()].transpose(1, 2).flatten(0, 1)[:t + 1]]) for x in held)
            o, tol, _, _ = AP.attend(b[0][s:s + 1], kk, vv, [len(kk)], 128 ** -0.5)
            assert bool(((b[6][s].double() - o[0]).abs() <= tol[0]).all()), (t, s)
            assert torch.equal(b[6][s], steps[s, t].cpu())
