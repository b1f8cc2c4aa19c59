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
