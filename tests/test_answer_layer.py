"""The attention layer behind a compressed prompt (examples/answer_layer.py): prefill and decode
outputs against the definition in 64 bits, on the keys and values that the layer's own projections give."""
import os
import sys

import pytest
import torch

import attention_plain as AP
import paper_2607_19368_amd as P
import parity as PR
from workloads import make_inputs

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import answer_layer as AL  # noqa: E402

pytestmark = pytest.mark.gpu


def test_answers_behind_a_compressed_prompt():
    inp = make_inputs("tiny")
    wl = inp.workload
    B, n = 5, 19                                  # own keys end inside their second page
    layer = AL.Layer(wl.D, 4, 2, n_pos=wl.N + n)
    ctx = P.slh_create(wl.N, wl.D, wl.m, wl.r, wl.bits, 0)
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    asked = torch.randn((B, n, wl.D), generator=g, device="cuda")
    E, pos, out, steps = AL.run(PR.to_device_x(inp), ctx, wl.n_it, layer, asked)
    M = len(E)
    assert 1 < M < wl.N and out.shape == (M, 4, 128) and steps.shape == (B, n, 4, 128)
    assert bool((pos[1:] > pos[:-1]).all())

    def rows(x, at):
        q, k, v = layer.project(x)
        q, k = P.slh_qk_norm_rope(q, k, layer.wq, layer.wk, table=layer.table, pos=at)
        return q.cpu(), k.cpu(), v.cpu()

    q, k, v = rows(E, pos)
    scale = 128 ** -0.5
    o, tol, _, _ = AP.attend(q, k, v, range(1, M + 1), scale)
    assert bool(((out.double().cpu() - o).abs() <= tol).all())
    for b in range(B):
        for t in (0, 1, 15, 16, n - 1):
            # the step's own projection of one row a question, as decode makes it
            own = [rows(asked[:, i], torch.full((B,), wl.N + i, dtype=torch.int32, device="cuda")) for i in range(t + 1)]
            kk = torch.cat([k] + [r[1][b:b + 1] for r in own])
            vv = torch.cat([v] + [r[2][b:b + 1] for r in own])
            o, tol, _, _ = AP.attend(own[t][0][b:b + 1], kk, vv, [M + t + 1], scale)
            assert bool(((steps[b, t].double().cpu() - o[0]).abs() <= tol[0]).all()), (b, t)


@pytest.mark.parametrize("name", ["local16", "qwen7b_exact"])
def test_workloads_are_run_with_their_options(name):
    """Windows, preserved suffix and exact length are the workload's."""
    inp = make_inputs(name)
    wl = inp.workload
    ctx = AL.context(wl)
    layer = AL.Layer(wl.D, *AL.HEADS[wl.D], n_pos=wl.N + 1)
    asked = torch.zeros((2, 1, wl.D), device="cuda")
    E, pos, out, _ = AL.run(PR.to_device_x(inp), ctx, wl.n_it, layer, asked)
    assert len(out) == len(E) == len(pos)
    if wl.target:
        assert len(E) == wl.target
    if wl.window:
        assert ctx.n_windows == (wl.N - wl.keep_last) // wl.window and len(E) >= ctx.n_windows + wl.keep_last
        assert pos[-wl.keep_last:].tolist() == list(range(wl.N - wl.keep_last, wl.N))
