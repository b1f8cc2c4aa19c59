"""What the attention operators' binding takes and refuses (attention.py)."""
import pytest
import torch

import paper_2607_19368_amd as P

gpu = pytest.mark.gpu
BF = torch.bfloat16


def _calls():
    """{name: (call, its tensors of numbers)}"""
    g = torch.Generator(device="cuda")
    g.manual_seed(1)

    def rows(*shape):
        return torch.randn(shape, generator=g, device="cuda").to(BF)

    cu = torch.tensor([0, 4], dtype=torch.int32, device="cuda")
    slots = torch.arange(4, device="cuda")
    pages, lens = torch.zeros(4, 1, dtype=torch.int32, device="cuda"), torch.ones(4, dtype=torch.int32, device="cuda")
    pos = torch.arange(4, dtype=torch.int32, device="cuda")
    table = P.slh_rope_table(8, 64)
    return {
        "norm": (lambda q, k, wq, wk, t: P.slh_qk_norm_rope(q, k, wq, wk, table=t, pos=pos)[1],
                 [rows(4, 2, 64), rows(4, 2, 64), rows(64), rows(64), table]),
        "append": (lambda k, v, w, kc, vc: P.slh_kv_append(k, v, kc, vc, slots, w)[0],
                   [rows(4, 2, 64), rows(4, 2, 64), rows(64), rows(2, 2, 16, 64), rows(2, 2, 16, 64)]),
        "attend": (lambda q, k, v, out: P.slh_attend(q, k, v, cu, out=out),
                   [rows(4, 2, 64), rows(4, 2, 64), rows(4, 2, 64), rows(4, 2, 64)]),
        "paged": (lambda q, kc, vc, out: P.slh_attend_paged(q, kc, vc, pages, lens, out=out),
                  [rows(4, 2, 64), rows(2, 2, 16, 64), rows(2, 2, 16, 64), rows(4, 2, 64)]),
    }


@gpu
@pytest.mark.parametrize("name", ["norm", "append", "attend", "paged"])
def test_gradients_are_refused_and_not_lost(name):
    call, tensors = _calls()[name]
    want = call(*tensors).clone()
    for i in range(len(tensors)):
        with_grad = [t.clone().requires_grad_() if j == i else t for j, t in enumerate(tensors)]
        with pytest.raises(P.SLHError, match="gradient"):
            call(*with_grad)
        with torch.no_grad():
            assert torch.equal(call(*with_grad), want)


@gpu
@pytest.mark.parametrize("T,H", [(1, 4), (5, 1), (1, 1)])
@pytest.mark.parametrize("odd", [7, 2 ** 25 + 8])
def test_strides_of_dimensions_of_one_do_not_matter(T, H, odd):
    """A single token or head of a large buffer: its stride may be anything, unaligned or past the limit."""
    def same(x):
        return x.as_strided(x.shape, [odd if n == 1 else s for n, s in zip(x.shape, x.stride())])

    g = torch.Generator(device="cuda")
    g.manual_seed(T)
    q, k, v, out = (torch.randn(T, H, 64, generator=g, device="cuda").to(BF) for _ in range(4))
    w = torch.ones(64, dtype=BF, device="cuda")
    cu = torch.tensor([0, T], dtype=torch.int32, device="cuda")
    for a, b in zip(P.slh_qk_norm_rope(same(q), same(k), w, w, q_out=same(out)), P.slh_qk_norm_rope(q, k, w, w)):
        assert torch.equal(a, b)
    assert torch.equal(P.slh_attend(same(q), same(k), same(v), cu, out=same(out)), P.slh_attend(q, k, v, cu))
    slots = torch.arange(T, device="cuda")
    caches = [[torch.zeros(1, H, 16, 64, dtype=BF, device="cuda") for _ in range(2)] for _ in range(2)]
    P.slh_kv_append(same(k), same(v), *caches[0], slots)
    P.slh_kv_append(k, v, *caches[1], slots)
    assert torch.equal(caches[0][0], caches[1][0]) and torch.equal(caches[0][1], caches[1][1])
    pages, lens = torch.zeros(1, 1, dtype=torch.int32, device="cuda"), torch.tensor([T], dtype=torch.int32, device="cuda")
    assert torch.equal(P.slh_attend_paged(same(q[None]), *caches[1], pages, lens, out=same(out[None])),
                       P.slh_attend_paged(q[None], *caches[1], pages, lens))
    if T == 1:
        assert torch.equal(P.slh_attend_paged(same(q), *caches[1], pages, lens), P.slh_attend_paged(q, *caches[1], pages, lens))
