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
