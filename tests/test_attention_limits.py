"""The operators behind a compressed prompt at the limits that the library states (include/slh.h)."""
import pytest
import torch

import paper_2607_19368_amd as P
from paper_2607_19368_amd import slh as B

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
