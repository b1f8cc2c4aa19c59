"""One attention layer behind a compressed prompt: what an LLM does with the macro-tokens.

A document is compressed (slh_feature_map -> slh_lanczos -> slh_simhash -> slh_merge), its
macro-tokens go through a layer's projections, their queries and keys are normed and rotated at
the positions that the compression left them (increasing, with gaps), and the layer attends over
them (slh_qk_norm_rope, slh_attend).  Keys and values stay in a paged cache (slh_kv_append), and a batch of
questions is decoded token by token behind that prefix, which all of them share
(slh_kv_append, slh_attend_paged).

    python examples/answer_layer.py [workload] [questions] [tokens each]
"""
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2607_19368_amd as P  # noqa: E402
from paper_2607_19368_amd import slh as B  # noqa: E402

PAGE = 16
# query and key/value heads of 128 elements of the workloads' models
HEADS = {256: (2, 1), 3584: (28, 4), 4096: (32, 8), 5120: (40, 8)}


class Layer:
    """Projections and norms of one attention layer, with random weights."""

    def __init__(self, D, Hq, Hkv, d=128, n_pos=65536, seed=0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.Hq, self.Hkv, self.d = Hq, Hkv, d
        self.w = (torch.randn((D, (Hq + 2 * Hkv) * d), generator=g, device="cuda") / D ** 0.5).bfloat16()
        self.wq, self.wk = ((1 + 0.1 * torch.randn(d, generator=g, device="cuda")).bfloat16() for _ in range(2))
        self.table = P.slh_rope_table(n_pos, d)

    def project(self, x):
        """Queries, keys and values [T, heads, d] of hidden states x [T, D]: parts of one product."""
        qkv = (x.bfloat16() @ self.w).view(len(x), self.Hq + 2 * self.Hkv, self.d)
        return qkv[:, :self.Hq], qkv[:, self.Hq:self.Hq + self.Hkv], qkv[:, self.Hq + self.Hkv:]


def prefill(layer, E, pos, cache, pages):
    """Attention over a compressed prompt; its keys and values go to `pages` of the cache."""
    q, k, v = layer.project(E)
    q, k = P.slh_qk_norm_rope(q, k, layer.wq, layer.wk, table=layer.table, pos=pos, q_out=q, k_out=k)
    i = torch.arange(len(E), device=E.device)
    P.slh_kv_append(k, v, *cache, pages.long()[i // PAGE] * PAGE + i % PAGE)
    cu = torch.tensor([0, len(E)], dtype=torch.int32, device=E.device)
    return P.slh_attend(q, k, v, cu)


def decode(layer, x, pos, cache, table, lens, pages, M):
    """One new token of each question (hidden states x [B, D] at positions pos), behind the document.
    lens: own tokens so far; counted up."""
    q, k, v = layer.project(x)
    q, _ = P.slh_qk_norm_rope(q, q_weight=layer.wq, table=layer.table, pos=pos, q_out=q)
    at = lens.long()
    slots = table.gather(1, (at // PAGE)[:, None])[:, 0].long() * PAGE + at % PAGE
    P.slh_kv_append(k, v, *cache, slots, layer.wk, table=layer.table, pos=pos)
    lens += 1
    return P.slh_attend_paged(q, *cache, table, lens, pages, M)


def context(wl):
    """A context for prompts of a workload, with its windows, preserved suffix, operator and exact length."""
    ctx = P.slh_create(wl.N, wl.D, wl.m, wl.r, wl.bits, 0)
    for key, value in ((B.SLH_OPT_KEEP_LAST, wl.keep_last), (B.SLH_OPT_WINDOW_LEN, wl.window),
                       (B.SLH_OPT_NORMALIZE, int(wl.normalise)), (B.SLH_OPT_TARGET_LEN, wl.target)):
        if value:
            P.slh_set_option(ctx, key, value)
    return ctx


def run(X, ctx, n_it, layer, questions, rho=None):
    """Compresses X [N, D] (rho: routed, as P.compress), prefills the layer with its macro-tokens and decodes questions
    [n_seq, n, D].  Returns (E, positions, prefill output [M, Hq, d], decode outputs [n_seq, n, Hq, d])."""
    N = X.shape[0]
    E, pos, _, M, _ = P.compress(ctx, X, n_it, rho)
    n_seq, n, _ = questions.shape
    n_pre, n_own = -(-M // PAGE), -(-n // PAGE)
    cache = [torch.empty((n_pre + n_seq * n_own, layer.Hkv, PAGE, layer.d), dtype=torch.bfloat16, device=X.device) for _ in range(2)]
    pages = torch.arange(n_pre, dtype=torch.int32, device=X.device)
    table = (n_pre + torch.arange(n_seq * n_own, dtype=torch.int32, device=X.device)).view(n_seq, n_own)
    out = prefill(layer, E, pos, cache, pages)
    lens = torch.zeros(n_seq, dtype=torch.int32, device=X.device)
    steps = []
    for t in range(n):
        at = torch.full((n_seq,), N + t, dtype=torch.int32, device=X.device)     # behind the whole document
        steps.append(decode(layer, questions[:, t], at, cache, table, lens, pages, M))
    return E, pos, out, torch.stack(steps, 1)


def main():
    from workloads import make_inputs
    name = sys.argv[1] if len(sys.argv) > 1 else "qwen7b"
    n_seq = int(sys.argv[2]) if len(sys.argv) > 2 else 16
    n = int(sys.argv[3]) if len(sys.argv) > 3 else 8
    inp = make_inputs(name)
    wl = inp.workload
    X = torch.from_numpy(inp.X if inp.X.dtype == "float32" else inp.X.view("int16"))
    X = X.cuda() if X.dtype == torch.float32 else X.view(torch.bfloat16).cuda()
    ctx = context(wl)
    rho = wl.rho if wl.adaptive else None
    layer = Layer(wl.D, *HEADS[wl.D], n_pos=wl.N + n)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    questions = torch.randn((n_seq, n, wl.D), generator=g, device="cuda") * 0.02
    run(X, ctx, wl.n_it, layer, questions, rho)
    torch.cuda.synchronize()
    t = time.perf_counter()
    E, pos, out, steps = run(X, ctx, wl.n_it, layer, questions, rho)
    torch.cuda.synchronize()
    ms = (time.perf_counter() - t) * 1e3
    print(f"{name}: {wl.N} tokens -> {len(E)} macro-tokens at positions 0..{int(pos[-1])}; prefill {tuple(out.shape)}, "
          f"{n_seq} questions of {n} tokens {tuple(steps.shape)}: {ms:.2f} ms in all")


if __name__ == "__main__":
    main()
