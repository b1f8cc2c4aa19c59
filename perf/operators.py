"""The operators that follow a compressed prompt into an LLM's attention layers, as
measurable cases.

A prompt of N tokens leaves the package as M macro-tokens with increasing positions that
have gaps.  Its user's next steps, each through the package's entry points:

  qk      slh_qk_norm_rope: per-head RMS norm of queries and keys and the rotation at the
          macro-tokens' positions, in one pass
  append  slh_kv_append: new keys (normed, rotated) and values into a paged cache
  attend  slh_attend: causal attention of packed prompts of different lengths, with or
          without cached keys in front of the queries
  paged   slh_attend_paged: the new tokens of a batch against the paged cache, behind a
          prefix that all sequences share (one compressed document, many questions)

Heads are those of hidden widths 3584 (28 query, 4 key/value heads), 4096 (32, 8) and
5120 (40, 8) with 128 elements a head, and of width 256 (4, 4 with 64).  Where `own` is
false, run() computes the plain form: elementary operations in 32 bits, rounded once at
the end.  The rotation table, the cache, its pages and the output buffers are what a
user's program keeps.
"""
import math
import random

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
_EPS = 1e-6


def _case(name, op, **kw):
    c = {"name": name, "op": op, "type": "bf16", "Hq": 32, "Hkv": 8, "d": 128}
    c.update({"qk": {"T": 0, "rot": 128, "inter": False, "norm": True, "reach": 16},
              "append": {"T": 0, "B": 1, "rot": 128, "inter": False, "norm": True, "reach": 16, "page": 16},
              "attend": {"B": 1, "T": 0, "ctx": 0, "causal": True, "lse": False, "mix": 0},
              "paged": {"B": 1, "n_q": 1, "prefix": 0, "own": 0, "page": 16, "mix": 0}}[op])
    c.update(kw)
    return c


def listed():
    return [
        # the smallest call: one decode step of a small batch, launches and latency count
        _case("qk_step", "qk", T=24, reach=1),
        # a long prompt before compression, 28 heads: a large ordinary pass
        _case("qk_prompt", "qk", T=32768, Hq=28, Hkv=4, reach=1),
        # fp32 hidden states of an odd length, part of an 80-element head, interleaved, no norms
        _case("qk_partial_f32", "qk", T=5003, Hq=12, Hkv=12, d=80, rot=32, type="f32", inter=True, norm=False),
        # one decode step of a batch into the cache
        _case("append_step", "append", T=61, B=61, Hq=28, Hkv=4, reach=1),
        # compressed prompts written into 64-token pages after prefill
        _case("append_prompt", "append", T=16384, B=9, Hq=40, Hkv=8, page=64, type="f16"),
        # one compressed prompt: 8192 tokens at ratio 16
        _case("attend_macro", "attend", T=512, Hq=28, Hkv=4),
        # a batch of compressed prompts of many lengths, packed
        _case("attend_packed", "attend", B=23, T=12007, mix=1, lse=True),
        # a question after a cached document: few queries, many keys
        _case("attend_question", "attend", B=2, T=387, ctx=9001, Hq=40, Hkv=8, type="f16", mix=2),
        # the longest prompt: 16384 tokens at once
        _case("attend_prompt", "attend", T=16384, Hq=40, Hkv=8),
        # decode behind one compressed prompt, a small batch
        _case("paged_step", "paged", B=8, prefix=512, own=96, Hq=28, Hkv=4, mix=3),
        # many questions to one long document
        _case("paged_shared", "paged", B=128, prefix=32768, own=640, Hq=28, Hkv=4, page=64, mix=4),
        # a few long chats without a common prefix, two new tokens each
        _case("paged_long", "paged", B=6, n_q=2, own=49157, page=32, mix=5, type="f16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["qk", "append", "attend", "attend", "paged", "paged"])
    Hq, Hkv, d = rng.choice([(28, 4, 128), (32, 8, 128), (40, 8, 128), (4, 4, 64), (12, 12, 80)])
    c = _case("", op, Hq=Hq, Hkv=Hkv, d=d)
    del c["name"]
    c["type"] = rng.choice(["bf16", "bf16", "f16"])
    if op in ("qk", "append"):
        c["type"] = rng.choice(["bf16", "bf16", "f16", "f32"])
        c["T"] = _log(rng, 1, 32768 if op == "qk" else 16384)
        c["rot"] = 16 * rng.randint(1, d // 16) if rng.random() < 0.4 else d
        c["inter"] = rng.random() < 0.3
        c["norm"] = rng.random() < 0.6
        c["reach"] = rng.choice([1, 4, 16])
        if op == "append":
            c["B"] = min(c["T"], _log(rng, 1, 64))
            c["page"] = rng.choice([16, 32, 64, 128])
    elif op == "attend":
        c["mix"] = rng.randrange(1, 1000)
        c["lse"] = rng.random() < 0.3
        c["causal"] = rng.random() < 0.85
        c["T"] = _log(rng, 1, 12000)
        c["B"] = min(c["T"], rng.choice([1, 1, _log(rng, 2, 48)]))
        if rng.random() < 0.4:
            c["ctx"] = _log(rng, 1, 8192)
        longest = max(_lengths(c["B"], c["T"], c["mix"])) + c["ctx"]
        while c["B"] * Hq * longest * (longest - c["ctx"]) > 5 << 30:    # the plain form's scores
            c["T"] = c["T"] * 3 // 4
            c["ctx"] = c["ctx"] * 3 // 4
            c["B"] = min(c["B"], c["T"])
            longest = max(_lengths(c["B"], c["T"], c["mix"])) + c["ctx"]
    else:
        c["mix"] = rng.randrange(1, 1000)
        c["page"] = rng.choice([16, 32, 64, 128])
        c["B"] = _log(rng, 1, 128)
        c["n_q"] = rng.choice([1, 1, 1, 2, 3, 5])
        c["prefix"] = rng.choice([0, _log(rng, 16, 32768), _log(rng, 256, 32768)])
        c["own"] = _log(rng, 1, min(32768, max(16, 260000 // c["B"])))
    return c


def _lengths(n, total, mix):
    """n lengths of at least 1 that sum to total, spread over a factor of about 30."""
    r = random.Random(mix)
    w = [math.exp(r.uniform(0.0, 3.4)) for _ in range(n)]
    left, out = total - n, []
    for i in range(n):
        take = int(left * w[i] / sum(w[i:])) if i < n - 1 else left
        out.append(1 + take)
        left -= take
    return out


def _own_lengths(c):
    """Keys of each sequence's own, the new tokens included: up to c["own"] + n_q."""
    r = random.Random(c["mix"])
    return [c["n_q"] + int(c["own"] * (1.0 if b == 0 else r.uniform(0.05, 1.0))) for b in range(c["B"])]


def _table(n_pos, rot, device):
    f = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=device) / rot)
    a = torch.arange(n_pos, dtype=torch.float64, device=device)[:, None] * f
    return torch.stack([a.cos(), a.sin()], 1).float().contiguous()


def _positions(T, reach, g, dev):
    """Increasing positions with gaps of up to 2 reach - 1, as macro-tokens have them."""
    return (torch.randint(1, 2 * reach, (T,), generator=g, device=dev).cumsum(0) - 1).to(torch.int32)


def _rows(shape, g, dev, dt, spread=1.0):
    return (torch.randn(shape, generator=g, device=dev) * spread).to(dt)


def _keys(shape, g, dev, dt):
    """Keys share a mean over the tokens, as trained projections' do."""
    return (torch.randn(shape, generator=g, device=dev) + torch.randn((1,) * (len(shape) - 1) + shape[-1:], generator=g, device=dev)).to(dt)


def prepare(case, seed):
    c, dev = case, "cuda"
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    dt = _TYPES[c["type"]]
    Hq, Hkv, d = c["Hq"], c["Hkv"], c["d"]
    s = {"c": c, "scale": 1.0 / math.sqrt(d)}
    if c["op"] in ("qk", "append"):
        T = c["T"]
        # one projection's rows: queries, keys and values of a token side by side
        qkv = _rows((T, Hq + 2 * Hkv, d), g, dev, dt, 1.7)
        s["q"], s["k"], s["v"] = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
        s["wq"], s["wk"] = ((1.0 + 0.2 * torch.randn(d, generator=g, device=dev)).to(dt) if c["norm"] else None for _ in range(2))
        s["pos"] = _positions(T, c["reach"], g, dev)
        s["table"] = _table(T * (2 * c["reach"] - 1), c["rot"], dev)
        if c["op"] == "qk":
            s["q_out"] = torch.empty((T, Hq, d), dtype=dt, device=dev)
            s["k_out"] = torch.empty((T, Hkv, d), dtype=dt, device=dev)
        else:
            ps = c["page"]
            lens = _lengths(c["B"], T, 7)
            pages = [-(-(n + 5) // ps) for n in lens]       # each sequence continues 5 tokens into its first page
            order = torch.randperm(sum(pages), generator=g, device=dev)
            slots, at = [], 0
            for n, p in zip(lens, pages):
                i = torch.arange(5, 5 + n, device=dev)
                slots.append(order[at + i // ps] * ps + i % ps)
                at += p
            s["slots"] = torch.cat(slots)
            s["kc"], s["vc"] = (_rows((sum(pages), Hkv, ps, d), g, dev, dt) for _ in range(2))
    elif c["op"] == "attend":
        lq = _lengths(c["B"], c["T"], c["mix"])
        lk = [n + c["ctx"] for n in lq]
        s["q"] = _rows((sum(lq), Hq, d), g, dev, dt, 1.3)
        s["k"] = _keys((sum(lk), Hkv, d), g, dev, dt)
        s["v"] = _rows((sum(lk), Hkv, d), g, dev, dt)
        s["cu_q"], s["cu_k"] = (torch.tensor([0] + v, device=dev).cumsum(0).to(torch.int32) for v in (lq, lk))
        s["longest"] = (max(lq), max(lk))
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty((sum(lq), Hq), device=dev) if c["lse"] else None
    else:
        B, ps, P = c["B"], c["page"], c["prefix"]
        lens = _own_lengths(c)
        most, n_pre = -(-max(lens) // ps), -(-P // ps)
        used = [-(-n // ps) for n in lens]
        order = torch.randperm(n_pre + sum(used), generator=g, device=dev).to(torch.int32)
        s["prefix_pages"] = order[:n_pre].clone()
        s["page_table"] = torch.zeros((B, most), dtype=torch.int32, device=dev)
        at = n_pre
        for b, n in enumerate(used):
            s["page_table"][b, :n] = order[at:at + n]
            at += n
        s["lens"] = torch.tensor(lens, dtype=torch.int32, device=dev)
        s["kc"] = _keys((len(order), Hkv, ps, d), g, dev, dt)
        s["vc"] = _rows((len(order), Hkv, ps, d), g, dev, dt)
        s["q"] = _rows((B, c["n_q"], Hq, d), g, dev, dt, 1.3)
        s["out"] = torch.empty_like(s["q"])
    return s


# ---------------------------------------------------------------- the plain forms
def _norm_rope(x, w, table, pos, inter):
    """32-bit rows of x [T, H, d], normed and rotated."""
    x = x.float()
    if w is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + _EPS) * w.float()
    t = table[pos.long()][:, :, None]
    cos, sin = t[:, 0], t[:, 1]
    h = cos.shape[-1]
    a, b = (x[..., 0:2 * h:2], x[..., 1:2 * h:2]) if inter else (x[..., :h], x[..., h:2 * h])
    y = (a * cos - b * sin, b * cos + a * sin)
    y = torch.stack(y, -1).flatten(-2) if inter else torch.cat(y, -1)
    return torch.cat([y, x[..., 2 * h:]], -1)


def _weights(s, seen):
    """exp(s - max) over the last axis where `seen`, in place, and the sums and maxima."""
    s.masked_fill_(~seen, -math.inf)
    top = s.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    s.sub_(top).exp_()
    return s, s.sum(-1, keepdim=True), top


def _plain_attend(s):
    c, q, k, v = s["c"], s["q"], s["k"], s["v"]
    B, (Lq, Lk), Hkv, d = c["B"], s["longest"], c["Hkv"], c["d"]
    cq, ck = s["cu_q"].long(), s["cu_k"].long()
    nq, nk = cq.diff()[:, None], ck.diff()[:, None]
    i, j = torch.arange(Lq, device=q.device)[None], torch.arange(Lk, device=q.device)[None]
    at_q, at_k = (cq[:-1, None] + i).clamp(max=len(q) - 1), (ck[:-1, None] + j).clamp(max=len(k) - 1)
    g = c["Hq"] // Hkv
    qp = (q.float() * s["scale"])[at_q].view(B, Lq, Hkv, g, d).permute(0, 2, 3, 1, 4).reshape(B, Hkv, g * Lq, d)
    kp = k.float()[at_k].permute(0, 2, 3, 1).contiguous()
    vp = v.float()[at_k].permute(0, 2, 1, 3).contiguous()
    seen = (j < nk)[:, None, :] & ((j[:, None, :] <= (i + nk - nq)[:, :, None]) | (not c["causal"]))
    sc = torch.matmul(qp, kp).view(B, Hkv, g, Lq, Lk)
    del kp
    sc, total, top = _weights(sc, seen[:, None, None])
    o = torch.matmul(sc.view(B, Hkv, g * Lq, Lk), vp).view(B, Hkv, g, Lq, d)
    o = torch.where(total > 0, o / total, torch.zeros_like(o)).permute(0, 3, 1, 2, 4)
    lse = (total.log() + top)[..., 0].permute(0, 3, 1, 2)
    there = i < nq
    out = o[there].reshape(len(q), c["Hq"], d).to(q.dtype)
    return (out, lse[there].reshape(len(q), c["Hq"])) if c["lse"] else out


def _plain_paged(s):
    c, q = s["c"], s["q"]
    B, n_q, Hkv, d, P, ps = c["B"], c["n_q"], c["Hkv"], c["d"], c["prefix"], c["page"]
    g = c["Hq"] // Hkv
    qf = (q.float() * s["scale"]).view(B, n_q, Hkv, g, d).permute(2, 0, 3, 1, 4)       # [Hkv, B, g, n_q, d]
    n = s["page_table"].shape[1] * ps
    pages = s["page_table"].long()
    ko, vo = (t[pages].permute(2, 0, 1, 3, 4).reshape(Hkv, B, n, d).float() for t in (s["kc"], s["vc"]))
    own_s = torch.matmul(qf.reshape(Hkv, B, g * n_q, d), ko.transpose(-1, -2).contiguous()).view(Hkv, B, g, n_q, n)
    limit = s["lens"].long()[:, None] - n_q + 1 + torch.arange(n_q, device=q.device)    # [B, n_q]
    seen = (torch.arange(n, device=q.device) < limit[:, :, None])[None, :, None]
    first = s["prefix_pages"].long()
    kp, vp = (t[first].permute(1, 0, 2, 3).reshape(Hkv, -1, d)[:, :P].float() for t in (s["kc"], s["vc"]))
    pre_s = torch.matmul(qf.reshape(Hkv, B * g * n_q, d), kp.transpose(-1, -2).contiguous()).view(Hkv, B, g, n_q, P)
    sc = torch.cat([pre_s, own_s], -1)
    seen = torch.cat([torch.ones((1, B, 1, n_q, P), dtype=torch.bool, device=q.device), seen], -1)
    sc, total, _ = _weights(sc, seen)
    o = torch.matmul(sc[..., :P].reshape(Hkv, B * g * n_q, P), vp).view(Hkv, B, g, n_q, d)
    o += torch.matmul(sc[..., P:].reshape(Hkv, B, g * n_q, n), vo).view(Hkv, B, g, n_q, d)
    o = torch.where(total > 0, o / total, torch.zeros_like(o))
    return o.permute(1, 3, 0, 2, 4).reshape(q.shape).to(q.dtype)


def _plain_append(s):
    c, ps = s["c"], s["c"]["page"]
    k = _norm_rope(s["k"], s["wk"], s["table"], s["pos"], c["inter"]).to(s["k"].dtype)
    page, at = s["slots"] // ps, s["slots"] % ps
    s["kc"][page, :, at] = k
    s["vc"][page, :, at] = s["v"]
    return s["kc"], s["vc"]


def run(state):
    s, c = state, state["c"]
    op = c["op"]
    if not own:
        if op == "qk":
            return tuple(_norm_rope(s[x], s["w" + x], s["table"], s["pos"], c["inter"]).to(s[x].dtype) for x in ("q", "k"))
        return {"append": _plain_append, "attend": _plain_attend, "paged": _plain_paged}[op](s)
    import paper_2607_19368_amd as P
    if op == "qk":
        return P.slh_qk_norm_rope(s["q"], s["k"], q_weight=s["wq"], k_weight=s["wk"], eps=_EPS, table=s["table"],
                                  pos=s["pos"], interleaved=c["inter"], q_out=s["q_out"], k_out=s["k_out"])
    if op == "append":
        P.slh_kv_append(s["k"], s["v"], s["kc"], s["vc"], s["slots"], k_weight=s["wk"], eps=_EPS, table=s["table"],
                        pos=s["pos"], interleaved=c["inter"])
        return s["kc"], s["vc"]
    if op == "attend":
        out = P.slh_attend(s["q"], s["k"], s["v"], s["cu_q"], s["cu_k"], scale=s["scale"], causal=c["causal"],
                           out=s["out"], lse_out=s["lse"])
        return (out, s["lse"]) if c["lse"] else out
    return P.slh_attend_paged(s["q"], s["kc"], s["vc"], s["page_table"], s["lens"], prefix_pages=s["prefix_pages"],
                              prefix_len=c["prefix"], scale=s["scale"], out=s["out"])


# ---------------------------------------------------------------- what a pass has to do
def _pairs(nq, nk, causal):
    """Visible (query, key) pairs of one sequence and head."""
    if not causal:
        return nq * nk
    low = max(0, nq - nk)                      # queries that see nothing
    n = nq - low
    return n * (nk - nq + low + 1) + n * (n - 1) // 2


def work(case):
    c = case
    e = 4 if c["type"] == "f32" else 2
    Hq, Hkv, d = c["Hq"], c["Hkv"], c["d"]
    if c["op"] in ("qk", "append"):
        heads = Hq + Hkv if c["op"] == "qk" else 2 * Hkv
        turned = Hq + Hkv if c["op"] == "qk" else Hkv
        return {"bytes": c["T"] * (2 * heads * d * e + 4 * c["rot"] + (4 if c["op"] == "qk" else 12)),
                "flops": c["T"] * turned * (3 * c["rot"] + (4 * d if c["norm"] else 0))}
    if c["op"] == "attend":
        lq = _lengths(c["B"], c["T"], c["mix"])
        lk = [n + c["ctx"] for n in lq]
        return {"bytes": 2 * e * d * (Hq * sum(lq) + Hkv * sum(lk)) + (4 * Hq * sum(lq) if c["lse"] else 0),
                "flops": 4 * d * Hq * sum(_pairs(a, b, c["causal"]) for a, b in zip(lq, lk))}
    lens = _own_lengths(c)
    keys = c["prefix"] + sum(lens)
    return {"bytes": 2 * e * d * (Hkv * keys + Hq * c["B"] * c["n_q"]),
            "flops": 4 * d * Hq * sum(c["n_q"] * c["prefix"] + _pairs(c["n_q"], n, True) for n in lens)}


# ---------------------------------------------------------------- the definition in 64 bits
def _exact_rows(x, w, pos, c):
    """Each pair (a, b) as the complex number a + i b, turned by exp(i p f)."""
    x = x.double()
    if w is not None:
        x = x / ((x ** 2).sum(-1, keepdim=True) / x.shape[-1] + _EPS).sqrt() * w.double()
    rot, y = c["rot"], x.clone()
    # the angles' table is an input of the operator, in 32 bits
    f = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=x.device) / rot)
    ang = pos.double()[:, None, None] * f
    turn = torch.complex(ang.cos().float().double(), ang.sin().float().double())
    at = (slice(0, rot, 2), slice(1, rot, 2)) if c["inter"] else (slice(0, rot // 2), slice(rot // 2, rot))
    z = torch.complex(x[..., at[0]].contiguous(), x[..., at[1]].contiguous()) * turn
    y[..., at[0]], y[..., at[1]] = z.real, z.imag
    return y


def _exact_attention(q, k, v, scale, limit):
    """q [n, d] against k, v [m, d]; row i sees the first limit[i] keys."""
    s = (q @ k.T) * scale
    s = s.masked_fill(torch.arange(len(k), device=q.device)[None] >= limit[:, None], -math.inf)
    lse = torch.logsumexp(s, -1)
    p = torch.exp(s - torch.where(lse == -math.inf, torch.zeros_like(lse), lse)[:, None])
    return p @ v, lse


def exact(case, seed):
    c = case
    s = prepare(case, seed)
    Hq, Hkv, d = c["Hq"], c["Hkv"], c["d"]
    g = Hq // Hkv
    if c["op"] == "qk":
        return tuple(_exact_rows(s[x], s["w" + x], s["pos"], c) for x in ("q", "k"))
    if c["op"] == "append":
        kc, vc = s["kc"].double(), s["vc"].double()
        flat = [t.permute(0, 2, 1, 3).reshape(-1, Hkv, d) for t in (kc, vc)]
        flat[0][s["slots"]] = _exact_rows(s["k"], s["wk"], s["pos"], c)
        flat[1][s["slots"]] = s["v"].double()
        return tuple(t.view(-1, c["page"], Hkv, d).permute(0, 2, 1, 3).contiguous() for t in flat)
    if c["op"] == "attend":
        out = torch.zeros(s["q"].shape, dtype=torch.float64, device=s["q"].device)
        lse = torch.zeros(s["q"].shape[:2], dtype=torch.float64, device=s["q"].device)
        cq, ck = s["cu_q"].tolist(), s["cu_k"].tolist()
        for b in range(c["B"]):
            nq, nk = cq[b + 1] - cq[b], ck[b + 1] - ck[b]
            limit = torch.arange(nq, device=out.device) + nk - nq + 1 if c["causal"] else torch.full((nq,), nk, device=out.device)
            for h in range(Hq):
                k, v = (s[x][ck[b]:ck[b + 1], h // g].double() for x in ("k", "v"))
                for r in range(0, nq, 8192):
                    rows = slice(cq[b] + r, min(cq[b + 1], cq[b] + r + 8192))
                    o, t = _exact_attention(s["q"][rows, h].double(), k, v, s["scale"], limit[r:r + 8192])
                    out[rows, h], lse[rows, h] = o, t
        return (out, lse) if c["lse"] else out
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=s["q"].device)
    ps = c["page"]
    for b, n in enumerate(_own_lengths(c)):
        pages = torch.cat([s["prefix_pages"], s["page_table"][b, :-(-n // ps)]]).long()
        keep = torch.ones(len(pages) * ps, dtype=torch.bool, device=out.device)
        n_pre = len(s["prefix_pages"]) * ps
        keep[c["prefix"]:n_pre] = False
        keep[n_pre + n:] = False
        limit = c["prefix"] + n - c["n_q"] + 1 + torch.arange(c["n_q"], device=out.device)
        for h in range(Hkv):
            k, v = (t[pages, h].reshape(-1, d)[keep].double() for t in (s["kc"], s["vc"]))
            q = s["q"][b, :, h * g:(h + 1) * g].reshape(-1, d).double()
            o, _ = _exact_attention(q, k, v, s["scale"], limit.repeat_interleave(g))
            out[b, :, h * g:(h + 1) * g] = o.view(c["n_q"], g, d)
    return out
