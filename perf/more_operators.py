"""The operators of a smaller cache behind a compressed prompt, as measurable cases.

A user who decodes behind a compressed prompt (perf/operators.py) keeps the keys and values of what is
not compressed, and of the macro-tokens, in a paged cache.  Two things make it smaller, each through
the package's entry points:

  append   slh_kv_append_e4m3: new keys (normed, rotated) and values into a cache held in 8 bits, e4m3
           codes with a power of two for each block of rows and head; a block that grows keeps
           its earlier rows
  paged    slh_attend_paged_e4m3: the new tokens of a batch against that cache, behind a prefix
           that all sequences share
  weights  slh_attend_weights: the attention weight that each cached key received from a call's
           queries, added up by key and key/value head
  evict    slh_kv_evict: of each sequence and head the rows with the most weight stay, beside the
           first and the last ones, and move together in their order

Heads are those of hidden widths 3584 (28 query, 4 key/value heads), 4096 (32, 8) and 5120 (40, 8) with
128 elements a head, and of width 256 (4, 4 with 64).  Where `own` is false, run() computes the
plain form: elementary operations in 32 bits, in 64 where codes are chosen, rounded once at the end.
The rotation table, the cache, its pages and the buffers of results are what a user's program keeps.
"""
import math
import random

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
_EPS = 1e-6


def _case(name, op, **kw):
    c = {"name": name, "op": op, "type": "bf16", "Hq": 32, "Hkv": 8, "d": 128, "page": 16, "B": 1, "mix": 0}
    c.update({"append": {"T": 0, "own": 0, "block": 16, "rot": 128, "inter": False, "norm": True, "reach": 16},
              "paged": {"n_q": 1, "prefix": 0, "own": 0, "block": 16},
              "weights": {"T": 0, "own": 0, "block": 0},            # block 0: a cache in the inputs' type
              "evict": {"own": 0, "budget": 0, "first": 0, "last": 0, "block": 0}}[op])
    c.update(kw)
    return c


def listed():
    return [
        # one decode step of a batch into the cache: launches and latency count
        _case("append_step", "append", T=61, B=61, own=640, Hq=28, Hkv=4, page=64, block=64, mix=1),
        # compressed prompts written after prefill, behind a few rows that are there
        _case("append_prompt", "append", T=16384, B=9, own=21, Hq=40, Hkv=8, page=64, type="f16", mix=2),
        # decode behind one compressed prompt, a small batch
        _case("paged_step", "paged", B=8, prefix=512, own=96, Hq=28, Hkv=4, mix=3),
        # many questions to one long document
        _case("paged_shared", "paged", B=128, prefix=32768, own=640, Hq=28, Hkv=4, page=64, block=64, mix=4),
        # a few long chats without a common prefix, two new tokens each
        _case("paged_long", "paged", B=6, n_q=2, own=49157, page=32, block=32, mix=5, type="f16"),
        # the weights of one decode step of a batch
        _case("weights_step", "weights", B=61, T=61, own=1500, Hq=28, Hkv=4, mix=6),
        # whole prompts of many lengths, packed, against their own keys
        _case("weights_prompt", "weights", B=23, T=12007, own=0, page=64, mix=1),
        # the last queries of a few long prompts: what they look at is what stays
        _case("weights_window", "weights", B=3, T=192, own=9001, Hq=40, page=64, type="f16", mix=7),
        # a decode step of long chats whose cache is held in 8 bits
        _case("weights_long", "weights", B=6, T=12, own=49157, page=32, block=32, mix=5, type="f16"),
        # short chats cut to four pages each
        _case("evict_step", "evict", B=8, own=97, budget=64, first=4, last=16, Hq=28, Hkv=4, mix=3),
        # long prompts cut to an eighth after prefill
        _case("evict_prompt", "evict", B=3, own=16384, budget=2048, first=4, last=64, Hq=40, page=64, mix=8),
        # long chats in 8 bits cut to a quarter
        _case("evict_long", "evict", B=6, own=49157, budget=12301, first=4, last=256, page=32, block=32, mix=5, type="f16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "paged", "weights", "evict"])
    Hq, Hkv, d = rng.choice([(28, 4, 128), (32, 8, 128), (40, 8, 128), (4, 4, 64), (12, 12, 80)])
    c = _case("", op, Hq=Hq, Hkv=Hkv, d=d)
    del c["name"]
    c["type"] = rng.choice(["bf16", "bf16", "f16"])
    c["page"] = rng.choice([16, 32, 64, 128])
    c["mix"] = rng.randrange(1, 1000)
    c["block"] = rng.choice([b for b in (16, 32, 64, 128) if b <= c["page"]])
    if op == "append":
        c["type"] = rng.choice(["bf16", "bf16", "f16", "f32"])
        c["T"] = _log(rng, 1, 16384)
        c["B"] = min(c["T"], _log(rng, 1, 64))
        c["own"] = _log(rng, 1, 640)
        c["rot"] = 16 * rng.randint(1, d // 16) if rng.random() < 0.4 else d
        c["inter"] = rng.random() < 0.3
        c["norm"] = rng.random() < 0.6
        c["reach"] = rng.choice([1, 4, 16])
    elif op == "paged":
        c["B"] = _log(rng, 1, 128)
        c["n_q"] = rng.choice([1, 1, 1, 2, 3, 5])
        c["prefix"] = rng.choice([0, _log(rng, 16, 32768), _log(rng, 256, 32768)])
        c["own"] = _log(rng, 1, min(32768, max(16, 260000 // c["B"])))
    elif op == "weights":
        c["block"] = rng.choice([0, c["block"]])
        if rng.random() < 0.5:                      # a step of a batch
            c["B"] = _log(rng, 1, 128)
            c["T"] = c["B"] * rng.choice([1, 1, 2, 5])
            c["own"] = _log(rng, 1, min(32768, max(16, 260000 // c["B"])))
        else:                                       # prompts, whole or their last queries
            c["T"] = _log(rng, 1, 12000)
            c["B"] = min(c["T"], rng.choice([1, 1, _log(rng, 2, 32)]))
            c["own"] = rng.choice([0, _log(rng, 1, 8192)])
        longest = max(_lengths(c["B"], c["T"], c["mix"]))
        while c["B"] * Hq * longest * (longest + c["own"]) > 4 << 30:          # the plain form's scores
            c["T"] = c["T"] * 3 // 4
            c["own"] = c["own"] * 3 // 4
            c["B"] = min(c["B"], c["T"])
            longest = max(_lengths(c["B"], c["T"], c["mix"]))
    else:
        c["block"] = rng.choice([0, c["block"]])
        c["B"] = _log(rng, 1, 64)
        c["own"] = _log(rng, 2, min(49152, max(64, 260000 // c["B"])))
        c["budget"] = max(1, int(c["own"] * rng.uniform(0.05, 1.0)))
        c["first"] = min(rng.choice([0, 4, 16]), c["budget"])
        c["last"] = min(_log(rng, 1, 256), c["budget"] - c["first"])
    return c


def _lengths(n, total, mix):
    """n lengths of at least 1 that sum to total, spread over a factor of about 30; one each where that is all."""
    r = random.Random(mix)
    w = [math.exp(r.uniform(0.0, 3.4)) for _ in range(n)]
    if total % n == 0 and total // n <= 8:
        return [total // n] * n
    left, out = total - n, []
    for i in range(n):
        take = int(left * w[i] / sum(w[i:])) if i < n - 1 else left
        out.append(1 + take)
        left -= take
    return out


def _before(c):
    """Rows of each sequence that are in the cache before a call's own: up to c["own"]."""
    r = random.Random(c["mix"])
    low = 1 if c["op"] == "evict" else 0
    return [max(low, int(c["own"] * (1.0 if b == 0 else r.uniform(0.05, 1.0)))) for b in range(c["B"])]


def _rows_of(c):
    """(rows in the cache, new ones among them) of each sequence."""
    n = [c["n_q"]] * c["B"] if c["op"] == "paged" else [0] * c["B"] if c["op"] == "evict" else _lengths(c["B"], c["T"], c["mix"])
    return [a + b for a, b in zip(_before(c), n)], n


def _table(n_pos, rot, device):
    f = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=device) / rot)
    a = torch.arange(n_pos, dtype=torch.float64, device=device)[:, None] * f
    return torch.stack([a.cos(), a.sin()], 1).float().contiguous()


def _rows(shape, g, dev, dt, spread=1.0):
    return (torch.randn(shape, generator=g, device=dev) * spread).to(dt)


def _keys(shape, g, dev):
    """Keys share a mean over the tokens, as trained projections' do."""
    return torch.randn(shape, generator=g, device=dev) + torch.randn((1,) * (len(shape) - 1) + shape[-1:], generator=g, device=dev)


def _two(e):
    """2^e, for whole e of normal numbers."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _held(x, block):
    """x [pages, H, page, d] in 8 bits: codes, and the powers of two of each block [pages, H, page / block]."""
    p, H, ps, d = x.shape
    y = x.view(p, H, ps // block, block * d)
    m, e = torch.frexp(y.abs().amax(-1))
    k = e - 9 + (m > 0.875).int()
    return (y * _two(-k)[..., None]).to(torch.float8_e4m3fn).view(p, H, ps, d), (k + 127).to(torch.uint8).view(torch.float8_e8m0fnu)


def prepare(case, seed):
    c, dev = case, "cuda"
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    dt = _TYPES[c["type"]]
    Hq, Hkv, d, ps, B = c["Hq"], c["Hkv"], c["d"], c["page"], c["B"]
    s = {"c": c, "scale": 1.0 / math.sqrt(d), "pre": None}
    # the cache: pages in any order, those of a prefix among them
    lens, new = _rows_of(c)
    n_pre = -(-c.get("prefix", 0) // ps)
    used = [-(-n // ps) for n in lens]
    order = torch.randperm(n_pre + sum(used), generator=g, device=dev).to(torch.int32)
    s["pre"] = order[:n_pre].clone()
    s["pages"] = torch.zeros((B, max(used)), dtype=torch.int32, device=dev)
    at = n_pre
    for b, n in enumerate(used):
        s["pages"][b, :n] = order[at:at + n]
        at += n
    s["lens"] = torch.tensor(lens, dtype=torch.int32, device=dev)
    shape = (len(order), Hkv, ps, d)
    kc, vc = _keys(shape, g, dev), _rows(shape, g, dev, torch.float32)
    if c["block"]:
        (s["kc"], s["ks"]), (s["vc"], s["vs"]) = _held(kc, c["block"]), _held(vc, c["block"])
    else:
        s["kc"], s["vc"], s["ks"], s["vs"] = kc.to(dt), vc.to(dt), None, None
    del kc, vc
    if c["op"] == "append":
        T = c["T"]
        # one projection's rows: queries, keys and values of a token side by side
        qkv = _rows((T, Hq + 2 * Hkv, d), g, dev, dt, 1.7)
        s["k"], s["v"] = qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
        s["cu"] = torch.tensor([0] + new, device=dev).cumsum(0).to(torch.int32)
        s["wk"] = (1.0 + 0.2 * torch.randn(d, generator=g, device=dev)).to(dt) if c["norm"] else None
        # increasing positions with gaps of up to 2 reach - 1, as macro-tokens have them
        s["pos"] = (torch.randint(1, 2 * c["reach"], (T,), generator=g, device=dev).cumsum(0) - 1).to(torch.int32)
        s["table"] = _table(T * (2 * c["reach"] - 1), c["rot"], dev)
    elif c["op"] == "paged":
        s["q"] = _rows((B, c["n_q"], Hq, d), g, dev, dt, 1.3)
        s["out"] = torch.empty_like(s["q"])
    elif c["op"] == "weights":
        s["q"] = _rows((sum(new), Hq, d), g, dev, dt, 1.3)
        s["cu"] = torch.tensor([0] + new, device=dev).cumsum(0).to(torch.int32)
        s["longest"] = max(new)
        s["w"] = torch.rand((B, Hkv, s["pages"].shape[1] * ps), generator=g, device=dev)
        sc, seen, there = _scores(s)
        sc.masked_fill_(~seen, -math.inf)
        lse = torch.logsumexp(sc, -1).permute(0, 3, 1, 2)                     # [B, longest, Hkv, g]
        s["lse"] = lse[there].reshape(len(s["q"]), Hq).contiguous()
    else:
        # weights as a decode leaves them: most keys little, a few much, some none at all
        w = torch.randn((B, Hkv, s["pages"].shape[1] * ps), generator=g, device=dev).mul_(2.0).exp_()
        w[torch.rand(w.shape, generator=g, device=dev) < 0.05] = 0.0
        w[torch.arange(w.shape[-1], device=dev) >= s["lens"][:, None, None].expand(B, Hkv, 1)] = 0.0
        s["w"] = w
        s["w_out"], s["lens_out"] = torch.empty_like(w), torch.empty_like(s["lens"])
        s["kept"] = torch.empty((B, Hkv, c["budget"]), dtype=torch.int32, device=dev)
    return s


# ---------------------------------------------------------------- the plain forms
def _values(codes, scales, block):
    """What codes [..., rows, d] with scales [..., rows / block] stand for, in 32 bits."""
    x = codes.float()
    return x if scales is None else x * _two(scales.int() - 127).repeat_interleave(block, -1)[..., None]


def _exponent(top):
    """Of the smallest power of two whose 448-fold is at least `top`."""
    m, e = torch.frexp(top)
    return torch.where(top > 0, e - 9 + (m > 0.875).int(), torch.full_like(e, -126)).clamp(min=-126)


def _plain_append(s):
    c, ps, blk = s["c"], s["c"]["page"], s["c"]["block"]
    dev, H, d = s["k"].device, c["Hkv"], c["d"]
    k, v = s["k"].double(), s["v"].double()
    if c["norm"]:
        k = k * torch.rsqrt((k * k).mean(-1, keepdim=True) + _EPS) * s["wk"].double()
    t = s["table"][s["pos"].long()][:, :, None].double()
    cos, sin = t[:, 0], t[:, 1]
    h = cos.shape[-1]
    a, b = (k[..., 0:2 * h:2], k[..., 1:2 * h:2]) if c["inter"] else (k[..., :h], k[..., h:2 * h])
    y = (a * cos - b * sin, b * cos + a * sin)
    y = torch.stack(y, -1).flatten(-2) if c["inter"] else torch.cat(y, -1)
    k = torch.cat([y, k[..., 2 * h:]], -1)
    # where each token goes
    cu, lens = s["cu"].long(), s["lens"].long()
    n, t = cu.diff(), torch.arange(c["T"], device=dev)
    b = torch.searchsorted(cu, t, right=True) - 1
    begin = lens - n
    row = begin[b] + t - cu[b]
    page, at = s["pages"][b, row // ps].long(), row % ps
    per = ps // blk
    block_of = page * per + at // blk
    # the block that a sequence's first new row shares with earlier ones
    p1, a1 = s["pages"][torch.arange(c["B"], device=dev), begin // ps].long(), begin % ps
    shared, first = begin % blk > 0, p1 * per + a1 // blk
    earlier = (torch.arange(blk, device=dev) < (begin % blk)[:, None])[..., None, None]            # [B, blk, 1, 1]
    rows = ((p1 * ps + a1 // blk * blk)[:, None] + torch.arange(blk, device=dev))                   # [B, blk]
    for x, codes, scales in ((k, s["kc"], s["ks"]), (v, s["vc"], s["vs"])):
        e = scales.view(torch.uint8).permute(0, 2, 1).reshape(-1, H).int() - 127                     # [pages * per, H]
        top = torch.zeros((len(e), H), dtype=torch.float64, device=dev)
        top.index_reduce_(0, block_of, x.abs().amax(-1), "amax")
        old = e[first]
        e[block_of] = _exponent(top)[block_of]
        new = torch.where(shared[:, None], torch.maximum(e[first], old), e[first])
        e[first] = new
        scales.view(torch.uint8).copy_((e + 127).to(torch.uint8).view(-1, per, H).permute(0, 2, 1))
        was = codes[rows // ps, :, rows % ps]                                                        # [B, blk, H, d]
        now = (was.float() * _two(old - new)[:, None, :, None]).to(codes.dtype)
        codes[rows // ps, :, rows % ps] = torch.where(earlier, now.float(), was.float()).to(codes.dtype)
        codes[page, :, at] = (x * _two(-e[block_of]).double()[..., None]).clamp(-448.0, 448.0).to(codes.dtype)
    return s["kc"], s["vc"], s["ks"], s["vs"]


def _plain_paged(s):
    c, q = s["c"], s["q"]
    B, n_q, Hkv, d, P, ps, blk = c["B"], c["n_q"], c["Hkv"], c["d"], c["prefix"], c["page"], c["block"]
    g = c["Hq"] // Hkv
    qf = (q.float() * s["scale"]).view(B, n_q, Hkv, g, d).permute(2, 0, 3, 1, 4)       # [Hkv, B, g, n_q, d]
    n = s["pages"].shape[1] * ps
    pages, first = s["pages"].long(), s["pre"].long()
    ko, vo = (_values(x[pages], y.view(torch.uint8)[pages], blk).permute(2, 0, 1, 3, 4).reshape(Hkv, B, n, d)
              for x, y in ((s["kc"], s["ks"]), (s["vc"], s["vs"])))
    kp, vp = (_values(x[first], y.view(torch.uint8)[first], blk).permute(1, 0, 2, 3).reshape(Hkv, -1, d)[:, :P]
              for x, y in ((s["kc"], s["ks"]), (s["vc"], s["vs"])))
    own_s = torch.matmul(qf.reshape(Hkv, B, g * n_q, d), ko.transpose(-1, -2).contiguous()).view(Hkv, B, g, n_q, n)
    pre_s = torch.matmul(qf.reshape(Hkv, B * g * n_q, d), kp.transpose(-1, -2).contiguous()).view(Hkv, B, g, n_q, P)
    limit = s["lens"].long()[:, None] - n_q + 1 + torch.arange(n_q, device=q.device)    # [B, n_q]
    seen = (torch.arange(n, device=q.device) < limit[:, :, None])[None, :, None]
    own_s.masked_fill_(~seen, -math.inf)
    sc = torch.cat([pre_s, own_s], -1)
    sc = sc.sub_(sc.amax(-1, keepdim=True)).exp_()
    o = torch.matmul(sc[..., :P].reshape(Hkv, B * g * n_q, P), vp).view(Hkv, B, g, n_q, d)
    o += torch.matmul(sc[..., P:].reshape(Hkv, B, g * n_q, n), vo).view(Hkv, B, g, n_q, d)
    o /= sc.sum(-1, keepdim=True)
    return o.permute(1, 3, 0, 2, 4).reshape(q.shape).to(q.dtype)


def _scores(s):
    """Scaled scores [B, Hkv, g, queries, keys] of padded sequences, where a query sees a key, and which queries exist."""
    c, q, Lq = s["c"], s["q"], s["longest"]
    B, Hkv, d, ps = c["B"], c["Hkv"], c["d"], c["page"]
    g, n, dev = c["Hq"] // Hkv, s["pages"].shape[1] * ps, q.device
    cu, pages = s["cu"].long(), s["pages"].long()
    nq, i, j = cu.diff()[:, None], torch.arange(Lq, device=dev)[None], torch.arange(n, device=dev)
    at = (cu[:-1, None] + i).clamp(max=len(q) - 1)
    qp = (q.float() * s["scale"])[at].view(B, Lq, Hkv, g, d).permute(0, 2, 3, 1, 4).reshape(B, Hkv, g * Lq, d)
    k = _values(s["kc"][pages], None if s["ks"] is None else s["ks"].view(torch.uint8)[pages], c["block"])   # [B, pages, Hkv, ps, d]
    k = k.permute(0, 2, 4, 1, 3).reshape(B, Hkv, d, n)
    limit = (s["lens"].long()[:, None] - nq + 1 + i)
    there = i < nq
    seen = (j < limit[..., None]) & there[..., None]
    return torch.matmul(qp, k).view(B, Hkv, g, Lq, n), seen[:, None, None], there


def _plain_weights(s):
    c, Hkv = s["c"], s["c"]["Hkv"]
    g = c["Hq"] // Hkv
    sc, seen, there = _scores(s)
    at = (s["cu"].long()[:-1, None] + torch.arange(s["longest"], device=sc.device)).clamp(max=len(s["q"]) - 1)
    lse = s["lse"][at].view(*at.shape, Hkv, g).permute(0, 2, 3, 1)                            # [B, Hkv, g, Lq]
    sc.sub_(lse[..., None]).masked_fill_(~seen, -math.inf)
    s["w"] += sc.exp_().sum((2, 3))
    return s["w"]


def _plain_evict(s):
    c, ps, blk = s["c"], s["c"]["page"], s["c"]["block"]
    B, H, d = c["B"], c["Hkv"], c["d"]
    w, lens, dev = s["w"], s["lens"].long(), s["w"].device
    rows = w.shape[-1]
    n = min(c["budget"], rows)
    j = torch.arange(rows, device=dev)
    always = (j < c["first"]) | (j >= lens[:, None] - c["last"])
    rank = torch.where(always[:, None], torch.full_like(w, math.inf), w)
    rank = torch.where((j < lens[:, None])[:, None], rank, torch.full_like(w, -1.0))          # weights are not negative
    order = rank.sort(dim=-1, descending=True, stable=True)[1][..., :n].sort(-1)[0]              # [B, H, n]
    cut = lens > c["budget"]                                                                 # the others stay as they are
    there = torch.arange(n, device=dev) < lens[:, None]
    # rows behind a short sequence's last: its last again
    i = torch.minimum(torch.arange(n, device=dev), lens[:, None] - 1)[:, None]               # [B, 1, n]
    src = torch.where(cut[:, None, None], order, i)
    s["kept"].fill_(-1)
    s["kept"][..., :n] = torch.where(there[:, None], src, torch.full_like(src, -1)).int()
    moved = w.gather(-1, src)
    s["w_out"].zero_()
    s["w_out"][..., :n] = torch.where(there[:, None], moved, torch.zeros_like(moved))
    s["lens_out"].copy_(lens.clamp(max=c["budget"]))
    pages, h, b = s["pages"].long(), torch.arange(H, device=dev)[None, :, None], torch.arange(B, device=dev)[:, None, None]
    at = (pages[b, src // ps], h, src % ps)
    to = (pages[b, i // ps], h, i % ps)
    for codes, scales in ((s["kc"], s["ks"]), (s["vc"], s["vs"])):
        if scales is None:
            codes[to] = codes[at]                                                            # [B, H, n, d]
            continue
        e = scales.view(torch.uint8)
        x, was = codes[at].float() * _two(e[at[0], h, at[2] // blk].int() - 127)[..., None], codes[to]
        lead = torch.arange(0, n, blk, device=dev)
        y = torch.nn.functional.pad(x, (0, 0, 0, -n % blk)).view(B, H, len(lead), blk * d)
        k = _exponent(y.abs().amax(-1))                                                      # [B, H, blocks]
        y = (y * _two(-k)[..., None]).view(B, H, -1, d)[:, :, :n]
        codes[to] = torch.where(cut[:, None, None, None], y, was.float()).to(codes.dtype)
        lead = torch.minimum(lead, lens[:, None] - 1)[:, None]
        lead = (pages[b, lead // ps], h, lead % ps // blk)
        e[lead] = torch.where(cut[:, None, None], k + 127, e[lead].int()).to(torch.uint8)
    return _evicted(s)


def _evicted(s):
    return tuple(s[x] for x in ("kc", "vc", "ks", "vs", "w_out", "lens_out", "kept") if s[x] is not None)


def run(state):
    s, c = state, state["c"]
    op = c["op"]
    if not own:
        return {"append": _plain_append, "paged": _plain_paged, "weights": _plain_weights, "evict": _plain_evict}[op](s)
    import paper_2607_19368_amd as P
    if op == "append":
        return P.slh_kv_append_e4m3(s["k"], s["v"], s["kc"], s["vc"], s["ks"], s["vs"], s["pages"], s["lens"], s["cu"], s["wk"],
                                    eps=_EPS, table=s["table"], pos=s["pos"], interleaved=c["inter"])
    if op == "paged":
        return P.slh_attend_paged_e4m3(s["q"], s["kc"], s["vc"], s["ks"], s["vs"], s["pages"], s["lens"], prefix_pages=s["pre"],
                                       prefix_len=c["prefix"], scale=s["scale"], out=s["out"])
    if op == "weights":
        return P.slh_attend_weights(s["q"], s["kc"], s["pages"], s["lens"], s["lse"], s["w"], cu_q=s["cu"], k_scale=s["ks"],
                                    scale=s["scale"])
    P.slh_kv_evict(s["kc"], s["vc"], s["w"], s["pages"], s["lens"], c["budget"], first=c["first"], last=c["last"],
                   k_scale=s["ks"], v_scale=s["vs"], weights_out=s["w_out"], lens_out=s["lens_out"], kept=s["kept"])
    return _evicted(s)


# ---------------------------------------------------------------- what a pass has to do
def _pairs(nq, nk):
    """(query, key) pairs of one sequence and head, where the last query sees every key."""
    return nq * (nk - nq + 1) + nq * (nq - 1) // 2


def work(case):
    c = case
    e = 4 if c["type"] == "f32" else 2
    Hq, Hkv, d, blk = c["Hq"], c["Hkv"], c["d"], c["block"]
    lens, new = _rows_of(c)
    held = d + 1.0 / blk if blk else e * d                       # bytes of a row of the cache
    if c["op"] == "append":
        T = c["T"]
        return {"bytes": T * (2 * Hkv * (e * d + held) + 4 * c["rot"] + 4), "flops": T * Hkv * (3 * c["rot"] + (4 * d if c["norm"] else 0) + 4 * d)}
    if c["op"] == "paged":
        keys = c["prefix"] + sum(lens)
        return {"bytes": 2 * Hkv * held * keys + 2 * e * d * Hq * sum(new),
                "flops": 4 * d * Hq * sum(n * c["prefix"] + _pairs(n, m) for n, m in zip(new, lens))}
    if c["op"] == "weights":
        return {"bytes": Hkv * sum(lens) * (held + 8) + sum(new) * Hq * (e * d + 4),
                "flops": 2 * d * Hq * sum(_pairs(n, m) for n, m in zip(new, lens))}
    n = c["budget"]
    cut = [m for m in lens if m > n]
    # weights read and written, the list of what stays, and the rows behind the first ones, which move
    return {"bytes": Hkv * (8 * sum(lens) + 4 * n * len(lens) + len(cut) * 4 * held * (n - c["first"])),
            "flops": Hkv * sum(lens)}


# ---------------------------------------------------------------- the definition in 64 bits
def _held_values(codes, scales, block):
    """Rows of the cache by page, head and row, in 64 bits."""
    x = codes.double()
    return x if scales is None else (x.unflatten(2, (-1, block)) * scales.double()[..., None, None]).flatten(2, 3)


def _own(x, s, b, n):
    """The first n rows of sequence b, [heads, n, d], of a cache's values by page."""
    ps = s["c"]["page"]
    return x[s["pages"][b, :-(-n // ps)].long()].transpose(0, 1).flatten(1, 2)[:, :n]


def _spread(x, s, b, n, rows):
    """Writes `rows` [heads, n, ...] as the first n of sequence b into x [pages, heads, per page, ...]."""
    per = x.shape[2]
    for i in range(0, n, per):
        m = min(per, n - i)
        x[int(s["pages"][b, i // per]), :, :m] = rows[:, i:i + m]


def _blocks(x, block):
    """2^k of each block of rows of x [heads, n, d], and x over them: the codes before they are rounded."""
    n = x.shape[1]
    y = torch.nn.functional.pad(x, (0, 0, 0, -n % block)).unflatten(1, (-1, block))
    top = y.abs().amax((-1, -2)).clamp(min=448 * 2.0 ** -126)
    k = torch.ceil(torch.log2(top / 448))
    k = torch.where(448 * 2.0 ** (k - 1) >= top, k - 1, torch.where(448 * 2.0 ** k < top, k + 1, k))
    return 2.0 ** k, (y / (2.0 ** k)[..., None, None]).flatten(1, 2)[:, :n]


def _exact_keys(s):
    """Each pair (a, b) of a normed key as the complex number a + i b, turned by exp(i p f)."""
    c, x = s["c"], s["k"].double()
    if s["wk"] is not None:
        x = x / ((x ** 2).sum(-1, keepdim=True) / x.shape[-1] + _EPS).sqrt() * s["wk"].double()
    rot, y = c["rot"], x.clone()
    # the angles' table is an input of the operator, in 32 bits
    f = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=x.device) / rot)
    ang = s["pos"].double()[:, None, None] * f
    turn = torch.complex(ang.cos().float().double(), ang.sin().float().double())
    at = (slice(0, rot, 2), slice(1, rot, 2)) if c["inter"] else (slice(0, rot // 2), slice(rot // 2, rot))
    z = torch.complex(x[..., at[0]].contiguous(), x[..., at[1]].contiguous()) * turn
    y[..., at[0]], y[..., at[1]] = z.real, z.imag
    return y


def exact(case, seed):
    c = case
    s = prepare(case, seed)
    Hq, Hkv, d, blk = c["Hq"], c["Hkv"], c["d"], c["block"]
    g, dev = Hq // Hkv, s["lens"].device
    lens, new = _rows_of(c)
    if c["op"] == "append":
        out = [s["kc"].double(), s["vc"].double(), s["ks"].double(), s["vs"].double()]
        cu = s["cu"].tolist()
        for x, codes, scales in ((_exact_keys(s), out[0], out[2]), (s["v"].double(), out[1], out[3])):
            for b, (n, m) in enumerate(zip(lens, new)):
                lo = (n - m) // blk * blk                         # where the first block that changes begins
                kept = n - m - lo
                rows = x[cu[b]:cu[b + 1]].transpose(0, 1)
                two, code = _blocks(torch.cat([torch.zeros((Hkv, kept, d), dtype=x.dtype, device=dev), rows], 1), blk)
                all_codes, all_two = _own(codes, s, b, n).clone(), _own_scales(scales, s, b, n)
                if kept:
                    old = all_two[:, lo // blk]
                    grown = torch.maximum(two[:, 0], old)
                    code[:, :blk] *= (two[:, 0] / grown)[:, None, None]
                    code[:, :kept] = all_codes[:, lo:lo + kept] * (old / grown)[:, None, None]
                    two[:, 0] = grown
                all_codes[:, lo:], all_two[:, lo // blk:] = code, two
                _spread(codes, s, b, n, all_codes)
                _spread(scales, s, b, all_two.shape[1], all_two)
        return tuple(out)
    if c["op"] == "paged":
        out = torch.zeros(s["q"].shape, dtype=torch.float64, device=dev)
        P, n_q = c["prefix"], c["n_q"]
        k, v = (_held_values(x, y, blk) for x, y in ((s["kc"], s["ks"]), (s["vc"], s["vs"])))
        first = [x[s["pre"].long()].transpose(0, 1).flatten(1, 2)[:, :P] for x in (k, v)]
        for b, n in enumerate(lens):
            limit = (P + n - n_q + 1 + torch.arange(n_q, device=dev)).repeat_interleave(g)
            kk, vv = (torch.cat([f, _own(x, s, b, n)], 1) for f, x in zip(first, (k, v)))
            q = s["q"][b].double().view(n_q, Hkv, g, d).transpose(0, 1).flatten(1, 2)             # [Hkv, n_q g, d]
            sc = torch.matmul(q, kk.transpose(-1, -2).contiguous()) * s["scale"]
            sc = sc.masked_fill(torch.arange(P + n, device=dev) >= limit[:, None], -math.inf)
            out[b] = torch.matmul(torch.softmax(sc, -1), vv).view(Hkv, n_q, g, d).transpose(0, 1).flatten(1, 2)
        return out
    if c["op"] == "weights":
        w = s["w"].double()
        k = _held_values(s["kc"], s["ks"], blk)
        cu = s["cu"].tolist()
        for b, (n, m) in enumerate(zip(lens, new)):
            kk = _own(k, s, b, n)
            limit = n - m + 1 + torch.arange(m, device=dev)
            hide = torch.arange(n, device=dev)[None] >= limit[:, None]
            for h in range(Hq):
                sc = s["q"][cu[b]:cu[b + 1], h].double() @ kk[h // g].T * s["scale"]
                p = torch.exp(sc - s["lse"][cu[b]:cu[b + 1], h].double()[:, None])
                w[b, h // g, :n] += p.masked_fill(hide, 0.0).sum(0)
        return w
    caches = [x.double() for x in (s["kc"], s["vc"])] + [x.double() for x in (s["ks"], s["vs"]) if x is not None]
    values = [_held_values(x, y, blk) for x, y in ((s["kc"], s["ks"]), (s["vc"], s["vs"]))]
    w, w_out = s["w"].double(), torch.zeros(s["w"].shape, dtype=torch.float64, device=dev)
    n = c["budget"]
    for b, m in enumerate(lens):
        if m <= n:
            w_out[b, :, :m] = w[b, :, :m]
            continue
        free = n - c["first"] - c["last"]
        mid = w[b, :, c["first"]:m - c["last"]]
        best = mid.argsort(dim=-1, descending=True, stable=True)[:, :free] + c["first"]
        ends = torch.cat([torch.arange(c["first"], device=dev), torch.arange(m - c["last"], m, device=dev)])
        stays = torch.cat([best, ends.expand(Hkv, -1)], 1).sort(-1)[0]
        w_out[b, :, :n] = w[b].gather(-1, stays)
        for x in range(2):
            rows = _own(values[x], s, b, m).gather(1, stays[..., None].expand(-1, -1, d))
            if blk:
                two, rows = _blocks(rows, blk)
                _spread(caches[2 + x], s, b, two.shape[1], two)
            _spread(caches[x], s, b, n, rows)
    return (*caches, w_out, None, None)


def _own_scales(x, s, b, n):
    """The powers of two of the blocks of sequence b's first n rows, [heads, blocks]."""
    blk = s["c"]["block"]
    return x[s["pages"][b, :-(-n // s["c"]["page"])].long()].transpose(0, 1).flatten(1, 2)[:, :-(-n // blk)].clone()
