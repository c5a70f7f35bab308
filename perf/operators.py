"""Operators around a paged KV cache, as measurable cases: rotary positions, appending to the cache, attention over it.

  rope     queries and keys of one layer rotated to their positions (or gradients rotated back)
  append   new keys and values, rotated on the way, go into the pages of their sequences; the queries are rotated beside them
  attend   the queries of each sequence's new tokens attend to all of its cached tokens that their mask leaves

Every sequence of a case has its own length and number of new tokens, drawn from the case alone, so that the work of a
case does not depend on the inputs' seed.
"""
from __future__ import annotations

import math
import random

import torch

own = False
DEV = "cuda:0"

BASE = dict(op="attend", batch=1, hq=32, hkv=8, d=128, page=64, context=0, context_min=0, new=1, new_min=0, dtype="bf16",
            rot=0, interleaved=False, scaling="none", factor=1.0, original=0, amplitude=1.0, backward=False,
            softcap=0.0, window=0, slopes=False, documents=False, prefix=False)


def _case(name=None, **kw):
    c = dict(BASE, **kw)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # one layer of a decode step of a small serving batch: eight tokens, launches are all there is
        _case("rope step x8", op="rope", batch=8, context=32768),
        # a long prompt; half of each head rotated, in neighbouring pairs, frequencies stretched for a longer context
        _case("rope prompt 4x8k part", op="rope", batch=4, new=8192, rot=64, interleaved=True, scaling="ramp", factor=8.0, original=8192, amplitude=1.2),
        # the gradients of a training batch in 32 bits, small heads, positions stretched linearly
        _case("rope gradient f32", op="rope", batch=3, new=2731, hq=16, hkv=4, d=64, dtype="f32", scaling="linear", factor=4.0, backward=True),
        # one layer of a decode step of a full serving batch: a token for each of 64 sequences
        _case("append step x64", op="append", batch=64, context=8192, context_min=500),
        # turns of conversations: another number of new tokens for each sequence, on top of their histories
        _case("append turn x16", op="append", batch=16, context=12288, context_min=3000, new=700, new_min=50, scaling="ramp", factor=4.0, original=8192),
        # a prompt into small pages, in 32 bits, half of each small head rotated in neighbouring pairs
        _case("append prompt 16k f32", op="append", hq=16, hkv=4, d=64, page=16, new=16384, dtype="f32", rot=32, interleaved=True),
        # the smallest attention: one head, one sequence, 32 bits
        _case("attend step 4k f32", hq=1, hkv=1, d=64, context=4096, dtype="f32"),
        # a decode step of a small serving batch at an ordinary context
        _case("attend step 32k x8", batch=8, context=32768),
        # a decode step of a full serving batch of very different lengths; heads in groups of five, capped scores
        _case("attend step ragged x64", batch=64, hq=40, context=32000, context_min=2000, softcap=30.0),
        # a prompt from its first token on
        _case("attend prompt 8k", new=8192),
        # chunked prefill of a serving loop: a chunk on top of a long context
        _case("attend 512 on 32k x2", batch=2, context=32768, new=512),
        # a mixed batch: single tokens and turns together, small heads and pages, scores that fall off with the distance,
        # a window, packed documents and a prefix that all of its tokens see
        _case("attend mixed x24", batch=24, hq=16, hkv=4, d=64, page=16, context=9000, context_min=100, new=600, new_min=1,
              window=4096, slopes=True, documents=True, prefix=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rope", "append", "attend", "attend"])
    hkv = rng.choice([1, 2, 4, 8, 8])
    d = rng.choice([64, 128, 128])
    c = dict(op=op, hkv=hkv, hq=hkv * rng.choice([1, 2, 4, 4, 5, 8]), d=d, dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]))
    if op != "attend":
        c["batch"] = _log(rng, 1, 64)
        c["context"] = _log(rng, 1, 8192) - 1
        c["new"] = min(_log(rng, 1, 8192), max(1, (1 << 27) // (c["batch"] * (c["hq"] + hkv) * d)))
        c["rot"] = rng.choice([0, 0, d // 2, 16 * rng.randint(1, d // 16)])
        c["interleaved"] = rng.random() < 0.5
        c["scaling"] = rng.choice(["none", "linear", "base", "ramp"])
        if c["scaling"] != "none":
            c["factor"], c["original"] = rng.choice([2.0, 4.0, 8.0, 32.0]), rng.choice([2048, 4096, 8192])
        c["amplitude"] = rng.choice([1.0, 1.0, 1.1386])
    if op == "rope":
        c["backward"] = rng.random() < 0.3
        return _case(**c)
    c["page"] = rng.choice([16, 32, 64, 64, 128])
    if op == "append":
        c["new_min"] = rng.choice([0, max(1, c["new"] // 10)])
        c["context_min"] = rng.choice([0, c["context"] // 8])
        return _case(**c)
    # no more (query, key) pairs and no more cached values than the largest listed cases have
    pairs, values = (1 << 31, 1 << 30) if c["dtype"] == "bf16" else (1 << 27, 1 << 28)
    c["batch"] = _log(rng, 1, 64)
    c["new"] = min(rng.choice([1, 1, _log(rng, 2, 40), _log(rng, 16, 8192)]), math.isqrt(pairs // (c["hq"] * c["batch"])))
    most = min(pairs // (c["hq"] * c["new"] * c["batch"]), values // (hkv * d * c["batch"]), 131072)
    c["context"] = _log(rng, 1, max(1, most - c["new"])) - 1
    c["context_min"] = rng.choice([0, c["context"] // 10])
    c["new_min"] = rng.choice([0, 1, max(1, c["new"] // 4)])
    c["softcap"] = rng.choice([0.0, 0.0, 0.0, 20.0, 50.0])
    c["window"] = rng.choice([0, 0, 0, _log(rng, 1, 8192)])
    c["slopes"] = rng.random() < 0.2
    c["documents"] = rng.random() < 0.2
    c["prefix"] = rng.random() < 0.2
    return _case(**c)


def _lens(c):
    """New tokens and cached tokens before them, of every sequence: uniform between the case's bounds, the largest first."""
    r = random.Random(c["batch"] * 1009 + c["new"] * 31 + c["context"])
    new = [c["new"]] + [r.randint(c["new_min"], c["new"]) if c["new_min"] else c["new"] for _ in range(c["batch"] - 1)]
    old = [c["context"]] + [r.randint(c["context_min"], c["context"]) if c["context_min"] else c["context"] for _ in range(c["batch"] - 1)]
    return new, old


def _first(c, new, old):
    """First key each new token may see where documents are packed: its sequence holds documents of about 500 tokens."""
    first = []
    for n, o in zip(new, old):
        r = random.Random(n * 7919 + o)
        starts = [0]
        while starts[-1] < o + n:
            starts.append(starts[-1] + r.randint(1, 1000))
        at = 0
        for pos in range(o, o + n):
            while starts[at + 1] <= pos:
                at += 1
            first.append(starts[at])
    return first


def _prefix(c, new, old):
    """Tokens at the start that every token of the sequence sees, later ones of the prefix too: in two of three sequences."""
    return [0 if b % 3 == 2 else min(n + o, o + n // 2) for b, (n, o) in enumerate(zip(new, old))]


def prepare(case, seed):
    c = dict(BASE, **case)
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    r = torch.Generator(device="cpu")
    r.manual_seed(seed)
    t = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    B, hq, hkv, d, P = c["batch"], c["hq"], c["hkv"], c["d"], c["page"]
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    randn = lambda *shape: torch.randn(*shape, device=DEV, generator=g).to(t)  # noqa: E731
    s = dict(case=c)
    if c["op"] == "rope":
        # queries [batch][tokens][heads][d] as a projection leaves them; keys [batch][heads][tokens][d], as the cache takes them
        n = c["new"]
        start = torch.randint(max(0, c["context"] - 1000), c["context"] + 1, (B, 1), generator=r)
        s["positions"] = (start + torch.arange(n)).to(torch.int32).to(DEV)
        s["q"] = randn(B, n, hq, d)
        s["k"] = randn(B, hkv, n, d).transpose(1, 2)
        return s
    new, old = _lens(c)
    lens = [a + b for a, b in zip(new, old)]
    total, longest = sum(new), max(lens)
    cols = -(-longest // P)
    pages = sum(-(-x // P) for x in lens)
    # every sequence's pages lie anywhere in the pool; columns behind its last page are not used
    order = torch.randperm(pages, generator=r).to(torch.int32)
    table = torch.zeros(B, cols, dtype=torch.int32)
    at = 0
    for b, x in enumerate(lens):
        m = -(-x // P)
        table[b, :m] = order[at:at + m]
        at += m
    s["table"] = table.to(DEV)
    s["cu"] = ints([0] + torch.tensor(new).cumsum(0).tolist())
    s["lens"] = ints(lens)
    s["max_new"], s["max_len"] = max(new), longest
    s["k_pages"], s["v_pages"] = randn(pages, hkv, P, d), randn(pages, hkv, P, d)
    if c["op"] == "append":
        # one projection gives queries, keys and values of a token side by side
        qkv = randn(total, hq + 2 * hkv, d)
        s["q"], s["k"], s["v"] = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    else:
        s["q"] = (1.5 * torch.randn(total, hq, d, device=DEV, generator=g)).to(t)
        s["slopes"] = torch.exp2(-8.0 * torch.arange(1, hq + 1, device=DEV, dtype=torch.float32) / hq) if c["slopes"] else None
        s["first_key"] = ints(_first(c, new, old)) if c["documents"] else None
        s["prefix_lens"] = ints(_prefix(c, new, old)) if c["prefix"] else None
    return s


def run(state):
    return {"rope": _rope, "append": _append, "attend": _attend}[state["case"]["op"]](state)


def _plan(c):
    """The frequencies that a program keeps for all layers and steps."""
    from paper_2601_22379_b200 import binding
    return binding.Rope(c["d"], rot_dim=c["rot"] or c["d"], base=10000.0, interleaved=c["interleaved"], scaling=c["scaling"],
                        factor=c["factor"], original_len=c["original"], ramp=(1.0, 32.0), amplitude=c["amplitude"])


def _cache(s):
    """The handle that a program keeps for its pages."""
    from paper_2601_22379_b200 import binding
    return binding.PagedCache(s["k_pages"], s["v_pages"], n_q_heads=s["case"]["hq"], q_dtype=s["case"]["dtype"])


def _angles(c, positions):
    """cos and sin of every position and pair, amplitude included: angles in 64 bits, which positions far out need."""
    R = c["rot"] or c["d"]
    base, turn = 10000.0, 2.0 * math.pi
    if c["scaling"] == "base":
        base *= c["factor"] ** (R / (R - 2))
    f = base ** (-2.0 * torch.arange(R // 2, dtype=torch.float64, device=positions.device) / R)
    if c["scaling"] == "linear":
        f = f / c["factor"]
    if c["scaling"] == "ramp":
        w = ((c["original"] * f / turn - 1.0) / 31.0).clamp(0.0, 1.0)
        f = w * f + (1.0 - w) * f / c["factor"]
    angle = positions.double().unsqueeze(-1) * f
    return (angle.cos() * c["amplitude"]).float(), (angle.sin() * c["amplitude"]).float()


def _rotate(c, x, cos, sin):
    """x [..., heads, d] in 32 bits, rounded once at the end; cos, sin [..., R / 2]."""
    R = c["rot"] or c["d"]
    cos, sin, y = cos.unsqueeze(-2), sin.unsqueeze(-2), x.float()
    part, rest = y[..., :R], y[..., R:]
    if c["interleaved"]:
        a, b = part[..., 0::2], part[..., 1::2]
        turned = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    else:
        a, b = part[..., :R // 2], part[..., R // 2:]
        turned = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    return torch.cat((turned, rest), -1).to(x.dtype)


def _rope(s):
    c = s["case"]
    if own:
        if "rope" not in s:
            s["rope"] = _plan(c)
        return s["rope"].apply(s["positions"], s["q"], s["k"], transpose=c["backward"])
    cos, sin = _angles(c, s["positions"])
    if c["backward"]:
        sin = -sin
    return _rotate(c, s["q"], cos, sin), _rotate(c, s["k"], cos, sin)


def _token_places(s):
    """Sequence and position of every new token."""
    row = torch.arange(s["q"].shape[0], device=DEV)
    seq = torch.searchsorted(s["cu"].long(), row, right=True) - 1
    pos = row - s["cu"].long()[seq + 1] + s["lens"].long()[seq]
    return seq, pos


def _append(s):
    c = s["case"]
    if own:
        if "cache" not in s:
            s["cache"], s["rope"] = _cache(s), _plan(c)
        q = s["cache"].append(s["k"], s["v"], s["cu"], s["lens"], s["table"], q=s["q"], rope=s["rope"])
        return q, s["k_pages"], s["v_pages"]
    seq, pos = _token_places(s)
    cos, sin = _angles(c, pos)
    page, at = s["table"].long()[seq, pos // c["page"]], pos % c["page"]
    s["k_pages"][page, :, at] = _rotate(c, s["k"], cos, sin)
    s["v_pages"][page, :, at] = s["v"]
    return _rotate(c, s["q"], cos, sin), s["k_pages"], s["v_pages"]


def _attend(s):
    c = s["case"]
    if own:
        if "cache" not in s:
            s["cache"] = _cache(s)
        return s["cache"].attend(s["q"], s["cu"], s["lens"], s["table"], s["max_new"], s["max_len"], softcap=c["softcap"],
                                 window=c["window"], slopes=s["slopes"], first_key=s["first_key"], prefix_lens=s["prefix_lens"])
    B, hq, hkv, d, n, L = c["batch"], c["hq"], c["hkv"], c["d"], s["max_new"], s["max_len"]
    G = hq // hkv
    seq, pos = _token_places(s)
    i_of = torch.arange(s["q"].shape[0], device=DEV) - s["cu"].long()[seq]
    # sequences padded to the longest: queries [B][hkv][G n][d], keys and values [B][hkv][L][d]
    q = torch.zeros(B, n, hq, d, device=DEV)
    q[seq, i_of] = s["q"].float()
    q = q.view(B, n, hkv, G, d).permute(0, 2, 3, 1, 4).reshape(B, hkv, G * n, d)
    table = s["table"].long()
    k = s["k_pages"][table].transpose(1, 2).reshape(B, hkv, -1, d)[:, :, :L].float()
    x = torch.matmul(q, k.transpose(2, 3)).view(B, hkv, G, n, L)
    del k
    x *= 1.0 / math.sqrt(d)
    if c["softcap"]:
        x = torch.tanh(x / c["softcap"]) * c["softcap"]
    j = torch.arange(L, device=DEV)
    p = torch.full((B, n), -1, device=DEV)                        # (places without a token see nothing)
    p[seq, i_of] = pos
    if c["slopes"]:
        x -= s["slopes"].view(1, hkv, G, 1, 1) * (p.unsqueeze(-1) - j).abs().float().view(B, 1, 1, n, L)
    hi = p + 1
    if c["prefix"]:
        hi = torch.where(p >= 0, torch.maximum(hi, s["prefix_lens"].long().unsqueeze(-1)), hi)
    hi = torch.minimum(hi, s["lens"].long().unsqueeze(-1))
    seen = j < hi.unsqueeze(-1)
    if c["window"]:
        seen &= j > (p - c["window"]).unsqueeze(-1)
    if c["documents"]:
        lo = torch.zeros(B, n, dtype=torch.long, device=DEV)
        lo[seq, i_of] = s["first_key"].long()
        seen &= j >= lo.unsqueeze(-1)
    x.masked_fill_(~seen.view(B, 1, 1, n, L), -math.inf)
    m = x.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    x = x.sub_(m).exp_()
    z = x.sum(-1, keepdim=True)
    v = s["v_pages"][table].transpose(1, 2).reshape(B, hkv, -1, d)[:, :, :L].float()
    o = torch.matmul(x.view(B, hkv, G * n, L), v).view(B, hkv, G, n, d) / torch.where(z == 0, torch.ones_like(z), z)
    lse = (m + z.log()).squeeze(-1)
    return o.permute(0, 3, 1, 2, 4).reshape(B, n, hq, d)[seq, i_of].to(s["q"].dtype), lse.permute(0, 3, 1, 2).reshape(B, n, hq)[seq, i_of]


def _bounds(c, new, old):
    """First visible key and the one after the last, of every new token."""
    first = _first(c, new, old) if c["documents"] else None
    prefix = _prefix(c, new, old) if c["prefix"] else [0] * len(new)
    lo, hi = [], []
    for n, o, pre in zip(new, old, prefix):
        for pos in range(o, o + n):
            a = max(0, pos - c["window"] + 1) if c["window"] else 0
            lo.append(max(a, first[len(lo)]) if first else a)
            hi.append(min(o + n, max(pos + 1, pre)))
    return lo, hi


def work(case):
    c = dict(BASE, **case)
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    e = 2 if c["dtype"] == "bf16" else 4
    pairs = (c["rot"] or d) // 2
    if c["op"] == "rope":
        n = c["batch"] * c["new"]
        return {"bytes": n * (2 * (hq + hkv) * d * e + 4), "flops": 6 * n * (hq + hkv) * pairs}
    new, old = _lens(c)
    n = sum(new)
    if c["op"] == "append":
        return {"bytes": n * 2 * (hq + 2 * hkv) * d * e, "flops": 6 * n * (hq + hkv) * pairs}
    lo, hi = _bounds(c, new, old)
    at, keys = 0, 0                                               # keys that any new token of the sequence sees
    for k in new:
        keys += max(hi[at:at + k]) - min(lo[at:at + k]) if k else 0
        at += k
    return {"bytes": n * hq * (2 * d * e + 4) + keys * 2 * hkv * d * e, "flops": 4 * d * hq * sum(max(0, b - a) for a, b in zip(lo, hi))}


def _turned(c, x, pos):
    """x [..., tokens, heads, d] rotated to pos [..., tokens], everything in 64 bits, as a product of complex numbers."""
    R = c["rot"] or c["d"]
    i = torch.arange(0, R, 2, dtype=torch.float64, device=x.device)
    stretched = c["factor"] ** (R / (R - 2)) if c["scaling"] == "base" else 1.0
    f = torch.exp(-i / R * math.log(10000.0 * stretched))
    if c["scaling"] == "linear":
        f = f / c["factor"]
    elif c["scaling"] == "ramp":
        turns = f * c["original"] / (2 * math.pi)
        w = torch.clamp((turns - 1) / (32 - 1), 0, 1)
        f = f * (w + (1 - w) / c["factor"])
    sign = -1.0 if c["backward"] else 1.0
    angle = pos.double()[..., None] * f
    unit = c["amplitude"] * torch.complex(torch.cos(angle), sign * torch.sin(angle))
    y = x.double().clone()
    if c["interleaved"]:
        z = torch.complex(y[..., 0:R:2], y[..., 1:R:2]) * unit[..., None, :]
        y[..., 0:R:2], y[..., 1:R:2] = z.real, z.imag
    else:
        z = torch.complex(y[..., :R // 2], y[..., R // 2:R]) * unit[..., None, :]
        y[..., :R // 2], y[..., R // 2:R] = z.real, z.imag
    return y


def exact(case, seed):
    c = dict(BASE, **case)
    s = prepare(case, seed)
    if c["op"] == "rope":
        return _turned(c, s["q"], s["positions"]), _turned(c, s["k"], s["positions"])
    new, old = _lens(c)
    P, G = c["page"], c["hq"] // c["hkv"]
    if c["op"] == "append":
        pos = torch.cat([torch.arange(o, o + n) for n, o in zip(new, old)]).to(DEV)
        k, q = _turned(c, s["k"], pos), _turned(c, s["q"], pos)
        kp, vp = s["k_pages"].double(), s["v_pages"].double()
        at = 0
        for b, (n, o) in enumerate(zip(new, old)):
            where = torch.arange(o, o + n, device=DEV)
            page = s["table"][b].long()[where // P]
            kp[page, :, where % P] = k[at:at + n]
            vp[page, :, where % P] = s["v"][at:at + n].double()
            at += n
        return q, kp, vp
    lo, hi = (torch.tensor(x, device=DEV) for x in _bounds(c, new, old))
    out = torch.zeros(sum(new), c["hq"], c["d"], dtype=torch.float64, device=DEV)
    lse = torch.full((sum(new), c["hq"]), -math.inf, dtype=torch.float64, device=DEV)
    at = 0
    for b, (n, o) in enumerate(zip(new, old)):
        if not n:
            continue
        rows = slice(at, at + n)
        at += n
        pages = s["table"][b, :-(-(o + n) // P)].long()
        j = torch.arange(o + n, device=DEV)
        away = (torch.arange(o, o + n, device=DEV)[:, None] - j).abs().double()
        hidden = (j < lo[rows, None]) | (j >= hi[rows, None])
        for h in range(c["hkv"]):
            k = s["k_pages"][pages, h].reshape(-1, c["d"])[:o + n].double()
            v = s["v_pages"][pages, h].reshape(-1, c["d"])[:o + n].double()
            for m in range(h * G, h * G + G):
                x = s["q"][rows, m].double() @ k.T / math.sqrt(c["d"])
                if c["softcap"]:
                    x = c["softcap"] * torch.tanh(x / c["softcap"])
                if c["slopes"]:
                    x = x - s["slopes"][m].double() * away
                x = x.masked_fill(hidden, -math.inf)
                lse[rows, m] = torch.logsumexp(x, -1)
                out[rows, m] = torch.nan_to_num(torch.softmax(x, -1), nan=0.0) @ v
    return out, lse
