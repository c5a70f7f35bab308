"""Operators around a paged cache held in 8 bits, as measurable cases.

  norm     queries and keys of one layer normed head by head, then rotated to their positions; or the gradients of that
  store    new keys (normed and rotated on the way) and values go into 8-bit pages, with a scale for every 16 tokens of a head
  read     cached tokens come back out of the pages as rows in 16 or 32 bits
  attend   the queries of each sequence's new tokens attend to the 8-bit pages: all that is cached, or a window and a few first tokens

Every sequence of a case has its own length and number of new tokens, drawn from the case alone, so that the work of a
case does not depend on the inputs' seed.
"""
from __future__ import annotations

import math
import random

import torch

own = False
DEV = "cuda:0"
BLOCK = 16                                    # tokens that share a scale
TOP = 448.0                                   # the largest value of the 8-bit type

BASE = dict(op="attend", batch=1, hq=32, hkv=8, d=128, page=64, context=0, context_min=0, new=1, new_min=0, dtype="bf16",
            rot=0, interleaved=False, normed=True, eps=1e-6, backward=False, softcap=0.0, window=0, sinks=0, slopes=False, prefix=False)


def _case(name=None, **kw):
    c = dict(BASE, **kw)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # one layer of a decode step of a small serving batch: eight tokens, launches are all there is
        _case("norm step x8", op="norm", batch=8, context=32768),
        # a long prompt, or the forward pass of a training batch
        _case("norm prompt 4x8k", op="norm", batch=4, new=8192),
        # the gradients of a training batch: of queries, keys and both weights; small heads, half of each rotated in neighbouring pairs
        _case("norm gradient 3x2731", op="norm", batch=3, new=2731, hq=16, hkv=4, d=64, rot=32, interleaved=True, eps=1e-5, backward=True),
        # one layer of a decode step of a full serving batch: a token for each of 64 sequences, into blocks begun before
        _case("store step x64", op="store", batch=64, context=8192, context_min=500),
        # a prompt into small pages, in 32 bits, without norms
        _case("store prompt 16k f32", op="store", hq=16, hkv=4, d=64, page=16, new=16384, dtype="f32", rot=32, interleaved=True, normed=False),
        # histories taken out of the cache as a prefill wants them
        _case("read history 32k x4", op="read", batch=4, new=32768),
        # the last turns of conversations, in 32 bits, out of small pages
        _case("read turn x16 f32", op="read", batch=16, hq=16, hkv=4, d=64, page=16, context=9000, context_min=1000, new=700, new_min=50, dtype="f32"),
        # the smallest attention: one sequence, two heads, 32 bits
        _case("attend step 4k f32", hq=8, hkv=2, d=64, context=4096, dtype="f32"),
        # a decode step of a small serving batch at an ordinary context
        _case("attend step 32k x8", batch=8, context=32768),
        # a decode step of a full serving batch of very different lengths; heads in groups of five, capped scores
        _case("attend step ragged x64", batch=64, hq=40, context=32000, context_min=2000, softcap=30.0),
        # a prompt from its first token on
        _case("attend prompt 8k", new=8192),
        # a mixed batch: single tokens and turns together, small heads and pages, a window with a few first tokens that stay visible
        _case("attend mixed x24", batch=24, hq=16, hkv=4, d=64, page=16, context=9000, context_min=100, new=600, new_min=1,
              window=2048, sinks=4, slopes=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "norm", "store", "read", "attend", "attend", "attend"])
    hkv = rng.choice([1, 2, 4, 8, 8])
    d = rng.choice([64, 128, 128])
    c = dict(op=op, hkv=hkv, hq=hkv * rng.choice([1, 2, 4, 4, 5, 8]), d=d, dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]))
    if op != "attend":
        c["batch"] = _log(rng, 1, 64)
        c["context"] = _log(rng, 1, 8192) - 1
        # no more values than the largest listed cases have
        heads, values = (2 * hkv, 1 << 28) if op == "read" else (c["hq"] + hkv, 1 << 27)
        c["new"] = min(_log(rng, 1, 8192), max(1, values // (c["batch"] * heads * d)))
        c["rot"] = rng.choice([0, 0, d // 2, 16 * rng.randint(1, d // 16)])
        c["interleaved"] = rng.random() < 0.5
        c["eps"] = rng.choice([1e-6, 1e-5])
    if op == "norm":
        c["backward"] = rng.random() < 0.4
        return _case(**c)
    c["page"] = rng.choice([16, 32, 64, 64, 128])
    if op in ("store", "read"):
        c["normed"] = rng.random() < 0.7
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
    c["window"] = rng.choice([0, 0, _log(rng, 1, 8192)])
    c["sinks"] = rng.choice([0, 1, 4, 130]) if c["window"] else 0
    c["slopes"] = rng.random() < 0.2
    c["prefix"] = rng.random() < 0.2
    return _case(**c)


def _lens(c):
    """New tokens and cached tokens before them, of every sequence: uniform between the case's bounds, the largest first."""
    r = random.Random(c["batch"] * 1009 + c["new"] * 31 + c["context"])
    new = [c["new"]] + [r.randint(c["new_min"], c["new"]) if c["new_min"] else c["new"] for _ in range(c["batch"] - 1)]
    old = [c["context"]] + [r.randint(c["context_min"], c["context"]) if c["context_min"] else c["context"] for _ in range(c["batch"] - 1)]
    return new, old


def _prefix(c, new, old):
    """Tokens at the start that every token of the sequence sees, later ones of the prefix too: in two of three sequences."""
    return [0 if b % 3 == 2 else min(n + o, o + n // 2) for b, (n, o) in enumerate(zip(new, old))]


def _exponent(top):
    """The least e with top <= 448 2^e, for e of -40 to 40 (448 = 7/8 of 2^9)."""
    m, x = torch.frexp(top)
    e = (x - 9 + (m > 0.875)).clamp(-40, 40)
    return torch.where(top > 0, e, torch.full_like(e, -40))


def _power(e):
    return torch.ldexp(torch.ones(e.shape, device=e.device), e)


def _to_pages(x):
    """x [pages][heads][P][d] in 32 bits as 8-bit values and the exponents [pages][heads][P / 16] of their scales."""
    n, h, P, d = x.shape
    y = x.view(n, h, P // BLOCK, BLOCK, d)
    e = _exponent(y.abs().amax((-1, -2)))
    return (y / _power(e)[..., None, None]).clamp(-TOP, TOP).to(torch.float8_e4m3fn).view(n, h, P, d), e


def _scales(e):
    return (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)


def _bytes(x):
    return x.view(torch.uint8)


def _values(b):
    return b.view(torch.float8_e4m3fn).float()


def prepare(case, seed):
    c = dict(BASE, **case)
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    r = torch.Generator(device="cpu")
    r.manual_seed(seed)
    t = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    B, hq, hkv, d, P = c["batch"], c["hq"], c["hkv"], c["d"], c["page"]
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    randn = lambda *shape: torch.randn(*shape, device=DEV, generator=g)  # noqa: E731
    s = dict(case=c)
    if c["normed"]:
        s["q_weight"], s["k_weight"] = 1.0 + 0.2 * randn(d), 1.0 + 0.2 * randn(d)
    else:
        s["q_weight"] = s["k_weight"] = None
    if c["op"] == "norm":
        # queries and keys as one projection leaves them; the gradients [batch][heads][tokens][d], as attention's backward pass leaves them
        n = c["new"]
        start = torch.randint(max(0, c["context"] - 1000), c["context"] + 1, (B, 1), generator=r)
        s["positions"] = (start + torch.arange(n)).to(torch.int32).to(DEV)
        qk = (1.7 * randn(B, n, hq + hkv, d)).to(t)
        s["q"], s["k"] = qk[:, :, :hq], qk[:, :, hq:]
        if c["backward"]:
            s["gq"], s["gk"] = randn(B, hq, n, d).to(t).transpose(1, 2), randn(B, hkv, n, d).to(t).transpose(1, 2)
        return s
    new, old = _lens(c)
    lens = [a + b for a, b in zip(new, old)]
    s["total"], longest = sum(new), max(lens)
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
    for name in ("k", "v"):
        # what is in the pages: blocks of different sizes of values; no more than 2^26 of them in 32 bits at a time
        held = torch.empty(pages, hkv, P, d, dtype=torch.float8_e4m3fn, device=DEV)
        scales = torch.empty(pages, hkv, P // BLOCK, dtype=torch.float8_e8m0fnu, device=DEV)
        some = max(1, (1 << 26) // (hkv * P * d))
        for x in range(0, pages, some):
            y = randn(min(some, pages - x), hkv, P // BLOCK, BLOCK, d)
            y *= torch.exp2(0.5 * randn(*y.shape[:3]))[..., None, None]
            p, e = _to_pages(y.flatten(2, 3))
            _bytes(held)[x:x + some] = _bytes(p)
            _bytes(scales)[x:x + some] = _bytes(_scales(e))
        s[name + "_pages"], s[name + "_scales"] = held, scales
    if c["op"] == "store":
        # one projection gives queries, keys and values of a token side by side
        qkv = (1.7 * randn(s["total"], hq + 2 * hkv, d)).to(t)
        s["q"], s["k"], s["v"] = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    elif c["op"] == "attend":
        s["q"] = (1.5 * randn(s["total"], hq, d)).to(t)
        s["slopes"] = torch.exp2(-8.0 * torch.arange(1, hq + 1, device=DEV, dtype=torch.float32) / hq) if c["slopes"] else None
        s["prefix_lens"] = ints(_prefix(c, new, old)) if c["prefix"] else None
    return s


def run(state):
    return {"norm": _norm, "store": _store, "read": _read, "attend": _attend}[state["case"]["op"]](state)


def _plan(c):
    """The frequencies that a program keeps for all layers and steps."""
    from paper_2601_22379_b200 import binding
    return binding.Rope(c["d"], rot_dim=c["rot"] or c["d"], base=10000.0, interleaved=c["interleaved"])


def _cache(s):
    """The handle that a program keeps for its pages."""
    from paper_2601_22379_b200 import binding
    return binding.PagedCache(s["k_pages"], s["v_pages"], n_q_heads=s["case"]["hq"], q_dtype=s["case"]["dtype"],
                              k_scales=s["k_scales"], v_scales=s["v_scales"])


def _angles(c, positions):
    """cos and sin of every position and pair: angles in 64 bits, which positions far out need."""
    R = c["rot"] or c["d"]
    f = 10000.0 ** (-2.0 * torch.arange(R // 2, dtype=torch.float64, device=positions.device) / R)
    angle = positions.double().unsqueeze(-1) * f
    return angle.cos().float(), angle.sin().float()


def _rotate(c, y, cos, sin):
    """y [..., heads, d] in 32 bits; cos, sin [..., R / 2]."""
    R = c["rot"] or c["d"]
    cos, sin = cos.unsqueeze(-2), sin.unsqueeze(-2)
    part, rest = y[..., :R], y[..., R:]
    if c["interleaved"]:
        a, b = part[..., 0::2], part[..., 1::2]
        turned = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    else:
        a, b = part[..., :R // 2], part[..., R // 2:]
        turned = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    return torch.cat((turned, rest), -1)


def _normed(c, x, weight):
    y = x.float()
    if weight is None:
        return y
    return y * torch.rsqrt(y.square().mean(-1, keepdim=True) + c["eps"]) * weight


def _norm_gradient(c, x, g, weight, cos, sin):
    x, u = x.float(), _rotate(c, g.float(), cos, -sin)
    r = torch.rsqrt(x.square().mean(-1, keepdim=True) + c["eps"])
    dweight = (u * x * r).sum((0, 1, 2))
    u = u * weight
    return r * (u - x * (r * r * (u * x).mean(-1, keepdim=True))), dweight


def _norm(s):
    c = s["case"]
    if own:
        if "rope" not in s:
            s["rope"] = _plan(c)
        if c["backward"]:
            return s["rope"].norm_backward(s["positions"], s["gq"], s["q"], s["q_weight"], s["gk"], s["k"], s["k_weight"], eps=c["eps"])
        return s["rope"].norm_apply(s["positions"], s["q"], s["q_weight"], s["k"], s["k_weight"], eps=c["eps"])
    cos, sin = _angles(c, s["positions"])
    t = s["q"].dtype
    if c["backward"]:
        dq, dwq = _norm_gradient(c, s["q"], s["gq"], s["q_weight"], cos, sin)
        dk, dwk = _norm_gradient(c, s["k"], s["gk"], s["k_weight"], cos, sin)
        return dq.to(t), dwq, dk.to(t), dwk
    return _rotate(c, _normed(c, s["q"], s["q_weight"]), cos, sin).to(t), _rotate(c, _normed(c, s["k"], s["k_weight"]), cos, sin).to(t)


def _token_places(s):
    """Sequence and position of every new token."""
    row = torch.arange(s["total"], device=DEV)
    seq = torch.searchsorted(s["cu"].long(), row, right=True) - 1
    pos = row - s["cu"].long()[seq + 1] + s["lens"].long()[seq]
    return seq, pos


def _store(s):
    c = s["case"]
    if own:
        if "cache" not in s:
            s["cache"], s["rope"] = _cache(s), _plan(c)
        q = s["cache"].append(s["k"], s["v"], s["cu"], s["lens"], s["table"], q=s["q"], rope=s["rope"],
                              q_weight=s["q_weight"], k_weight=s["k_weight"], eps=c["eps"])
        return q, s["k_pages"], s["v_pages"], s["k_scales"], s["v_scales"]
    P = c["page"]
    seq, pos = _token_places(s)
    cos, sin = _angles(c, pos)
    q = _rotate(c, _normed(c, s["q"], s["q_weight"]), cos, sin).to(s["q"].dtype)
    k, v = _rotate(c, _normed(c, s["k"], s["k_weight"]), cos, sin), s["v"].float()
    page, at = s["table"].long()[seq, pos // P], pos % P
    # the blocks that new tokens lie in, and the first position of theirs that is new (0: the block starts anew)
    block = page * (P // BLOCK) + at // BLOCK
    first = torch.full((s["k_pages"].shape[0] * (P // BLOCK),), BLOCK, device=DEV).scatter_reduce(0, block, pos % BLOCK, "amin")
    touched = torch.unique(block)
    first = first[touched]
    where = torch.searchsorted(touched, block)
    tp, tb = touched // (P // BLOCK), touched % (P // BLOCK)
    tokens = (tb * BLOCK).unsqueeze(-1) + torch.arange(BLOCK, device=DEV)
    kept = torch.arange(BLOCK, device=DEV) < first.unsqueeze(-1)             # tokens that were there
    for x, pages, scales in ((k, s["k_pages"], s["k_scales"]), (v, s["v_pages"], s["v_scales"])):
        hkv, held, powers = x.shape[1], _bytes(pages), _bytes(scales)
        e = torch.full((len(touched), hkv), -40, dtype=torch.int32, device=DEV)
        e = e.scatter_reduce(0, where.unsqueeze(-1).expand(-1, hkv), _exponent(x.abs().amax(-1)), "amax")
        before = powers[tp, :, tb].int() - 127
        e = torch.where(first.unsqueeze(-1) > 0, torch.maximum(e, before), e)
        there = _values(held[tp.unsqueeze(-1), :, tokens])                   # [blocks][16][heads][d]
        less = torch.where(kept.unsqueeze(-1), _power(before - e).unsqueeze(1), torch.ones((), device=DEV))
        held[tp.unsqueeze(-1), :, tokens] = _bytes((there * less.unsqueeze(-1)).to(torch.float8_e4m3fn))
        held[page, :, at] = _bytes((x / _power(e)[where].unsqueeze(-1)).clamp(-TOP, TOP).to(torch.float8_e4m3fn))
        powers[tp, :, tb] = _bytes(_scales(e))
    return q, s["k_pages"], s["v_pages"], s["k_scales"], s["v_scales"]


def _read(s):
    c = s["case"]
    if own:
        if "cache" not in s:
            s["cache"] = _cache(s)
        return s["cache"].read(s["cu"], s["lens"], s["table"], s["total"])
    P = c["page"]
    seq, pos = _token_places(s)
    page, at = s["table"].long()[seq, pos // P], pos % P
    t = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    return tuple((_values(_bytes(p)[page, :, at]) * _power(_bytes(x)[page, :, at // BLOCK].int() - 127).unsqueeze(-1)).to(t)
                 for p, x in ((s["k_pages"], s["k_scales"]), (s["v_pages"], s["v_scales"])))


def _attend(s):
    c = s["case"]
    if own:
        if "cache" not in s:
            s["cache"] = _cache(s)
        return s["cache"].attend(s["q"], s["cu"], s["lens"], s["table"], s["max_new"], s["max_len"], softcap=c["softcap"],
                                 window=c["window"], sinks=c["sinks"], slopes=s["slopes"], prefix_lens=s["prefix_lens"])
    B, hq, hkv, d, n, L = c["batch"], c["hq"], c["hkv"], c["d"], s["max_new"], s["max_len"]
    G = hq // hkv
    seq, pos = _token_places(s)
    i_of = torch.arange(s["total"], device=DEV) - s["cu"].long()[seq]
    # sequences padded to the longest: queries [B][hkv][G n][d], keys and values [B][hkv][L][d]
    q = torch.zeros(B, n, hq, d, device=DEV)
    q[seq, i_of] = s["q"].float()
    q = q.view(B, n, hkv, G, d).permute(0, 2, 3, 1, 4).reshape(B, hkv, G * n, d)
    table = s["table"].long()

    def values(pages, scales):
        x = _values(_bytes(pages)[table])                                # [B][columns][hkv][P][d]
        e = _bytes(scales)[table].int() - 127
        x = x.unflatten(3, (-1, BLOCK)).mul_(_power(e)[..., None, None])
        return x.flatten(3, 4).transpose(1, 2).reshape(B, hkv, -1, d)[:, :, :L]

    x = torch.matmul(q, values(s["k_pages"], s["k_scales"]).transpose(2, 3)).view(B, hkv, G, n, L)
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
        seen &= (j > (p - c["window"]).unsqueeze(-1)) | (j < c["sinks"])
    x.masked_fill_(~seen.view(B, 1, 1, n, L), -math.inf)
    m = x.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    x = x.sub_(m).exp_()
    z = x.sum(-1, keepdim=True)
    o = torch.matmul(x.view(B, hkv, G * n, L), values(s["v_pages"], s["v_scales"])).view(B, hkv, G, n, d) / torch.where(z == 0, torch.ones_like(z), z)
    lse = (m + z.log()).squeeze(-1)
    return o.permute(0, 3, 1, 2, 4).reshape(B, n, hq, d)[seq, i_of].to(s["q"].dtype), lse.permute(0, 3, 1, 2).reshape(B, n, hq)[seq, i_of]


def _seen(c, new, old):
    """Of every new token: first key of its window, the one after its last key."""
    prefix = _prefix(c, new, old) if c["prefix"] else [0] * len(new)
    lo, hi = [], []
    for n, o, pre in zip(new, old, prefix):
        for pos in range(o, o + n):
            lo.append(max(0, pos - c["window"] + 1) if c["window"] else 0)
            hi.append(min(o + n, max(pos + 1, pre)))
    return lo, hi


def work(case):
    c = dict(BASE, **case)
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    e = 2 if c["dtype"] == "bf16" else 4
    pairs = (c["rot"] or d) // 2
    if c["op"] == "norm":
        n = c["batch"] * c["new"] * (hq + hkv)
        return {"bytes": n * d * e * (3 if c["backward"] else 2), "flops": n * (6 * pairs + (12 if c["backward"] else 4) * d)}
    new, old = _lens(c)
    n = sum(new)
    byte = 1 + 1 / (BLOCK * d)                                    # of a value in the pages, its share of the scale included
    if c["op"] == "store":
        return {"bytes": n * d * (hq * 2 * e + 2 * hkv * (e + byte)), "flops": n * (hq + hkv) * (6 * pairs + (4 * d if c["normed"] else 0)) + 4 * n * hkv * d}
    if c["op"] == "read":
        return {"bytes": n * d * 2 * hkv * (e + byte), "flops": n * d * 2 * hkv}
    lo, hi = _seen(c, new, old)
    at, keys, pairs = 0, 0, 0                                     # keys that any new token of the sequence sees; (query, key) pairs
    for k in new:
        if k:
            a, b = min(lo[at:at + k]), max(hi[at:at + k])
            keys += b - a + min(a, c["sinks"])
        pairs += sum(max(0, y - x) + min(x, c["sinks"]) for x, y in zip(lo[at:at + k], hi[at:at + k]))
        at += k
    return {"bytes": n * hq * (2 * d * e + 4) + keys * 2 * hkv * d * byte, "flops": 4 * d * hq * pairs}


def _turned(c, y, pos):
    """y [..., tokens, heads, d] in 64 bits, rotated to pos [..., tokens] as a product of complex numbers."""
    R = c["rot"] or c["d"]
    i = torch.arange(0, R, 2, dtype=torch.float64, device=y.device)
    angle = pos.double()[..., None] * torch.exp(-i / R * math.log(10000.0))
    unit = torch.complex(torch.cos(angle), torch.sin(angle))[..., None, :]
    if c["interleaved"]:
        z = torch.complex(y[..., 0:R:2], y[..., 1:R:2]) * unit
        return torch.cat((torch.view_as_real(z).flatten(-2), y[..., R:]), -1)
    z = torch.complex(y[..., :R // 2], y[..., R // 2:R]) * unit
    return torch.cat((z.real, z.imag, y[..., R:]), -1)


def _exact_norm(c, x, weight):
    x = x.double()
    if weight is None:
        return x
    return x / (x.pow(2).sum(-1, keepdim=True) / c["d"] + c["eps"]).sqrt() * weight.double()


def _block_values(held, scales):
    """What a sequence's cached rows [tokens][d] and the scales [tokens / 16] of one head stand for."""
    return held.double() * torch.pow(2.0, scales.view(torch.uint8).double() - 127.0).repeat_interleave(BLOCK)[:, None]


def exact(case, seed):
    c = dict(BASE, **case)
    s = prepare(case, seed)
    P, d, G = c["page"], c["d"], c["hq"] // c["hkv"]
    if c["op"] == "norm":
        if not c["backward"]:
            return tuple(_turned(c, _exact_norm(c, s[x], s[x + "_weight"]), s["positions"]) for x in ("q", "k"))
        found = []
        for x in ("q", "k"):
            a, w = s[x].double().requires_grad_(), s[x + "_weight"].double().requires_grad_()
            found += torch.autograd.grad(_turned(c, _exact_norm(c, a, w), s["positions"]), (a, w), s["g" + x].double())
        return tuple(found)
    new, old = _lens(c)
    if c["op"] == "store":
        if sum(new) > 1 << 17:
            return None
        pos = torch.cat([torch.arange(o, o + n) for n, o in zip(new, old)]).to(DEV)
        q = _turned(c, _exact_norm(c, s["q"], s["q_weight"]), pos)
        found = [q]
        powers = []
        for name, x in (("k", _turned(c, _exact_norm(c, s["k"], s["k_weight"]), pos)), ("v", s["v"].double())):
            held, e = s[name + "_pages"].double(), s[name + "_scales"].view(torch.uint8).double() - 127.0
            at = 0
            for b, (n, o) in enumerate(zip(new, old)):
                here = o
                while here < o + n:                               # block by block, as the tokens come
                    block, end = here // BLOCK, min(o + n, (here // BLOCK + 1) * BLOCK)
                    page, row = int(s["table"][b, here // P]), block * BLOCK % P
                    some = x[at:at + end - here]
                    need = torch.ceil(torch.log2(some.abs().amax((0, 2)) / TOP)).clamp(-40, 40)
                    was = e[page, :, row // BLOCK]
                    scale = torch.maximum(need, was) if here % BLOCK else need
                    if here % BLOCK:
                        held[page, :, row:row + here % BLOCK] *= torch.pow(2.0, was - scale)[:, None, None]
                    held[page, :, here % P:here % P + end - here] = (some / torch.pow(2.0, scale)[:, None]).transpose(0, 1)
                    e[page, :, row // BLOCK] = scale
                    at += end - here
                    here = end
            found.append(held)
            powers.append(torch.pow(2.0, e))
        return tuple(found + powers)
    if c["op"] == "read":
        found = []
        for name in ("k", "v"):
            rows = []
            for b, (n, o) in enumerate(zip(new, old)):
                pages = s["table"][b, :-(-(o + n) // P)].long()
                held = s[name + "_pages"].view(torch.uint8)[pages].view(torch.float8_e4m3fn).transpose(0, 1).reshape(c["hkv"], -1, d)
                scales = s[name + "_scales"].view(torch.uint8)[pages].transpose(0, 1).reshape(c["hkv"], -1)
                rows.append(torch.stack([_block_values(held[h], scales[h])[o:o + n] for h in range(c["hkv"])], 1))
            found.append(torch.cat(rows))
        return tuple(found)
    lo, hi = (torch.tensor(x, device=DEV) for x in _seen(c, new, old))
    out = torch.zeros(sum(new), c["hq"], d, dtype=torch.float64, device=DEV)
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
        hidden = (j >= hi[rows, None]) | ((j < lo[rows, None]) & (j >= c["sinks"]))
        for h in range(c["hkv"]):
            k, v = (_block_values(s[x + "_pages"][:, h].view(torch.uint8)[pages].view(torch.float8_e4m3fn).reshape(-1, d),
                                  s[x + "_scales"][:, h].view(torch.uint8)[pages].reshape(-1))[:o + n] for x in ("k", "v"))
            for m in range(h * G, h * G + G):
                x = s["q"][rows, m].double() @ k.T / math.sqrt(d)
                if c["softcap"]:
                    x = c["softcap"] * torch.tanh(x / c["softcap"])
                if c["slopes"]:
                    x = x - s["slopes"][m].double() * away
                x = x.masked_fill(hidden, -math.inf)
                lse[rows, m] = torch.logsumexp(x, -1)
                out[rows, m] = torch.nan_to_num(torch.softmax(x, -1), nan=0.0) @ v
    return out, lse
