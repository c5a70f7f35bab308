"""Attention over 8-bit pages with scores so large that fp32 counts them in steps of more than one: keys that tie for the largest share their weight."""
import math

import pytest
import torch

from paper_2601_22379_b200 import binding
from tests import paged_bytes_reference as ref8
from tests.test_gpu_paged_bytes import Batch, kinds

pytestmark = pytest.mark.gpu


def one_channel(new, old, q, flags, score, ev, d, hq=4, hkv=2, seed=0, fall=0.0):
    """Queries and keys with channel 0 alone: every third token's key is 1, the others' -1, so that the former's scores are `score` in base 2 and the latter's weight is 0.
    V's scales are 2^ev, ev drawn from a list.  fall: tokens before half of the cache have keys that much smaller."""
    b = Batch(new, old, hq=hq, hkv=hkv, d=d, P=64, q=q, flags=flags, seed=seed)
    g = torch.Generator().manual_seed(seed + 1)
    b.q[:] = 0
    natural = score * math.log(2.0) * math.sqrt(d)                            # of q . k
    b.q[:b.total, :, 0] = natural
    for n, (row, length) in enumerate(zip(b.table_cpu, b.lens)):
        at = torch.arange(length)
        page, rest = row.long()[at // b.P], at % b.P
        b.bytes["k"][page, :, rest] = 0
        b.bytes["k"][page, :, rest, 0] = torch.where(at % 3 == 0, torch.full_like(at, 0x38), torch.full_like(at, 0xb8)).to(torch.uint8)[:, None]   # 1 and -1 of e4m3
        if fall:
            half = at < length // 2
            b.bytes["k"][page[half], :, rest[half], 0] = 0x30                 # 0.5
    b.scales["k"][b.scales["k"] < 255] = 127
    drawn = torch.tensor(ev)[torch.randint(0, len(ev), b.scales["v"].shape, generator=g)]
    b.scales["v"] = torch.where(b.scales["v"] < 255, (drawn + 127).to(torch.uint8), b.scales["v"])
    b.put()
    return b


def visible_mean(b, fall=0.0):
    """Mean of the values that a row's largest keys have, and how many: what softmax leaves where all else has weight 0."""
    v = ref8.values(b.bytes["v"], b.scales["v"])
    rows, counts, most = [], [], []
    for s, (n, o) in enumerate(zip(b.new, b.old)):
        L = n + o
        at = torch.arange(L)
        held = v[b.table_cpu[s].long()[at // b.P], :, at % b.P]               # [L][hkv][d]
        for i in range(n):
            there = (at % 3 == 0) & (at < o + i + 1)
            if fall and bool((there & (at >= L // 2)).any()):
                there &= at >= L // 2
            rows.append(held[there].mean(0))
            most.append(held[there].abs().amax(0))
            counts.append(int(there.sum()))
    G = b.hq // b.hkv
    return torch.stack(rows).repeat_interleave(G, 1), torch.tensor(counts).double(), torch.stack(most).repeat_interleave(G, 1)


SHAPES = {"one": ([1, 1], [0, 500]), "few": ([3, 2, 1], [700, 30, 0]), "chunk": ([40, 1], [600, 90])}


@kinds
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("shape", list(SHAPES))
@pytest.mark.parametrize("power", [20, 24, 25, 26, 27, 28, 30, 34])
def test_ties_of_large_scores(q, flags, d, shape, power):
    """All blocks of V on one scale: equal weights for equal scores, whatever a step of the scores is.  The weights are equal powers of two (times a rounding that they share),
    so that the mean is off by the sums' roundings alone: 2^-22 of the magnitudes (sums of up to 600 values of 4 bits), and the weights' own, which the sum beside
    them may not share (2^-11 of fp16, 2^-8 of bf16)."""
    new, old = SHAPES[shape]
    for e, mant in ((-40, 1.0), (-3, 1.75), (0, 1.53), (40, 1.9)):
        b = one_channel(new, old, q, flags, 2.0 ** power * mant, [e], d)
        out, lse = b.attend()
        assert b.cache.sync_status() == 0
        want, count, most = visible_mean(b)
        rel = 2.0 ** -8 if b.wide or b.q_t == torch.bfloat16 else 2.0 ** -11
        got = out[:b.total].double().cpu()
        bound = most * (rel + 2.0 ** -20) * (1 + torch.finfo(b.q_t).eps / 2) + want.abs() * torch.finfo(b.q_t).eps / 2
        assert torch.isfinite(got).all() and ((got - want).abs() <= bound).all(), (e, mant, float((got - want).abs().max()), float(most.max()))
        s = b.q[:b.total, :, 0].double() / math.sqrt(d)
        exact = s + torch.log(count)[:, None]
        # the score: three products of fp32 and the sum's 2^-22; the exponents of scales and weights are added in steps of the score, three times at most; the logarithm 2^-20
        assert ((lse[:b.total].double().cpu() - exact).abs() <= exact.abs() * 2.0 ** -20 + 2.0 ** -18).all(), (e, mant)


@kinds
@pytest.mark.parametrize("shape", list(SHAPES))
@pytest.mark.parametrize("power", [22, 24, 25, 26, 27, 28, 30])
def test_large_scores_that_grow(q, flags, shape, power):
    """The largest keys come in the second half of the cache: what the first half left is behind, by far more than any exponent holds."""
    new, old = SHAPES[shape]
    b = one_channel(new, old, q, flags, 2.0 ** power * 1.37, [0], 64, fall=0.5)
    out, lse = b.attend()
    assert b.cache.sync_status() == 0 and torch.isfinite(out[:b.total]).all() and torch.isfinite(lse[:b.total]).all()
    want, _, most = visible_mean(b, fall=0.5)
    rows = torch.cat([torch.arange(o, o + n) >= (o + n) // 2 + 3 for n, o in zip(b.new, b.old)])   # (rows that see some of the second half)
    got = out[:b.total].double().cpu()
    bound = most * (2.0 ** -8 + 2.0 ** -20) + want.abs() * 2.0 ** -8
    assert ((got - want).abs() <= bound)[rows].all()


@kinds
@pytest.mark.parametrize("shape", list(SHAPES))
@pytest.mark.parametrize("power", [18, 24, 25, 26, 27, 28, 30, 33])
def test_large_scores_over_scales_of_all_sizes(q, flags, shape, power):
    """Blocks of V on scales of all sizes: scores are known to a step of fp32, more than the scales' exponents, so that any weights are right for those that tie: out lies
    between the values, and is finite."""
    new, old = SHAPES[shape]
    b = one_channel(new, old, q, flags, 2.0 ** power * 1.21, [-40, -17, -3, 0, 1, 16, 33, 40], 64)
    out, lse = b.attend()
    assert b.cache.sync_status() == 0 and torch.isfinite(out[:b.total]).all() and torch.isfinite(lse[:b.total]).all()
    _, _, most = visible_mean(b)
    assert (out[:b.total].double().cpu().abs() <= most * (1 + 2.0 ** -7)).all()


@pytest.mark.parametrize("what", ["inf", "nan"])
@pytest.mark.parametrize("q", ["bf16", "f32"])
def test_a_largest_score_that_is_not_finite(what, q):
    """NaN and infinity among the scores of a row make the row NaN, beside rows with large scores that stay finite."""
    for new, old in (([2], [40]), ([2, 3], [40, 700]), ([40, 1], [600, 90])):
        b = one_channel(new, old, q, 0, 2.0 ** 26, [0], 64)
        b.q[1, 2, 0] = math.inf if what == "inf" else math.nan
        b.put()
        out, lse = b.attend()
        bad = torch.zeros(b.total, b.hq, dtype=torch.bool)
        bad[1, 2] = True
        assert torch.equal(torch.isnan(out[:b.total]).any(-1).cpu(), bad) and torch.equal(torch.isnan(lse[:b.total]).cpu(), bad)
        assert torch.isnan(out[1, 2]).all()
