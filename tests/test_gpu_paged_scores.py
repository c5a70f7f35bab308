"""Attention on the tensor cores with scores far beyond what fp32 counts in steps of one: bf16 pages, and 8-bit pages whose keys and values are widened to bf16."""
import math

import pytest
import torch

from paper_2601_22379_b200 import binding
from tests import test_gpu_paged_bytes as bytes8
from tests.test_gpu_paged_bytes_scores import one_channel, visible_mean

pytestmark = pytest.mark.gpu
POWERS = [24, 28, 29, 30, 31, 32, 33, 34, 40, 60]


def check(got, lse, want, most, exact):
    """Equal weights for equal scores.  Off by the weights' rounding, 2^-8, the sums', and that of out; lse by three products of fp32 and the weights' own size, a step of the score."""
    bound = most * (2.0 ** -8 + 2.0 ** -20) * (1 + 2.0 ** -8) + want.abs() * 2.0 ** -8
    got = got.double().cpu()
    assert torch.isfinite(got).all() and ((got - want).abs() <= bound).all()
    assert ((lse.double().cpu() - exact).abs() <= exact.abs() * 2.0 ** -20 + 2.0 ** -18).all()


@pytest.mark.parametrize("power", POWERS)
@pytest.mark.parametrize("mant", [1.0, 1.3, 1.77])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new,old", [([1, 1], [0, 500]), ([3, 1], [40, 700]), ([150], [0]), ([200, 30], [100, 900])], ids=["one", "few", "prompt", "chunk"])
def test_bf16_pages(power, mant, d, new, old):
    """Every third key is 1, the others -1; and the same with a cap that is none and with sinks."""
    lens, P, hq, hkv = [a + b for a, b in zip(new, old)], 64, 4, 2
    g = torch.Generator().manual_seed(power)
    cols = -(-max(lens) // P)
    table = torch.randperm(len(lens) * cols, generator=g).to(torch.int32).view(len(lens), cols)
    k, v = torch.zeros(table.numel(), hkv, P, d), torch.randn(table.numel(), hkv, P, d, generator=g).to(torch.bfloat16)
    total = sum(new)
    q = torch.zeros(total, hq, d)
    q[..., 0] = 2.0 ** power * mant * math.log(2.0) * math.sqrt(d)
    q = q.to(torch.bfloat16)
    want, most, count = [], [], []
    for b, (n, o) in enumerate(zip(new, old)):
        at = torch.arange(lens[b])
        page = table[b].long()[at // P]
        k[page, :, at % P, 0] = torch.where(at % 3 == 0, 1.0, -1.0)[:, None]
        held = v[page, :, at % P].double()
        for i in range(n):
            some = held[(at % 3 == 0) & (at < o + i + 1)]
            want.append(some.mean(0))
            most.append(some.abs().amax(0))
            count.append(some.shape[0])
    want, most = (torch.stack(x).repeat_interleave(hq // hkv, 1) for x in (want, most))
    exact = q[..., 0].double() / math.sqrt(d) + torch.log(torch.tensor(count).double())[:, None]
    dev = lambda x: x.to(bytes8.DEV)  # noqa: E731
    cache = binding.PagedCache(dev(k.to(torch.bfloat16)), dev(v), n_q_heads=hq)
    cu = bytes8.ints([0] + torch.tensor(new).cumsum(0).tolist())
    for kw in ({}, dict(window=100000, sinks=3), dict(slopes=torch.zeros(hq, device=bytes8.DEV))):
        out, lse = cache.attend(dev(q), cu, bytes8.ints(lens), dev(table), max(new), max(lens), **kw)
        assert cache.sync_status() == 0
        check(out, lse, want, most, exact)


@pytest.mark.parametrize("power", POWERS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("ev", [-40, 0, 40])
def test_8_bit_prompts(power, d, ev):
    b = one_channel([150], [0], "bf16", 0, 2.0 ** power * 1.53, [ev], d)
    out, lse = b.attend()
    assert b.wide and b.cache.sync_status() == 0
    want, count, most = visible_mean(b)
    check(out, lse, want, most, b.q[:b.total, :, 0].double() / math.sqrt(d) + torch.log(count)[:, None])


def test_rows_of_all_sizes():
    """Rows with scores of 1 beside rows with scores of 2^33, each as alone."""
    b = one_channel([150], [0], "bf16", 0, 2.0 ** 33 * 1.53, [0], 128)
    large, large_lse = b.attend()
    big = b.q[:, :, 0].clone()
    b.q[1::2, :, 0] = 1.0
    b.put()
    out, lse = b.attend()
    assert torch.equal(out[::2], large[::2]) and torch.equal(lse[::2], large_lse[::2]) and torch.isfinite(out).all() and torch.isfinite(lse).all()
    b.q[:, :, 0] = 1.0
    b.put()
    small, small_lse = b.attend()
    assert torch.equal(out[1::2], small[1::2]) and torch.equal(lse[1::2], small_lse[1::2])
    assert float(big.abs().max()) > 2.0 ** 33
