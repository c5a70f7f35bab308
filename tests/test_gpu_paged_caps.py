"""Scales and caps far apart: capped scores that are exactly 0, saturated, or in between, whatever the scale."""
import math

import pytest
import torch

from paper_2601_22379_b200 import binding
from tests import paged_reference as ref
from tests.test_gpu_paged import DEV, Batch, kinds

pytestmark = pytest.mark.gpu


def _run(b, scale, **kw):
    cache = binding.PagedCache(b.kd, b.vd, n_q_heads=b.hq, q_dtype="bf16" if b.q_t == torch.bfloat16 else "f32", sm_scale=scale, flags=b.flags)
    out, lse = cache.attend(b.qd, b.cu, b.lens_t, b.table, b.max_new, b.max_len, **kw)
    assert cache.sync_status() == 0
    return out, lse


def _integers(b, size):
    """Queries and keys of -size, 0 and size: products exact, many of them 0; every fifth key is 0."""
    ints = lambda x: torch.randint(-1, 2, x.shape, generator=b.gen).to(x.dtype) * size  # noqa: E731
    b.q = ints(b.q)
    held = torch.isfinite(b.k)
    b.k = torch.where(held, ints(b.k), b.k)
    for s, x in enumerate(b.lens):
        j = torch.arange(0, x, 5)
        b.k[b.table_cpu[s].long()[j // b.P], :, j % b.P] = 0
    b.qd, b.kd = b.q.to(DEV), b.k.to(DEV)


@kinds
@pytest.mark.parametrize("new,old", [([1, 3], [400, 77]), ([150, 20], [100, 300])], ids=["few", "chunks"])
@pytest.mark.parametrize("scale,cap", [(4.0, 1e-6), (100.0, 1e-6), (1e4, 1e-2), (1e20, 3.0), (2e38, 1e-6), (1e30, 1e25)])
def test_saturated(kv, q, flags, new, old, scale, cap):
    """Every score is -cap, 0 or cap."""
    b = Batch(new, old, hq=4, hkv=2, d=64, P=32, kv=kv, q=q, flags=flags)
    b.flags = flags
    _integers(b, 1.0)
    out, lse = _run(b, scale, softcap=cap)
    if cap > 80:                                                              # e^-cap is nothing: the mean of the keys with the largest score
        for s in range(len(new)):
            assert bool(torch.isfinite(out[int(b.cu_cpu[s]):int(b.cu_cpu[s + 1])].float()).all())
        return
    for s, L in enumerate(b.lens):
        n, r0 = b.new[s], int(b.cu_cpu[s])
        seen = torch.arange(L) <= torch.arange(L - n, L)[:, None]
        for m in range(4):
            k, v = ref.gather(b.k, b.table_cpu[s], L, m // 2).double(), ref.gather(b.v, b.table_cpu[s], L, m // 2).double()
            x = b.q[r0:r0 + n, m].double() @ k.T
            p = torch.where(seen, torch.exp(cap * torch.sign(x)), torch.zeros_like(x))
            w = p / p.sum(-1, keepdim=True)
            # a score off by 2^-21 of the cap, an exponential by 2^-20, a probability (bf16) by half a step
            mass, e = w @ v.abs(), 2 * (cap * 2.0 ** -21 + 2.0 ** -20) + (2.0 ** -8 if b.tensor_cores else 0.0)
            ref.check(out[r0:r0 + n, m], w @ v, e * mass, b.q_t, "out")
            ref.check(lse[r0:r0 + n, m], torch.log(p.sum(-1)), torch.full((n,), cap * 2.0 ** -21 + 2.0 ** -20) + 2.0 ** -22 * torch.log(p.sum(-1)).abs(), what="lse")


@kinds
@pytest.mark.parametrize("new,old", [([1, 3], [400, 77]), ([150, 20], [100, 300])], ids=["few", "chunks"])
def test_small_products_and_a_large_scale(kv, q, flags, new, old):
    """Products of n 2^-26 and a scale of 2^26: scores of a few units, capped at 8."""
    b = Batch(new, old, hq=4, hkv=2, d=64, P=32, kv=kv, q=q, flags=flags)
    b.flags = flags
    _integers(b, 2.0 ** -13)
    out, lse = _run(b, 2.0 ** 26, softcap=8.0)
    b.check(out, lse, sm_scale=2.0 ** 26, softcap=8.0)


@kinds
def test_a_cap_that_caps_nothing(kv, q, flags):
    b = Batch([1, 150], [300, 20], hq=4, hkv=2, d=64, P=32, kv=kv, q=q, flags=flags)
    b.flags = flags
    out, lse = _run(b, 0.125, softcap=3e38)
    b.check(out, lse, sm_scale=0.125, softcap=0.0)
    assert math.isfinite(float(lse.sum()))
