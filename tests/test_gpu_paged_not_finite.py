"""Visible keys and values that are not finite: what the documentation says of each, on every kernel."""
import math

import pytest
import torch

from tests import paged_reference as ref
from tests.test_gpu_paged import DEV, Batch, kinds

pytestmark = pytest.mark.gpu

cases = pytest.mark.parametrize("new,old", [([1, 3, 1], [300, 5, 0]), ([150, 40, 1], [200, 0, 0])], ids=["few", "chunks"])


def _first_key(b, value):
    """The first token of every sequence gets an infinite channel in head 1; the queries' channel has either sign."""
    for s in range(len(b.new)):
        b.k[int(b.table_cpu[s, 0]), 1, 0, 3] = value
    b.kd.copy_(b.k)
    b.q[:, :, 3] = torch.where(torch.arange(b.rows)[:, None] % 3 == 0, -1.0, 1.5).to(b.q_t)
    b.qd = b.q.to(DEV)
    return b.q[:, 2:, 3].float() * (1.0 if value > 0 else -1.0) < 0          # rows and heads whose score of that key is -infinity


@kinds
@cases
@pytest.mark.parametrize("bad", [math.inf, -math.inf])
@pytest.mark.parametrize("slopes", [False, True])
def test_infinite_scores(kv, q, flags, new, old, bad, slopes):
    """+infinity spoils the row, -infinity is weight 0."""
    b = Batch(new, old, hq=4, hkv=2, d=64, P=32, kv=kv, q=q, flags=flags)
    kw = dict(slopes=torch.tensor([0.5, 0.0, 0.25, 0.0])) if slopes else {}
    low = _first_key(b, bad)
    out, lse = b.attend(**kw)
    assert b.cache.sync_status() == 0
    clean = torch.where(torch.isinf(b.k), torch.zeros_like(b.k), b.k)
    o0, l0, ob0, lb0 = ref.attend(b.q, clean, b.v, b.cu_cpu, b.lens, b.table_cpu, tensor_cores=b.tensor_cores, **kw)
    o1, l1, ob1, lb1 = ref.attend(b.q, clean, b.v, b.cu_cpu, b.lens, b.table_cpu, tensor_cores=b.tensor_cores, first_key=torch.ones(b.rows, dtype=torch.int32), **kw)
    for h in (0, 1):                                                          # heads of the other key are as ever
        ref.check(out[:, h], o0[:, h], ob0[:, h], b.q_t, "out")
        ref.check(lse[:, h], l0[:, h], lb0[:, h], what="lse")
    got, got_lse = out[:, 2:].cpu(), lse[:, 2:].cpu()
    assert bool(torch.isnan(got[~low]).all()) and bool(torch.isnan(got_lse[~low]).all())
    ref.check(got[low], o1[:, 2:][low], ob1[:, 2:][low], b.q_t, "out without the key")
    ref.check(got_lse[low], l1[:, 2:][low], lb1[:, 2:][low], what="lse without the key")
    # a row with that key alone: nothing left
    at = int(b.cu_cpu[2])
    for h in (0, 1):
        if low[at, h]:
            assert bool((got[at, h] == 0).all()) and float(got_lse[at, h]) == -math.inf


@kinds
@cases
@pytest.mark.parametrize("bad", [math.inf, -math.inf])
def test_infinite_scores_under_a_cap(kv, q, flags, new, old, bad):
    """An infinite score is the cap: as with a key of a huge finite score."""
    b = Batch(new, old, hq=4, hkv=2, d=64, P=32, kv=kv, q=q, flags=flags)
    _first_key(b, bad)
    out, lse = b.attend(softcap=2.0)
    assert b.cache.sync_status() == 0
    huge = torch.where(torch.isinf(b.k), torch.full_like(b.k, math.copysign(4096.0, bad)), b.k)
    o, l, ob, lb = ref.attend(b.q, huge, b.v, b.cu_cpu, b.lens, b.table_cpu, tensor_cores=b.tensor_cores, softcap=2.0)
    # (the bound counts the huge score's rounding as if it went through: 4096 x 1.5 / 8 x 72 2^-24 = 3e-3 in that key's weight)
    ref.check(out, o, ob, b.q_t, "out")
    ref.check(lse, l, lb, what="lse")


@kinds
@cases
@pytest.mark.parametrize("cap", [0.0, 2.0])
def test_nan_keys_and_values(kv, q, flags, new, old, cap):
    """A key of NaN spoils the rows of its heads; a value that is not finite the channels that it is in."""
    b = Batch(new, old, hq=4, hkv=2, d=64, P=32, kv=kv, q=q, flags=flags)
    base, base_lse = b.attend(softcap=cap)
    page = int(b.table_cpu[0, 0])
    k, v = b.kd.clone(), b.vd.clone()
    b.kd[page, 1, 0, 3] = math.nan
    out, lse = b.attend(softcap=cap)
    mine = slice(0, b.new[0])
    assert torch.isnan(out[mine, 2:]).all() and torch.isnan(lse[mine, 2:]).all()
    assert torch.equal(out[mine, :2], base[mine, :2]) and torch.equal(out[b.new[0]:], base[b.new[0]:]) and torch.equal(lse[b.new[0]:], base_lse[b.new[0]:])
    b.kd.copy_(k)
    for bad in (math.inf, -math.inf, math.nan):
        b.vd.copy_(v)
        b.vd[page, 1, 0, 7] = bad
        out, lse = b.attend(softcap=cap)
        assert not torch.isfinite(out[mine, 2:, 7]).any()
        assert torch.isfinite(out[mine, 2:, :7]).all() and torch.isfinite(out[mine, 2:, 8:]).all() and torch.isfinite(out[b.new[0]:]).all()
        assert torch.equal(lse, base_lse)
    assert b.cache.sync_status() == 0
