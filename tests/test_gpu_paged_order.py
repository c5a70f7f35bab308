"""Prefix sums that do not ascend: a row of the new tokens belongs to one sequence at most, the same one in every call."""
import random

import pytest
import torch

from paper_2601_22379_b200 import binding
from tests import paged_reference as ref
from tests.test_gpu_paged import DEV, Batch, kinds
from tests.test_paged_division import _sound, _spoilt

pytestmark = pytest.mark.gpu


def _batch(seed, kind, B, **kw):
    r = random.Random(seed)
    cu, total = _spoilt(r, B, kind)
    b = Batch([3] * B, [r.choice([1, 20, 60, 90]) for _ in range(B)], hq=2, hkv=1, d=64, P=32, **kw)
    if total > b.rows:
        b.q = torch.cat([b.q, torch.randn(total - b.rows, 2, 64, generator=b.gen).to(b.q_t)])
    b.q = torch.nan_to_num(b.q[:total], nan=1.0)
    b.qd, b.cu_cpu = b.q.to(DEV), torch.tensor(cu, dtype=torch.int32)
    b.cu = b.cu_cpu.to(DEV)
    own, served = _sound(cu, b.lens, total, min(total, b.max_len), b.max_len)
    return b, total, own, [s for s in range(B) if served[s]]


@kinds
@pytest.mark.parametrize("kind", ["one", "far", "several", "shuffled", "alternating"])
@pytest.mark.parametrize("B", [5, 45, 500])
def test_attend_serves_rows_once(kv, q, flags, kind, B):
    b, total, own, served = _batch(B + len(kind), kind, B, kv=kv, q=q, flags=flags)
    out, lse = torch.full((total, 2, 64), 7.0, dtype=b.q_t, device=DEV), torch.full((total, 2), 7.0, device=DEV)
    b.attend(max_new=min(total, b.max_len), out=out, lse=lse)
    assert b.cache.sync_status() == (0 if all(own) else binding.SPLA_ERR_BOUNDS)
    few = served if B < 100 else served[:20] + served[-20:]
    o, l, ob, lb = ref.attend(b.q, b.k, b.v, b.cu_cpu, b.lens, b.table_cpu, tensor_cores=b.tensor_cores, seqs=few)
    ref.check(lse, l, lb, what="lse")
    ref.check(out, o, ob, b.q_t, "out")
    mine = torch.zeros(total, dtype=torch.bool)
    for s in served:
        mine[int(b.cu_cpu[s]):int(b.cu_cpu[s + 1])] = True
    assert bool((out[~mine.to(DEV)] == 7).all()) and bool((lse[~mine.to(DEV)] == 7).all())


@pytest.mark.parametrize("kind", ["one", "far", "several", "shuffled", "alternating"])
@pytest.mark.parametrize("B", [5, 45, 500])
def test_append_stores_rows_once(kind, B):
    b, total, own, served = _batch(B + len(kind), kind, B)
    k, v = (torch.randn(total, 1, 64, generator=b.gen).bfloat16() for _ in range(2))
    want_k, want_v = b.k.clone(), b.v.clone()
    q_out = torch.full((total, 2, 64), 7.0, dtype=torch.bfloat16, device=DEV)
    want_q = q_out.cpu()
    for s in served:
        r0, r1 = int(b.cu_cpu[s]), int(b.cu_cpu[s + 1])
        if r1 == r0:
            continue
        j = torch.arange(b.lens[s] - (r1 - r0), b.lens[s])
        page = b.table_cpu[s].long()[j // b.P]
        want_k[page, :, j % b.P] = k[r0:r1]
        want_v[page, :, j % b.P] = v[r0:r1]
        want_q[r0:r1] = b.q[r0:r1]
    b.cache.append(k.to(DEV), v.to(DEV), b.cu, b.lens_t, b.table, q=b.qd, q_out=q_out)
    # (the append's own bounds are the page table's: the lengths here are within the attention's, too)
    assert b.cache.sync_status() == (0 if all(own) else binding.SPLA_ERR_BOUNDS)
    eq = lambda x, y: torch.equal(torch.nan_to_num(x.cpu().float(), nan=1e9), torch.nan_to_num(y.float(), nan=1e9))  # noqa: E731
    assert eq(b.kd, want_k) and eq(b.vd, want_v) and eq(q_out, want_q)
