"""The 8-bit cache in a captured step that is replayed with other lengths, other tokens and other pages; rotated to positions of the caller's own."""
import random

import pytest
import torch

from paper_2601_22379_b200 import binding
from tests.test_gpu_paged_bytes import DEV, TYPES, Batch, ints

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("q,new,old,kw", [
    ("bf16", [1, 2, 1], [3000, 40, 0], {}), ("f32", [1, 2, 1], [3000, 40, 0], dict(softcap=9.0)), ("bf16", [60, 1, 3], [900, 2000, 40], dict(window=300, sinks=5)),
    ("bf16", [150, 40, 9], [30, 0, 100], {}), ("bf16", [150, 40, 9], [300, 700, 100], dict(window=90, sinks=3)), ("f32", [60, 1, 3], [900, 2000, 40], {}),
    ("bf16", [8, 3, 5], [700, 700, 100], {})], ids=["few", "few-f32", "chunk", "wide", "wide-window", "f32", "chunk-few"])
def test_other_lengths(q, new, old, kw):
    """Bounds, tensors and places stay; lengths, prefix sums and the page table change between replays: the same bits as an eager call with the same bounds."""
    b = Batch(new, old, hq=8, hkv=2, d=64, P=32, q=q)
    b.run(**kw)
    r = random.Random(len(new) + sum(new))
    with torch.cuda.stream(torch.cuda.Stream()):
        b.attend(**kw)
        torch.cuda.synchronize()
    out, lse = torch.empty_like(b.qd), torch.empty(b.rows, b.hq, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.attend(out=out, lse=lse, **kw)
    for _ in range(12):
        some, lens = [], []
        for s, n in enumerate(b.new):
            most = b.lens[s]
            n = r.choice([0, 1, n, r.randint(0, n)])
            some.append(n)
            lens.append(r.randint(n, most))
        order = [r.randrange(len(new)) if r.random() < 0.2 else s for s in range(len(new))]     # (sequences may share the pages that they read)
        order = [s if b.lens[o] < lens[s] else o for s, o in enumerate(order)]
        b.cu.copy_(ints([0] + torch.tensor(some).cumsum(0).tolist()))
        b.lens_t.copy_(ints(lens))
        b.table.copy_(b.table_cpu[order].to(DEV))
        out.fill_(5.0)
        lse.fill_(6.0)
        graph.replay()
        mine = torch.full_like(out, 5.0), torch.full_like(lse, 6.0)
        b.attend(out=mine[0], lse=mine[1], **kw)
        assert b.cache.sync_status() == 0
        total = sum(some)
        assert torch.equal(out, mine[0]) and torch.equal(lse, mine[1]) and (out[total:] == 5).all() and (lse[total:] == 6).all()
        assert torch.isfinite(out).all() and torch.isfinite(lse).all()
    # the last lengths against float64
    b.new, b.lens, b.total, b.table_cpu = some, lens, total, b.table_cpu[order]
    b.old = [x - n for x, n in zip(lens, some)]
    b.cu_cpu = b.cu.cpu()
    b.check(out, lse, **kw)


@pytest.mark.parametrize("q", ["bf16", "f32"])
@pytest.mark.parametrize("kv", ["e4m3", "same"])
def test_positions_of_the_callers(q, kv):
    """Keys and queries rotated to given positions (far, negative, all alike), wherever they are stored: as norm_apply turns them."""
    new, old, hq, hkv, d, P = [3, 40, 17], [5, 0, 30], 4, 2, 64, 16
    total, t = sum(new), TYPES[q]
    g = torch.Generator(device=DEV).manual_seed(7)
    x = torch.randn(total, hq + 2 * hkv, d, device=DEV, generator=g).to(t)
    wq, wk = 1 + 0.3 * torch.randn(d, device=DEV, generator=g), 1 + 0.3 * torch.randn(d, device=DEV, generator=g)
    rope = binding.Rope(d, base=500000.0)
    pos = torch.randint(-(1 << 30), 1 << 30, (total,), device=DEV, generator=g).to(torch.int32)
    pos[10:20] = 4
    lens = [a + b for a, b in zip(new, old)]
    table, cu = torch.arange(15, dtype=torch.int32, device=DEV).view(3, 5), ints([0, 3, 43, 60])
    if kv == "e4m3":
        cache = binding.PagedCache(n_q_heads=hq, q_dtype=q, **binding.PagedCache.pages(15, hkv, P, d))
    else:
        cache = binding.PagedCache(*(torch.zeros(15, hkv, P, d, dtype=t, device=DEV) for _ in range(2)), n_q_heads=hq)
    out = cache.append(x[:, hq:hq + hkv], x[:, hq + hkv:], cu, ints(lens), table, q=x[:, :hq], rope=rope, positions=pos, q_weight=wq, k_weight=wk, eps=1e-5)
    want_q, want_k = rope.norm_apply(pos, x[:, :hq], wq, x[:, hq:hq + hkv], wk, eps=1e-5)
    assert cache.sync_status() == 0 and torch.equal(out, want_q)
    k, v = cache.read(cu, ints(lens), table, total)
    if kv == "same":
        assert torch.equal(k, want_k) and torch.equal(v, x[:, hq + hkv:])
    else:
        # y, the value that is stored, is rounded to e4m3, half a step, 2^-4 of itself; want_k is y rounded to its type, off by u = eps / 2 of it (bf16 2^-8), |y| <= |want| (1 + 2 u):
        # 2^-4 (1 + 2 u) + 2 u of want.  Below 2^-6 of the scale the step is 2^-9 of it, and the scale is at most 2 / 448 of the largest: 2^-10 2^-7.8.
        u = torch.finfo(t).eps / 2
        want = want_k.double().abs()
        # (Rows 0 to 2 and 43, 44 go to blocks that were begun before, tokens 0 to 4 and 16 to 29, whose scale of 1 is kept: half a step there is 2^-10.)
        least = want.amax((0, 2), keepdim=True).repeat(total, 1, 1) * 2.0 ** -17
        least[[0, 1, 2, 43, 44]] = 2.0 ** -10
        assert ((k.double() - want_k.double()).abs() <= want * (2.0 ** -4 * (1 + 2 * u) + 2 * u) + least).all()
