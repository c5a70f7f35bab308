"""Attention over a long paged cache: what the tensor cores add up stays as exact as the documentation says, however many keys there are."""
import math
import random

import pytest
import torch

from paper_2601_22379_b200 import binding
from tests import paged_reference as ref
from tests.test_gpu_paged import Batch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("sequences,new,G", [(1, 148 * 16, 16), (148, 1, 8)], ids=["chunk", "single"])
def test_sums_of_four_million_keys(d, sequences, new, G):
    """All keys alike, so that the result is the mean of the values: every unit is walked by one CTA from end to end."""
    L, P = 1 << 22, 128
    g = torch.Generator(device=DEV).manual_seed(1)
    k = torch.zeros(L // P, 1, P, d, device=DEV, dtype=torch.bfloat16)
    v = (torch.rand(L // P, 1, P, d, device=DEV, generator=g) + 0.5).to(torch.bfloat16)
    table = torch.arange(L // P, dtype=torch.int32, device=DEV).expand(sequences, -1).contiguous()
    q = torch.randn(sequences * new, G, d, device=DEV, generator=g).to(torch.bfloat16)
    cu = torch.arange(sequences + 1, dtype=torch.int32, device=DEV) * new
    lens = torch.full((sequences,), L, dtype=torch.int32, device=DEV)
    cache = binding.PagedCache(k, v, n_q_heads=G)
    out, lse = cache.attend(q, cu, lens, table, new, L, prefix_lens=lens)
    assert cache.sync_status() == 0
    want = v.view(-1, d).double().mean(0)
    # scores of 0: probabilities of 1, products exact.  1024 additions that truncate by less than 2^-23 of the sum between two drains; 256 drains, the
    # sum of l in as many parts, and the division round by 2^-24 each; the output by half a step
    err = 2.0 ** -13 + (256 + 256 + 8) * 2.0 ** -24
    assert float((out.double() / want - 1).abs().max()) <= err + (1 + err) * 2.0 ** -8
    assert abs(float((out.double() / want - 1).mean())) <= err + 2.0 ** -8 / 4     # (and the roundings of many outputs go either way)
    assert float((lse.double() - math.log(L)).abs().max()) <= 2.0 ** -22 * (1 + math.log(L))


def _rising(b, top):
    """Keys whose scores grow along the sequence, so that the running maximum moves again and again."""
    for s, x in enumerate(b.lens):
        j = torch.arange(x)
        page = b.table_cpu[s].long()[j // b.P]
        grow = (1 + top * j.double() / x).to(b.kv_t)
        b.k[page, :, j % b.P] = (b.k[page, :, j % b.P].double() * grow.double()[:, None, None]).to(b.kv_t)
    b.kd.copy_(b.k)


@pytest.mark.parametrize("d,hq,hkv", [(64, 4, 1), (128, 5, 1)])
@pytest.mark.parametrize("new,old", [([150], [40000]), ([40, 1], [33000, 70]), ([3], [70000]), ([70], [16384 - 70]), ([130], [16384 - 100])],
                         ids=["two-row-tiles", "one-row-tile", "few", "no-drain", "just-one"])
@pytest.mark.parametrize("mask", ["causal", "cap", "window"])
def test_walks_that_are_drained(d, hq, hkv, new, old, mask):
    """More tiles than are added up in one go, with maxima that move before and after.  One KV head and copies of the sequence keep all CTAs busy, so that a
    unit's walk is long."""
    copies = 160 if len(new) == 1 else 80
    b = Batch(new, old, hq=hq, hkv=hkv, d=d, P=128)
    _rising(b, 3.0)
    kw = {"causal": {}, "cap": dict(softcap=20.0), "window": dict(window=30000)}[mask]
    n = b.total
    cu = torch.cat([b.cu_cpu[:-1].long() + n * i for i in range(copies)] + [torch.tensor([n * copies])]).to(torch.int32).to(DEV)
    q = b.qd.repeat(copies, 1, 1)
    out, lse = b.cache.attend(q, cu, b.lens_t.repeat(copies), b.table.repeat(copies, 1), b.max_new, b.max_len, **kw)
    assert b.cache.sync_status() == 0
    o, l, ob, lb = ref.attend(b.q, b.k, b.v, b.cu_cpu, b.lens, b.table_cpu, tensor_cores=True, **kw)
    # (truncations between two drains: 2^-13 of the values' mean magnitude, a 32nd of what the probabilities' rounding may add)
    for i in (0, 1, copies // 2, copies - 1):
        ref.check(lse[i * n:(i + 1) * n], l, lb, what="lse")
        ref.check(out[i * n:(i + 1) * n], o, ob * (1 + 2.0 ** -5), b.q_t, "out")
    again, lse2 = b.cache.attend(q, cu, b.lens_t.repeat(copies), b.table.repeat(copies, 1), b.max_new, b.max_len, **kw)
    assert torch.equal(out, again) and torch.equal(lse, lse2)


@pytest.mark.parametrize("old", [16384 - 140, 16384 - 1, 32768 - 100, 32768 + 20])
@pytest.mark.parametrize("new", [150, 40])
def test_not_finite_values_just_after_a_drain(new, old):
    """Values that are not finite, of later tokens, in the first tiles after the sums were taken away."""
    copies = 160
    b = Batch([new], [old], hq=2, hkv=1, d=128, P=128)
    cu = (torch.arange(copies + 1, dtype=torch.int32) * new).to(DEV)
    args = (b.qd.repeat(copies, 1, 1), cu, b.lens_t.repeat(copies), b.table.repeat(copies, 1), b.max_new, b.max_len)
    o, l, ob, lb = ref.attend(b.q, b.k, b.v, b.cu_cpu, b.lens, b.table_cpu, tensor_cores=True)
    hit = old + new // 2                                                      # seen by the second half of the new tokens
    b.vd[int(b.table_cpu[0, hit // b.P]), 0, hit % b.P, 5] = math.nan
    out, lse = b.cache.attend(*args)
    assert b.cache.sync_status() == 0
    assert bool(torch.isnan(out.view(copies, new, 2, 128)[:, new // 2:, :, 5]).all())
    o[new // 2:, :, 5] = math.nan                                             # (left out of the comparison)
    for i in (0, copies - 1):
        ref.check(lse[i * new:(i + 1) * new], l, lb, what="lse")
        ref.check(out[i * new:(i + 1) * new], o, ob * (1 + 2.0 ** -5), b.q_t, "out")


@pytest.mark.parametrize("kv", ["bf16", "f32"])
@pytest.mark.parametrize("few", [True, False])
def test_bounds_whose_tiles_pass_32_bits(kv, few):
    """Bounds so loose that the tiles which they allow pass 2^31: the work is dealt out in 64 bits, the results are the same within rounding."""
    g = torch.Generator().manual_seed(5)
    n = 384
    new = torch.randint(0, 3 if few else 70, (n,), generator=g).tolist()
    old = torch.randint(0, 900, (n,), generator=g).tolist()
    hkv = 64
    b = Batch(new, old, hq=hkv, hkv=hkv, d=64, P=128, kv=kv, extra_cols=(1 << 24) // 128 - 8)
    assert hkv * n * (1 << 24) // 128 > 1 << 31
    tight, tight_lse = b.attend()
    out, lse = b.attend(max_len=1 << 24)
    assert b.cache.sync_status() == 0
    some = [0, 1, 2, 200, n - 2, n - 1]
    b.check(out, lse, seqs=some)
    b.check(tight, tight_lse, seqs=some)
    # (both within half a step of the type and the probabilities' rounding of the same numbers: values' mean magnitude below 1)
    lim = 2.0 ** -8 * (tight.float().abs() + 2) * 2 if kv == "bf16" else torch.full_like(tight, 1e-5)
    assert bool(((out.float() - tight.float()).abs() <= lim).all()) and float((lse - tight_lse).abs().max()) < 1e-5


@pytest.mark.parametrize("seed", range(40))
def test_drawn_with_the_bounds_of_a_long_cache(seed):
    """Anything the documentation allows, with bounds that let a sequence be 20000 to 200000 tokens long, as a program plans that serves any length."""
    r = random.Random(400 + seed)
    B, hkv, G, d, P = r.choice([1, 2, 5, 40]), r.choice([1, 2, 3]), r.choice([1, 2, 4, 5, 8, 16]), r.choice([64, 128]), r.choice([16, 64, 128])
    few = r.random() < 0.5
    new = [r.choice([0, 1, r.randint(1, 2 if few else 200)]) for _ in range(B)]
    new[0] = new[0] or 1
    old = [r.choice([0, r.randint(0, 700), r.randint(0, 3000), 17000 if B < 5 else 100]) for _ in range(B)]
    top = r.choice([20000, 200000])
    b = Batch(new, old, hq=G * hkv, hkv=hkv, d=d, P=P, seed=seed, extra_cols=top // P)
    kw = {}
    if r.random() < 0.3:
        kw["softcap"] = r.choice([5.0, 30.0])
    if r.random() < 0.3:
        kw["window"] = r.choice([1, 200, 16500])
    if r.random() < 0.3:
        kw["slopes"] = torch.tensor([r.choice([0.0, 0.01, 0.3]) for _ in range(G * hkv)])
    if r.random() < 0.3:
        kw["first_key"] = torch.tensor([max(-1, r.choice([0, p, p - r.randint(0, 200), p + 1])) for n, o in zip(new, old) for p in range(o, o + n)], dtype=torch.int32)
    if r.random() < 0.3:
        kw["prefix_lens"] = torch.tensor([r.choice([0, 100, 18000]) for _ in range(B)], dtype=torch.int32)
    bounds = dict(max_len=max(top, b.max_len))
    out, lse = b.attend(**kw, **bounds)
    assert b.cache.sync_status() == 0
    b.check(out, lse, **kw)
    again, lse2 = b.attend(**kw, **bounds)
    assert torch.equal(out, again) and torch.equal(lse, lse2)


@pytest.mark.parametrize("new,old", [([1, 2], [500, 900]), ([150, 40], [500, 900]), ([150] * 40, [20000] * 40)], ids=["few", "chunks", "drained"])
def test_waits_that_run_out_in_a_long_cache(new, old):
    """As for short ones: the kernel gives up, reports it, and works again afterwards."""
    b = Batch(new, old, hq=8, hkv=2, d=128, kv="bf16", extra_cols=40000 // 64)
    want, want_lse = b.attend(max_len=40000)
    assert b.cache.sync_status() == 0
    b.check(want, want_lse, seqs=[0, 1])
    b.cache.debug_wait_hook(1 << 14, 16)
    b.attend(max_len=40000)
    assert b.cache.sync_status() == binding.SPLA_ERR_TIMEOUT
    b.cache.debug_wait_hook(0, 0)
    out, lse = b.attend(max_len=40000)
    assert b.cache.sync_status() == 0 and torch.equal(out, want) and torch.equal(lse, want_lse)


def test_graphs_of_a_long_cache():
    """Two captured calls whose walks are drained, replayed at once, beside an eager one: each has sums of its own."""
    b = Batch([130] * 20, [34000] * 20, hq=8, hkv=1, d=64, P=128)
    want, want_lse = b.attend()
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            res = b.attend()
        graphs.append((g, res))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        with torch.cuda.stream(side):
            graphs[0][0].replay()
        graphs[1][0].replay()
        out, lse = b.attend()
    torch.cuda.synchronize()
    assert b.cache.sync_status() == 0 and torch.equal(out, want) and torch.equal(lse, want_lse)
    for _, (go, gl) in graphs:
        assert torch.equal(go, want) and torch.equal(gl, want_lse)
