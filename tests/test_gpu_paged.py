"""The paged cache: appending (with the rotation on the way) and attention over it, against plain float64 forms."""
import math
import os
import random

import pytest
import torch

from paper_2601_22379_b200 import binding
from tests import paged_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
GENERAL = binding.SPLA_GENERAL_KERNELS


class Batch:
    """Sequences with `new` tokens each on top of `old` ones, pages anywhere in the pool, queries, cache contents.  Memory that
    belongs to no sequence (rows behind a sequence's end, spare pages, rows behind the last sequence) holds NaN."""

    def __init__(self, new, old, hq=4, hkv=2, d=128, P=64, kv="bf16", q=None, seed=0, extra_rows=0, extra_cols=0, scale=1.5, flags=0):
        g = torch.Generator().manual_seed(seed)
        self.new, self.old, self.lens = new, old, [a + b for a, b in zip(new, old)]
        self.hq, self.hkv, self.d, self.P = hq, hkv, d, P
        self.kv_t, self.q_t = TYPES[kv], TYPES[q or kv]
        B, total = len(new), sum(new)
        self.total, self.rows = total, total + extra_rows
        need = [-(-x // P) for x in self.lens]
        n_pages = sum(need) + 3
        order = torch.randperm(n_pages, generator=g)
        table = torch.full((B, max(max(need), 1) + extra_cols), -7, dtype=torch.int32)
        at = 0
        for b, m in enumerate(need):
            table[b, :m] = order[at:at + m]
            at += m
        self.table_cpu = table
        self.k = torch.full((n_pages, hkv, P, d), math.nan, dtype=self.kv_t)
        self.v = torch.full((n_pages, hkv, P, d), math.nan, dtype=self.kv_t)
        for b, x in enumerate(self.lens):
            j = torch.arange(x)
            self.k[table[b].long()[j // P], :, j % P] = torch.randn(x, hkv, d, generator=g).to(self.kv_t)
            self.v[table[b].long()[j // P], :, j % P] = torch.randn(x, hkv, d, generator=g).to(self.kv_t)
        self.q = torch.full((self.rows, hq, d), math.nan, dtype=self.q_t)
        self.q[:total] = (scale * torch.randn(total, hq, d, generator=g)).to(self.q_t)
        self.cu_cpu = torch.tensor([0] + torch.tensor(new).cumsum(0).tolist(), dtype=torch.int32)
        self.cu, self.lens_t, self.table = self.cu_cpu.to(DEV), torch.tensor(self.lens, dtype=torch.int32, device=DEV), table.to(DEV)
        self.kd, self.vd, self.qd = self.k.to(DEV), self.v.to(DEV), self.q.to(DEV)
        self.max_new, self.max_len = max(max(new), 1), max(max(self.lens), 1)
        self.cache = binding.PagedCache(self.kd, self.vd, n_q_heads=hq, q_dtype="bf16" if self.q_t == torch.bfloat16 else "f32", flags=flags)
        self.tensor_cores = self.kv_t == self.q_t == torch.bfloat16 and not flags
        self.gen = g

    def attend(self, q=None, **kw):
        put = {x: kw.pop(x).to(DEV) for x in ("slopes", "first_key", "prefix_lens") if kw.get(x) is not None}
        max_new, max_len = kw.pop("max_new", self.max_new), kw.pop("max_len", self.max_len)
        return self.cache.attend(self.qd if q is None else q, self.cu, self.lens_t, self.table, max_new, max_len, **put, **kw)

    def check(self, out, lse, seqs=None, **kw):
        kw["prefix"] = kw.pop("prefix_lens", None)
        o, l, ob, lb = ref.attend(self.q[:self.total], self.k, self.v, self.cu_cpu, self.lens, self.table_cpu, tensor_cores=self.tensor_cores, seqs=seqs, **kw)
        ref.check(lse[:self.total], l, lb, what="lse")
        ref.check(out[:self.total], o, ob, self.q_t, "out")

    def run(self, **kw):
        out, lse = self.attend(**kw)
        assert self.cache.sync_status() == 0
        self.check(out, lse, **kw)
        return out, lse


KINDS = [("bf16", "bf16", 0), ("bf16", "bf16", GENERAL), ("f32", "f32", 0), ("bf16", "f32", 0), ("f32", "bf16", 0)]
kinds = pytest.mark.parametrize("kv,q,flags", KINDS, ids=["bf16", "bf16-general", "f32", "bf16-q32", "f32-q16"])


@kinds
@pytest.mark.parametrize("d,P", [(128, 64), (64, 16), (128, 128), (64, 32), (128, 16), (64, 128)])
@pytest.mark.parametrize("new,old", [([1], [0]), ([1, 1, 1], [0, 63, 64]), ([1, 1], [127, 500]), ([5, 0, 1, 33], [0, 3, 700, 130]), ([150, 2], [40, 1000]), ([0, 0, 7], [5, 0, 0])],
                         ids=["one", "page-ends", "tile-ends", "ragged", "chunk", "empty"])
def test_attend(kv, q, flags, d, P, new, old):
    Batch(new, old, d=d, P=P, kv=kv, q=q, flags=flags).run()


@kinds
@pytest.mark.parametrize("hq,hkv", [(1, 1), (6, 2), (5, 1), (7, 1), (16, 1), (8, 8), (24, 2)])
def test_groups(kv, q, flags, hq, hkv):
    Batch([1, 3, 140, 17], [300, 0, 5, 250], hq=hq, hkv=hkv, d=64, P=32, kv=kv, q=q, flags=flags).run()


@kinds
@pytest.mark.parametrize("mask", ["cap", "slopes", "window", "window-1", "documents", "prefix", "all"])
@pytest.mark.parametrize("d", [64, 128])
def test_masks(kv, q, flags, mask, d):
    """Every mask; documents whose start lies behind a token (its row is empty), prefixes beyond the end."""
    b = Batch([1, 70, 9, 1, 200], [400, 300, 0, 65, 31], hq=4, hkv=2, d=d, P=32, kv=kv, q=q, flags=flags, extra_cols=2)
    first = torch.cat([torch.arange(o, o + n, dtype=torch.int32) // 50 * 50 for n, o in zip(b.new, b.old)])
    first[::7] = 10000                                                        # sees nothing (unless the prefix lets it: it does not, the start holds)
    first[1::7] = -5
    kw = {"cap": dict(softcap=5.0), "slopes": dict(slopes=torch.tensor([0.5, 0.0, 0.01, 2.0])), "window": dict(window=37), "window-1": dict(window=1),
          "documents": dict(first_key=first), "prefix": dict(prefix_lens=torch.tensor([0, 340, 5, 10000, 100], dtype=torch.int32)),
          "all": dict(softcap=8.0, slopes=torch.tensor([0.25, 0.125, 0.0, 1.0]), window=90, first_key=first,
                      prefix_lens=torch.tensor([390, 350, 7, 0, 60], dtype=torch.int32))}[mask]
    b.run(**kw)


@kinds
@pytest.mark.parametrize("mask", ["cap", "cap-high", "slopes", "window", "documents", "prefix", "all"])
@pytest.mark.parametrize("hq,d", [(4, 128), (16, 64), (10, 64)])
def test_masks_of_few_tokens(kv, q, flags, mask, hq, d):
    """The same where no sequence has more than three new tokens."""
    b = Batch([1, 2, 3, 1, 0, 1], [400, 300, 0, 65, 31, 1000], hq=hq, hkv=2, d=d, P=32, kv=kv, q=q, flags=flags, extra_cols=2)
    first = torch.tensor([200, 10000, 290, 1, -5, 2, 66, 999], dtype=torch.int32)
    slopes = torch.arange(hq) % 4 * 0.25
    kw = {"cap": dict(softcap=5.0), "cap-high": dict(softcap=3000.0), "slopes": dict(slopes=slopes), "window": dict(window=37), "documents": dict(first_key=first),
          "prefix": dict(prefix_lens=torch.tensor([0, 340, 5, 10000, 3, 100], dtype=torch.int32)),
          "all": dict(softcap=8.0, slopes=slopes, window=90, first_key=first, prefix_lens=torch.tensor([390, 350, 7, 0, 0, 60], dtype=torch.int32))}[mask]
    b.run(**kw)


@kinds
def test_cold_and_busy(kv, q, flags):
    """The same bits whether the inputs are in the cache or not, whatever the scratch held before."""
    batches = [Batch([1, 1, 2, 130], [20000, 17, 5001, 9000], hq=8, hkv=2, d=128, P=64, kv=kv, q=q, flags=flags),
               Batch([1, 1, 2, 3], [9000, 17, 5001, 300], hq=8, hkv=2, d=128, P=64, kv=kv, q=q, flags=flags),
               Batch([200, 170, 300], [1000, 300, 0], hq=8, hkv=2, d=64, P=16, kv=kv, q=q, flags=flags)]
    flush = torch.empty(200 << 20, dtype=torch.uint8, device=DEV)
    first = [b.run() for b in batches]
    for it in range(30):
        for b, (o, l) in zip(batches, first):
            if it % 3 == 1:
                flush.fill_(it)
            torch.full((8 << 20,), math.nan, device=DEV)
            out, lse = b.attend()
            assert torch.equal(out, o) and torch.equal(lse, l), it


def test_waits_that_run_out():
    """Copies that never complete: the kernel gives up, reports it, and works again afterwards."""
    for new in ([1, 2], [150, 40]):
        b = Batch(new, [500, 900], hq=8, hkv=2, d=128, kv="bf16")
        want, want_lse = b.run()
        b.cache.debug_wait_hook(1 << 14, 16)
        b.attend()
        assert b.cache.sync_status() == binding.SPLA_ERR_TIMEOUT
        b.cache.debug_wait_hook(0, 0)
        out, lse = b.attend()
        assert b.cache.sync_status() == 0 and torch.equal(out, want) and torch.equal(lse, want_lse)


@pytest.mark.parametrize("kv", ["bf16", "f32"])
def test_offsets_past_32_bits(kv):
    """A pool of more than 2^32 elements, the sequences in its last pages and its first."""
    t = TYPES[kv]
    hkv, P, d = 8, 128, 128
    n_pages = (1 << 32) // (hkv * P * d) + 7
    kp, vp = (torch.empty(n_pages, hkv, P, d, dtype=t, device=DEV) for _ in range(2))
    table = torch.tensor([[n_pages - 1, 0, n_pages - 2], [n_pages - 3, n_pages - 4, 5]], dtype=torch.int32)
    lens, new = [300, 260], [300, 260]
    g = torch.Generator().manual_seed(2)
    k, v, q = (torch.randn(560, h, d, generator=g).to(t) for h in (hkv, hkv, 16))
    cu, ln, tb = torch.tensor([0, 300, 560], dtype=torch.int32, device=DEV), torch.tensor(lens, dtype=torch.int32, device=DEV), table.to(DEV)
    cache = binding.PagedCache(kp, vp, n_q_heads=16)
    cache.append(k.to(DEV), v.to(DEV), cu, ln, tb)
    out, lse = cache.attend(q.to(DEV), cu, ln, tb, 300, 300)
    assert cache.sync_status() == 0
    small_k, small_v = torch.zeros(6, hkv, P, d, dtype=t), torch.zeros(6, hkv, P, d, dtype=t)
    own = torch.arange(6, dtype=torch.int32).view(2, 3)
    for s in range(2):
        j = torch.arange(lens[s])
        small_k[own[s].long()[j // P], :, j % P] = k[int(cu[s]):int(cu[s]) + lens[s]]
        small_v[own[s].long()[j // P], :, j % P] = v[int(cu[s]):int(cu[s]) + lens[s]]
    o, l, ob, lb = ref.attend(q, small_k, small_v, cu.cpu(), lens, own, tensor_cores=kv == "bf16")
    ref.check(lse, l, lb, what="lse")
    ref.check(out, o, ob, t, "out")


@kinds
def test_long(kv, q, flags):
    """Long sequences beside short ones: units cut between many CTAs, joined in order; twice the same bits."""
    b = Batch([1, 1, 2, 130], [20000, 17, 5001, 9000], hq=8, hkv=2, d=128, P=64, kv=kv, q=q, flags=flags)
    out, lse = b.run()
    out2, lse2 = b.attend()
    assert torch.equal(out, out2) and torch.equal(lse, lse2)


@kinds
def test_bounds_may_be_loose(kv, q, flags):
    """max_new and max_len are bounds: larger ones change the division of the work, not the results."""
    b = Batch([1, 4, 40], [130, 77, 300], d=64, P=16, kv=kv, q=q, flags=flags, extra_cols=40)
    for kw in (dict(max_new=45), dict(max_len=900), dict(max_new=45, max_len=900)):
        out, lse = b.attend(**kw)
        assert b.cache.sync_status() == 0
        b.check(out, lse)


@kinds
def test_strided_queries(kv, q, flags):
    """Queries inside a packed projection; a stride or address that is no multiple of 16 bytes as well."""
    b = Batch([3, 20], [50, 100], hq=4, hkv=2, d=64, kv=kv, q=q, flags=flags)
    want, _ = b.run()
    for pad, at in ((128, 0), (128, 64), (4, 0), (1, 0), (8, 3)):
        wide = torch.full((b.rows, 4 * 64 + pad + at), math.nan, dtype=b.q_t, device=DEV)
        view = wide[:, at:at + 256].unflatten(1, (4, 64))
        view.copy_(b.qd)
        out, lse = b.attend(q=view)
        b.check(out, lse)


@kinds
def test_rows_behind_the_last_sequence(kv, q, flags):
    b = Batch([2, 30], [10, 60], d=64, kv=kv, q=q, flags=flags, extra_rows=5)
    out = torch.full((b.rows, b.hq, b.d), 7.0, dtype=b.q_t, device=DEV)
    lse = torch.full((b.rows, b.hq), 7.0, device=DEV)
    b.attend(out=out, lse=lse)
    assert b.cache.sync_status() == 0
    b.check(out, lse)
    assert bool((out[b.total:] == 7).all()) and bool((lse[b.total:] == 7).all())


@kinds
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("new,hit", [([60, 1, 140], (130, 100, 77)), ([3, 1, 2], (101, 100, 77)), ([3, 1, 1], (102, 141, 220))], ids=["chunks", "few", "few-edges"])
def test_not_finite_values_of_hidden_keys(kv, q, flags, bad, new, hit):
    """Values and keys that are not finite, of later tokens, before the window, in other documents: rows that do not see them are as without."""
    b = Batch(new, [100, 260, 0 if new[2] > 100 else 218], hq=4, hkv=2, d=128, kv=kv, q=q, flags=flags)
    b.run(window=120)
    want, want_lse, bound, lse_bound = ref.attend(b.q, b.k, b.v, b.cu_cpu, b.lens, b.table_cpu, window=120, tensor_cores=b.tensor_cores)
    hit = {s: t for s, t in enumerate(hit) if t < b.lens[s]}                  # sequence: token
    k, v = b.k.clone(), b.v.clone()
    for s, t in hit.items():
        page = int(b.table_cpu[s, t // b.P])
        v[page, :, t % b.P, 5] = bad
        k[page, 1, t % b.P, 3] = bad
    b.kd.copy_(k)
    b.vd.copy_(v)
    out, lse = b.attend(window=120)
    assert b.cache.sync_status() == 0
    for s, t in hit.items():
        for i in range(b.new[s]):
            pos, row = b.old[s] + i, int(b.cu_cpu[s]) + i
            if pos - 120 < t <= pos:                                          # sees it: the value's channel, and the heads that the key belongs to
                assert not bool(torch.isfinite(out[row, :2, 5]).any())
                want[row, :2, 5] = math.nan                                   # (left out of the comparison)
                want[row, 2:] = want_lse[row, 2:] = math.nan
    ref.check(lse, want_lse, lse_bound, what="lse")
    ref.check(out, want, bound, b.q_t, "out")


@kinds
def test_not_finite_scores_of_a_row(kv, q, flags):
    """A query of NaN spoils its own rows and no others."""
    b = Batch([3, 1], [200, 10], hq=4, hkv=2, d=64, kv=kv, q=q, flags=flags)
    base, base_lse = b.run()
    q2 = b.qd.clone()
    q2[1, 2, 0] = math.nan
    out, lse = b.attend(q=q2)
    assert torch.isnan(out[1, 2]).all() and torch.isnan(lse[1, 2])
    keep = torch.ones(b.rows, 4, dtype=torch.bool)
    keep[1, 2] = False
    assert torch.equal(out.cpu()[keep], base.cpu()[keep]) and torch.equal(lse.cpu()[keep], base_lse.cpu()[keep])


@kinds
def test_large_scores(kv, q, flags):
    """Scores far apart: one key takes all, others underflow."""
    b = Batch([1, 40], [300, 200], hq=4, hkv=2, d=64, kv=kv, q=q, flags=flags, scale=60.0)
    b.run()


@kinds
def test_inconsistent_sequences_and_pages(kv, q, flags):
    """A sequence whose numbers do not fit together is skipped, a page number outside the pool reads as zeros: both reported, the others served."""
    b = Batch([2, 3, 4, 5], [70, 100, 200, 90], d=64, P=32, kv=kv, q=q, flags=flags)
    good, _ = b.run()
    out = torch.full_like(good, 7.0)
    lens = b.lens_t.clone()
    lens[1] = 2                                                               # shorter than its own new tokens
    o, _ = b.cache.attend(b.qd, b.cu, lens, b.table, b.max_new, b.max_len, out=out)
    assert b.cache.sync_status() == binding.SPLA_ERR_BOUNDS and b.cache.sync_status() == 0
    assert bool((o[2:5] == 7).all()) and torch.equal(o[:2], good[:2]) and torch.equal(o[5:], good[5:])
    lens[1] = b.max_len + 1
    b.cache.attend(b.qd, b.cu, lens, b.table, b.max_new, b.max_len, out=out)
    assert b.cache.sync_status() == binding.SPLA_ERR_BOUNDS
    b.cache.attend(b.qd, b.cu, b.lens_t, b.table, 4, b.max_len, out=out)       # max_new too small for the last sequence
    assert b.cache.sync_status() == binding.SPLA_ERR_BOUNDS and bool((out[:9] == good[:9]).all())
    for page in (-1, 10 ** 6, b.kd.shape[0]):
        table = b.table.clone()
        table[2, 1] = page
        o, lse = b.cache.attend(b.qd, b.cu, b.lens_t, table, b.max_new, b.max_len)
        assert b.cache.sync_status() == binding.SPLA_ERR_BOUNDS
        assert torch.equal(o[:5], good[:5]) and torch.equal(o[9:], good[9:])
        k, v, t = torch.cat([b.k, torch.zeros_like(b.k[:1])]), torch.cat([b.v, torch.zeros_like(b.v[:1])]), b.table_cpu.clone()
        t[2, 1] = b.k.shape[0]
        want, l, ob, lb = ref.attend(b.q, k, v, b.cu_cpu, b.lens, t, tensor_cores=b.tensor_cores, seqs=[2])
        ref.check(o, want, ob, b.q_t)
        ref.check(lse, l, lb)


@kinds
def test_streams_and_graphs(kv, q, flags):
    """Calls on two streams at once and a captured call, replayed with other contents beside an eager one: no scratch is shared."""
    b = Batch([1, 1, 66], [4000, 30, 900], hq=8, hkv=2, d=128, kv=kv, q=q, flags=flags)
    want, want_lse = b.run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    results = []
    for _ in range(5):
        results.append(b.attend())
        with torch.cuda.stream(side):
            results.append(b.attend())
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) and torch.equal(l, want_lse) for o, l in results)
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            res = b.attend()
        graphs.append((g, res))
    q2 = (b.qd.float() * 0.5).to(b.q_t)
    b.qd.copy_(q2)
    for _ in range(3):
        with torch.cuda.stream(side):
            graphs[0][0].replay()
        graphs[1][0].replay()
    torch.cuda.synchronize()
    o, l = b.attend()
    b.q = q2.cpu()
    b.check(o, l)
    for _, (go, gl) in graphs:
        assert torch.equal(go, o) and torch.equal(gl, l)


@kinds
def test_many_sequences(kv, q, flags):
    """More sequences than a launch's table holds."""
    n = 1100
    g = torch.Generator().manual_seed(3)
    new = torch.randint(0, 3, (n,), generator=g).tolist()
    old = torch.randint(0, 40, (n,), generator=g).tolist()
    b = Batch(new, old, hq=2, hkv=1, d=64, P=16, kv=kv, q=q, flags=flags)
    b.run()


def test_two_threads():
    """Calls from two threads, each on its own stream: the handle holds nothing that a call changes."""
    import threading
    b = Batch([1, 1, 66], [4000, 30, 900], hq=8, hkv=2, d=128, kv="bf16")
    want, want_lse = b.run()
    wrong = []

    def work():
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            for _ in range(40):
                out, lse = b.attend()
                stream.synchronize()
                if not (torch.equal(out, want) and torch.equal(lse, want_lse)):
                    wrong.append(1)

    threads = [threading.Thread(target=work) for _ in range(2)]
    [t.start() for t in threads]
    [t.join() for t in threads]
    assert not wrong


@pytest.mark.parametrize("seed", [int(os.environ.get("SPLA_FUZZ_OFFSET", "0")) + i for i in range(60)])
def test_drawn(seed):
    """Anything the documentation allows, at once."""
    r = random.Random(9000 + seed)
    kv, q, flags = r.choice([KINDS[0]] * 4 + KINDS[1:])
    B, hkv, G, d, P = r.choice([1, 2, 3, 7, 20, 33]), r.choice([1, 2, 3]), r.choice([1, 2, 3, 4, 5, 7, 8, 11, 16]), r.choice([64, 128]), r.choice([16, 32, 64, 128])
    few = r.random() < 0.5
    new = [r.choice([0, 1, 1, r.randint(1, 3 if few else 150)]) for _ in range(B)]
    if not sum(new):
        new[0] = 1
    old = [r.choice([0, r.randint(0, 30), r.randint(0, 700), r.randint(0, 3000)]) for _ in range(B)]
    b = Batch(new, old, hq=G * hkv, hkv=hkv, d=d, P=P, kv=kv, q=q, flags=flags, seed=seed, extra_rows=r.choice([0, 3]), extra_cols=r.choice([0, 5]))
    kw = {}
    if r.random() < 0.3:
        kw["softcap"] = r.choice([1.0, 5.0, 30.0, 500.0])
    if r.random() < 0.3:
        kw["window"] = r.choice([1, 2, 17, 128, 400])
    if r.random() < 0.3:
        kw["slopes"] = torch.tensor([r.choice([0.0, 0.01, 0.3, 2.0]) for _ in range(G * hkv)])
    if r.random() < 0.3:
        kw["first_key"] = torch.tensor([max(-1, r.choice([0, p, p - r.randint(0, 200), p + 1])) for n, o in zip(new, old) for p in range(o, o + n)] + [0] * (b.rows - b.total),
                                       dtype=torch.int32)
    if r.random() < 0.3:
        kw["prefix_lens"] = torch.tensor([r.choice([0, 5, 100, 5000]) for _ in range(B)], dtype=torch.int32)
    bounds = dict(max_new=b.max_new + r.choice([0, 0, 40]), max_len=min(b.max_len + r.choice([0, 0, 300]), b.table.shape[1] * P))
    bounds["max_new"] = min(bounds["max_new"], bounds["max_len"])
    out, lse = b.attend(**kw, **bounds)
    assert b.cache.sync_status() == 0
    b.check(out, lse, **{k: (v[:b.total] if k == "first_key" else v) for k, v in kw.items()})
    again, lse2 = b.attend(**kw, **bounds)
    assert torch.equal(out[:b.total], again[:b.total]) and torch.equal(lse[:b.total], lse2[:b.total])


# ---- append ---------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("kv,q", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("d,P,rope", [(128, 64, dict()), (64, 16, dict(rot_dim=32, interleaved=True)), (128, 32, None), (64, 128, dict(rot_dim=6, amplitude=1.2))])
@pytest.mark.parametrize("packed", [False, True])
def test_append(kv, q, d, P, rope, packed):
    """New tokens to their pages, keys rotated, queries beside them; everything else in the pool stays as it was."""
    b = Batch([1, 0, 40, 7, 130], [0, 9, 25, 64, 511], hq=4, hkv=2, d=d, P=P, kv=kv, q=q, extra_rows=3)
    g = torch.Generator().manual_seed(11)
    n = b.rows
    if packed and kv == q:
        qkv = torch.randn(n, 4 + 2 * 2 + 1, d, generator=g).to(b.kv_t).to(DEV)
        qq, k, v = qkv[:, :4], qkv[:, 4:6], qkv[:, 6:8]
    else:
        qq, k, v = (torch.randn(n, h, d, generator=g).to(t).to(DEV) for h, t in ((4, b.q_t), (2, b.kv_t), (2, b.kv_t)))
    r = binding.Rope(d, **rope) if rope is not None else None
    q_out = torch.full((n, 4, d), 7.0, dtype=b.q_t, device=DEV)
    assert b.cache.append(k, v, b.cu, b.lens_t, b.table, q=qq, rope=r, q_out=q_out) is q_out
    assert b.cache.sync_status() == 0
    a = dict(rope or {})
    rot, inter, amp = a.get("rot_dim", d), a.get("interleaved", False), a.get("amplitude", 1.0)
    pos = torch.cat([torch.arange(o, o + m) for m, o in zip(b.new, b.old)])
    kk, vv = k[:b.total].cpu(), v[:b.total].cpu()
    if rope is None:
        wk, ek, wq, eq = kk.double(), torch.zeros_like(kk, dtype=torch.float64), qq[:b.total].double().cpu(), torch.zeros(b.total, 4, d, dtype=torch.float64)
    else:
        f = ref.frequencies(rot)
        wk, ek = ref.rotate(kk, pos, rot, inter, f, amp)
        wq, eq = ref.rotate(qq[:b.total], pos, rot, inter, f, amp)
    ref.check(q_out[:b.total], wq, eq, b.q_t)
    assert bool((q_out[b.total:] == 7).all())
    want_k, want_v, bound_k = b.k.double(), b.v.clone(), torch.zeros_like(b.k, dtype=torch.float64)
    at = 0
    for s, (m, o) in enumerate(zip(b.new, b.old)):
        j = torch.arange(o, o + m)
        page = b.table_cpu[s].long()[j // P]
        want_k[page, :, j % P] = wk[at:at + m]
        bound_k[page, :, j % P] = ek[at:at + m]
        want_v[page, :, j % P] = vv[at:at + m]
        at += m
    ref.check(b.kd, want_k, bound_k, b.kv_t)
    same = lambda x, y: torch.equal(torch.nan_to_num(x.cpu().float(), nan=1e9), torch.nan_to_num(y.float(), nan=1e9))  # noqa: E731
    assert same(b.vd, want_v) and torch.equal(torch.isnan(b.kd.cpu()), torch.isnan(want_k))
    if rope is not None:                                                      # positions of one's own, queries in place, the same bits from the rotation alone
        own = torch.arange(n, dtype=torch.int32, device=DEV) * 3
        alone = r.apply(own, qq)
        qi = qq.clone() if not packed else qq
        assert b.cache.append(k, v, b.cu, b.lens_t, b.table, q=qi, rope=r, positions=own, q_out=qi) is qi
        assert torch.equal(qi[:b.total], alone[:b.total])


@pytest.mark.parametrize("hq,hkv", [(1, 1), (4, 1)])
def test_append_of_many_tokens_of_few_heads(hq, hkv):
    """Blocks of many tokens across sequences of a few, empty ones among them."""
    g = torch.Generator().manual_seed(7)
    new = torch.randint(0, 60, (150,), generator=g).tolist()
    b = Batch(new, torch.randint(0, 70, (150,), generator=g).tolist(), hq=hq, hkv=hkv, d=128, P=16, extra_rows=9)
    k, v, q = (torch.randn(b.rows, h, 128, generator=g).to(torch.bfloat16).to(DEV) for h in (hkv, hkv, hq))
    r = binding.Rope(128)
    out = b.cache.append(k, v, b.cu, b.lens_t, b.table, q=q, rope=r)
    assert b.cache.sync_status() == 0
    pos = torch.cat([torch.arange(o, o + n) for n, o in zip(b.new, b.old)])
    f = ref.frequencies(128)
    wq, eq = ref.rotate(q[:b.total].cpu(), pos, 128, False, f)
    wk, ek = ref.rotate(k[:b.total].cpu(), pos, 128, False, f)
    ref.check(out[:b.total], wq, eq, torch.bfloat16)
    seq = torch.repeat_interleave(torch.arange(150), torch.tensor(b.new))
    page = b.table_cpu[seq, pos // 16].long()
    ref.check(b.kd.cpu()[page, :, pos % 16], wk, ek, torch.bfloat16)
    assert torch.equal(b.vd.cpu()[page, :, pos % 16], v[:b.total].cpu())


def test_append_skips_what_does_not_fit():
    b = Batch([2, 3, 4], [30, 10, 60], d=64, P=32)
    k = torch.randn(9, 2, 64, device=DEV).bfloat16()
    lens = b.lens_t.clone()
    lens[0] = 1
    table = b.table.clone()
    table[2, 1] = -1                                                          # tokens 60 .. 63 of the last sequence lie there
    before_k, before_v = b.kd.clone(), b.vd.clone()
    b.cache.append(k, k, b.cu, lens, table)
    assert b.cache.sync_status() == binding.SPLA_ERR_BOUNDS
    page = int(b.table_cpu[1, 0])
    before_k[page, :, 10:13] = k[2:5].transpose(0, 1)
    before_v[page, :, 10:13] = k[2:5].transpose(0, 1)
    eq = lambda x, y: torch.equal(torch.nan_to_num(x.float(), nan=1e9), torch.nan_to_num(y.float(), nan=1e9))  # noqa: E731
    assert eq(b.kd, before_k) and eq(b.vd, before_v)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_run_of_them(dtype):
    """A prompt in two chunks and decode steps, rotated, stored and attended to, against one dense pass over all tokens."""
    hq, hkv, d, P, total = 8, 2, 64, 16, 90
    t = TYPES[dtype]
    g = torch.Generator().manual_seed(4)
    q, k, v = (torch.randn(2, total, h, d, generator=g).to(t) for h in (hq, hkv, hkv))
    pages = torch.randperm(2 * 6, generator=g).to(torch.int32).view(2, 6).to(DEV)
    kp = torch.full((12, hkv, P, d), math.nan, dtype=t, device=DEV)
    vp = torch.full((12, hkv, P, d), math.nan, dtype=t, device=DEV)
    cache, rope = binding.PagedCache(kp, vp, n_q_heads=hq), binding.Rope(d, interleaved=True)
    outs = torch.zeros(2, total, hq, d)
    at = 0
    for step in (41, 30, 1, 1, 1, 16):
        rows = lambda x: x[:, at:at + step].reshape(2 * step, -1, d).to(DEV)  # noqa: E731
        cu = torch.tensor([0, step, 2 * step], dtype=torch.int32, device=DEV)
        lens = torch.full((2,), at + step, dtype=torch.int32, device=DEV)
        rq = cache.append(rows(k), rows(v), cu, lens, pages, q=rows(q), rope=rope)
        out, _ = cache.attend(rq, cu, lens, pages, step, at + step)
        outs[:, at:at + step] = out.float().cpu().view(2, step, hq, d)
        at += step
    assert at == total and cache.sync_status() == 0
    pos, f = torch.arange(total), ref.frequencies(d)
    rq, _ = ref.rotate(q, pos.expand(2, total), d, True, f)
    rk, _ = ref.rotate(k, pos.expand(2, total), d, True, f)
    rq, rk = rq.to(t).double(), rk.to(t).double()                             # (stored in their type)
    x = torch.einsum("bihd,bjhd->bhij", rq, rk.repeat_interleave(hq // hkv, 2)) / math.sqrt(d)
    w = torch.softmax(x.masked_fill(pos[None, :] > pos[:, None], -math.inf), -1)
    vv = v.double().repeat_interleave(hq // hkv, 2)
    want = torch.einsum("bhij,bjhd->bihd", w, vv)
    mass = torch.einsum("bhij,bjhd->bihd", w, vv.abs())
    # bf16: a rotated value may round to its neighbour (a step of 2^-7): scores of 64 terms of size one are off by 64 x 2^-8 / 8
    # in the sum of magnitudes at worst and a tenth of it in fact; probability and output are rounded too.  fp32: 2^-24 in place of 2^-8
    eps = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    assert bool(((outs.double() - want).abs() <= eps * (8 * mass + want.abs()) + 1e-6).all())


@pytest.mark.parametrize("kv", ["bf16", "f32"])
def test_over_an_spla_cache(kv):
    """Dense attention over an SPLA cache as it lies: the same as its own decode step with every block selected."""
    B, hq, hkv, d, T = 3, 8, 2, 128, 300
    cfg = binding.make_config(batch=B, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, block_size=64, top_k=8, max_context=512, kv_dtype=kv, flags=binding.SPLA_NO_RLA)
    cache = binding.SplaCache(cfg, DEV)
    g = torch.Generator(device=DEV).manual_seed(1)
    t = TYPES[kv]
    k, v = (torch.randn(B, hkv, T, d, device=DEV, generator=g).to(t) for _ in range(2))
    q = torch.randn(B, hq, d, device=DEV, generator=g).to(t)
    n_new = torch.tensor([300, 1, 129], dtype=torch.int32, device=DEV)
    cache.append_tokens(k, v, n_new)
    want = cache.decode(q, None)
    pages = binding.PagedCache.of(cache)
    cu = torch.arange(B + 1, dtype=torch.int32, device=DEV)
    out, _ = pages.attend(q, cu, cache.bufs.seq_lens, pages.table(), 1, 512)
    assert pages.sync_status() == 0
    # both within rounding of the exact result: an output of bf16 by 2^-8 of itself, probabilities in bf16 by 2^-8 of the values' mean magnitude (below 1)
    lim = 2.0 ** -8 * (want.abs() + 2) if kv == "bf16" else torch.full_like(want, 1e-5)
    assert bool(((out.float() - want).abs() <= lim).all())
