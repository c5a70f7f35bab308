"""The 8-bit paged cache: what is stored, bit for bit, what is read back, and the attention over it, against plain float64 forms."""
import math
import os
import random

import pytest
import torch

from paper_2601_22379_b200 import binding
from tests import paged_bytes_reference as ref8
from tests import paged_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
GENERAL = binding.SPLA_GENERAL_KERNELS
KINDS = [("bf16", 0), ("bf16", GENERAL), ("f32", 0)]
kinds = pytest.mark.parametrize("q,flags", KINDS, ids=["bf16", "general", "f32"])


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def on_device(pages, scales):
    return pages.to(DEV).view(torch.float8_e4m3fn), scales.to(DEV).view(torch.float8_e8m0fnu)


def widened(batch, total, hq, hkv, d, max_new, max_len, first_key=None, window=0, sinks=0):
    """Whether keys and values are widened to bf16: where they take at most four times the memory of the queries in two parts of 8 bits, or eight where there are
    512 rows a sequence; with a window its tiles only."""
    max_new, cols = min(max_new, total), -(-max_len // 128)
    slots = min(cols, -(-sinks // 128) + -(-(max_new + window - 1) // 128) + 1) if window else cols
    most = 8 if total * (hq // hkv) >= 512 * batch else 4
    return max_new * (hq // hkv) > 16 and first_key is None and 2 * batch * slots * hkv * 128 * d * 2 + 4 * batch * cols <= most * total * hq * (2 * d + 1)


class Batch:
    """Sequences with `new` tokens each on top of `old` ones, pages anywhere in the pool, blocks of different scales.  Memory that belongs to no sequence
    holds NaN, and the scales of such blocks 2^128."""

    def __init__(self, new, old, hq=4, hkv=2, d=128, P=64, q="bf16", flags=0, seed=0, extra_rows=0, extra_cols=0, spread=2, size=1.5, sm_scale=0.0):
        g = torch.Generator().manual_seed(seed)
        self.new, self.old, self.lens = new, old, [a + b for a, b in zip(new, old)]
        self.hq, self.hkv, self.d, self.P, self.q_t, self.flags, self.sm_scale = hq, hkv, d, P, TYPES[q], flags, sm_scale
        B, self.total = len(new), sum(new)
        self.rows = self.total + extra_rows
        need = [-(-x // P) for x in self.lens]
        n_pages = sum(need) + 3
        order = torch.randperm(n_pages, generator=g)
        table = torch.full((B, max(max(need), 1) + extra_cols), -7, dtype=torch.int32)
        at = 0
        for b, m in enumerate(need):
            table[b, :m] = order[at:at + m]
            at += m
        self.table_cpu = table
        self.bytes, self.scales = {}, {}
        for x in "kv":
            self.bytes[x] = torch.full((n_pages, hkv, P, d), 0x7f, dtype=torch.uint8)
            self.scales[x] = torch.full((n_pages, hkv, P // 16), 255, dtype=torch.uint8)
            for b, m in enumerate(self.lens):
                if m:
                    blocks = -(-m // 16)
                    y = torch.randn(blocks, hkv, 16, d, generator=g).double() * torch.pow(2.0, torch.randint(-spread, spread + 1, (blocks, hkv, 1, 1), generator=g).double())
                    e = ref8.exponent(y.abs().amax((-1, -2)))
                    held = ref8.e4m3(y * torch.pow(2.0, -e.double())[..., None, None]).view(torch.uint8)
                    j, i = torch.arange(m), torch.arange(blocks) * 16
                    self.bytes[x][table[b].long()[j // P], :, j % P] = held.transpose(1, 2).reshape(-1, hkv, d)[:m]
                    self.scales[x][table[b].long()[i // P], :, i % P // 16] = (e + 127).to(torch.uint8)
        self.q = torch.full((self.rows, hq, d), math.nan, dtype=self.q_t)
        self.q[:self.total] = (size * torch.randn(self.total, hq, d, generator=g)).to(self.q_t)
        self.cu_cpu = torch.tensor([0] + torch.tensor(new).cumsum(0).tolist(), dtype=torch.int32)
        self.cu, self.lens_t, self.table = self.cu_cpu.to(DEV), ints(self.lens), table.to(DEV)
        self.max_new, self.max_len = max(max(new), 1), max(max(self.lens), 1)
        self.wide = widened(B, self.rows, hq, hkv, d, self.max_new, self.max_len)
        self.put()

    def put(self):
        """(After a change of the CPU's copies.)"""
        self.kd, self.ks = on_device(self.bytes["k"], self.scales["k"])
        self.vd, self.vs = on_device(self.bytes["v"], self.scales["v"])
        self.qd = self.q.to(DEV)
        self.cache = binding.PagedCache(self.kd, self.vd, n_q_heads=self.hq, q_dtype="bf16" if self.q_t == torch.bfloat16 else "f32", flags=self.flags,
                                        k_scales=self.ks, v_scales=self.vs, sm_scale=self.sm_scale)

    def kernel(self, n):
        few = n * (self.hq // self.hkv) <= 16
        if self.flags or self.q_t == torch.float32:
            return "few32" if few and not self.flags else "general"
        return "wide" if self.wide else "few" if few else "chunk"

    def attend(self, q=None, **kw):
        put = {x: kw.pop(x).to(DEV) for x in ("slopes", "first_key", "prefix_lens") if kw.get(x) is not None}
        max_new, max_len = kw.pop("max_new", self.max_new), kw.pop("max_len", self.max_len)
        self.wide = widened(len(self.new), self.rows, self.hq, self.hkv, self.d, max_new, max_len, kw.get("first_key"), kw.get("window", 0), kw.get("sinks", 0))
        return self.cache.attend(self.qd if q is None else q, self.cu, self.lens_t, self.table, max_new, max_len, **put, **kw)

    def check(self, out, lse, seqs=None, none=False, kernel=None, **kw):
        kw["prefix"] = kw.pop("prefix_lens", None)
        k, v = (ref8.values(self.bytes[x], self.scales[x]) for x in "kv")
        inside = torch.cat([self.scales["v"][self.table_cpu[b, :-(-x // self.P)].long()].flatten() for b, x in enumerate(self.lens)] + [torch.zeros(1, dtype=torch.uint8)])
        exps = int(inside[inside < 255].max()) - 127
        o, l, ob, lb = ref8.attend(self.q[:self.total], k, v, self.cu_cpu, self.lens, self.table_cpu, kernel or self.kernel, exps, sm_scale=self.sm_scale or None, seqs=seqs, **kw)
        ref8.check(lse[:self.total], l, lb, what="lse", none=none)
        ref8.check(out[:self.total], o, ob, self.q_t, "out", none=none)

    def run(self, **kw):
        out, lse = self.attend(**kw)
        assert self.cache.sync_status() == 0
        self.check(out, lse, **kw)
        return out, lse


# ---- attention ------------------------------------------------------------------------------------------------------
@kinds
@pytest.mark.parametrize("d,P", [(128, 64), (64, 16), (128, 128), (64, 32), (128, 16), (64, 128)])
@pytest.mark.parametrize("new,old", [([1], [0]), ([1, 1, 1], [0, 63, 64]), ([1, 1], [127, 500]), ([5, 0, 1, 33], [0, 3, 700, 130]), ([150, 2], [40, 1000]), ([0, 0, 7], [5, 0, 0])],
                         ids=["one", "page-ends", "tile-ends", "ragged", "chunk", "empty"])
def test_attend(q, flags, d, P, new, old):
    Batch(new, old, d=d, P=P, q=q, flags=flags).run()


@kinds
@pytest.mark.parametrize("hq,hkv", [(1, 1), (6, 2), (5, 1), (7, 1), (16, 1), (8, 8), (24, 2), (9, 1), (8, 1)])
def test_groups(q, flags, hq, hkv):
    """Eight rows and sixteen, one more than each, row tiles that are not full."""
    Batch([1, 3, 140, 17], [300, 0, 5, 250], hq=hq, hkv=hkv, d=64, P=32, q=q, flags=flags).run()
    Batch([1, 2, 1], [300, 17, 1000], hq=hq, hkv=hkv, d=128, P=64, q=q, flags=flags, seed=1).run()


@kinds
@pytest.mark.parametrize("mask", ["cap", "cap-high", "slopes", "window", "window-1", "window-sinks", "sinks-1", "sinks-far", "documents", "prefix", "all", "all-sinks"])
@pytest.mark.parametrize("few", [False, True], ids=["mixed", "few"])
@pytest.mark.parametrize("d", [64, 128])
def test_masks(q, flags, mask, few, d):
    """Every mask; documents whose start lies behind a token (its row is empty), prefixes beyond the end, sinks beside windows near and far."""
    b = Batch([1, 3, 2, 1, 2] if few else [1, 70, 9, 1, 200], [400, 300, 0, 65, 31], hq=4, hkv=2, d=d, P=32, q=q, flags=flags, extra_cols=2)
    first = torch.cat([torch.arange(o, o + n, dtype=torch.int32) // 50 * 50 for n, o in zip(b.new, b.old)])
    first[::7] = 10000                                                        # sees nothing
    first[1::7] = -5
    slopes, prefix = torch.tensor([0.25, 0.125, 0.0, 1.0]), torch.tensor([390, 350, 7, 0, 60], dtype=torch.int32)
    b.run(**{"cap": dict(softcap=5.0), "cap-high": dict(softcap=200.0), "slopes": dict(slopes=torch.tensor([0.5, 0.0, 0.01, 2.0])), "window": dict(window=37),
             "window-1": dict(window=1), "window-sinks": dict(window=37, sinks=4), "sinks-1": dict(window=1, sinks=1), "sinks-far": dict(window=20, sinks=141),
             "documents": dict(first_key=first), "prefix": dict(prefix_lens=torch.tensor([0, 340, 5, 10000, 100], dtype=torch.int32)),
             "all": dict(softcap=8.0, slopes=slopes, window=90, first_key=first, prefix_lens=prefix),
             "all-sinks": dict(softcap=8.0, slopes=slopes, window=90, sinks=5, prefix_lens=prefix)}[mask])


@pytest.mark.parametrize("mask", ["none", "cap", "slopes", "window", "window-1", "window-sinks", "sinks-far", "prefix", "all"])
@pytest.mark.parametrize("d,P", [(128, 64), (64, 16), (128, 16), (64, 128)])
@pytest.mark.parametrize("new,old", [([300, 7, 1, 150], [0, 30, 90, 0]), ([129], [0]), ([700, 690], [20, 0]), ([4, 3, 1], [0, 9, 2])], ids=["ragged", "one", "two", "short"])
def test_prompts(mask, d, P, new, old):
    """Many rows for each key: keys and values are widened before.  Pages that no row's window reaches have no number."""
    b = Batch(new, old, hq=8, hkv=1, d=d, P=P, extra_cols=2, extra_rows=1)
    kw = {"none": {}, "cap": dict(softcap=5.0), "slopes": dict(slopes=torch.tensor([0.5, 0.0, 0.01, 2.0, 0.25, 0.125, 0.0, 1.0])), "window": dict(window=37), "window-1": dict(window=1),
          "window-sinks": dict(window=37, sinks=4), "sinks-far": dict(window=20, sinks=141), "prefix": dict(prefix_lens=torch.tensor([0, 20, 10000, 100][:len(new)], dtype=torch.int32)),
          "all": dict(softcap=8.0, slopes=torch.tensor([0.25, 0.125, 0.0, 1.0] * 2), window=90, sinks=5, prefix_lens=torch.tensor([290, 5, 0, 60][:len(new)], dtype=torch.int32))}[mask]
    b.run(**kw)
    assert b.wide == (sum(new) > 8)                                           # (eight tokens have too few rows)


def test_prompts_in_graphs_and_streams():
    """Captured calls hold their widened copies themselves: two graphs and an eager call on another stream at once, replayed with other tokens."""
    b = [Batch([300, 20 + 100 * x], [40, 0], hq=8, hkv=1, d=64, P=32, seed=x) for x in range(2)]
    want = [x.run() for x in b]
    assert all(x.wide for x in b)
    streams, graphs, outs = [torch.cuda.Stream() for _ in range(3)], [], []
    for x, s in zip(b, streams):
        with torch.cuda.stream(s):
            x.attend()
            s.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=s):
                outs.append(x.attend())
            graphs.append(g)
    for _ in range(3):
        for x, s, g in zip(b, streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
        with torch.cuda.stream(streams[2]):
            third = b[0].attend()
        torch.cuda.synchronize()
        for got, w in zip([*outs, third], [*want, want[0]]):
            assert all(torch.equal(p, r) for p, r in zip(got, w))
    for x in b:                                                               # other tokens in the same places
        x.kd.view(torch.uint8).copy_(x.kd.view(torch.uint8).flip(-1))
    for s, g in zip(streams, graphs):
        with torch.cuda.stream(s):
            g.replay()
    torch.cuda.synchronize()
    for x, got in zip(b, outs):
        x.bytes["k"] = x.kd.view(torch.uint8).cpu()
        x.check(*got)
        assert x.cache.sync_status() == 0


@pytest.mark.parametrize("sinks", [0, 100, 129])
def test_prompts_whose_first_pages_are_gone(sinks):
    """Pages before the window may have no number, or any, as long as no tile of 128 tokens that a row sees is in them."""
    b = Batch([300, 280], [700, 40], hq=8, hkv=1, d=64, P=32)
    b.table_cpu[0, -(-sinks // 128) * 4:16] = torch.tensor([-1, 1 << 30] * 8, dtype=torch.int32)[:16 - -(-sinks // 128) * 4]   # (token 700 sees from 601 on, tile 4)
    kept = b.table.clone()
    b.table = b.table_cpu.to(DEV)
    out, lse = b.attend(window=100, sinks=sinks)
    assert b.wide and b.cache.sync_status() == 0
    b.table_cpu = kept.cpu()
    b.check(out, lse, window=100, sinks=sinks)


@kinds
def test_sinks_of_a_long_cache(q, flags):
    """Tiles between the sinks' and the window's are passed over: one, many, none of them; more sinks than a window has."""
    for new, old, window, sinks in (([1, 2], [5000, 3000], 100, 4), ([1, 90], [5000, 3000], 300, 4), ([1, 130], [2000, 700], 128, 128), ([40], [1000], 50, 700), ([1], [1000], 50, 2000)):
        Batch(new, old, d=64, q=q, flags=flags).run(window=window, sinks=sinks)


@kinds
@pytest.mark.parametrize("spread", [0, 10])
def test_scales_of_blocks(q, flags, spread):
    """Blocks of one size and of sizes 2^20 apart."""
    Batch([1, 3, 70], [400, 300, 90], d=128, q=q, flags=flags, spread=spread, size=1.5 if spread == 0 else 2.0 ** -8).run()


@kinds
@pytest.mark.parametrize("ek,ev", [(-40, 40), (40, -40), (0, 0)])
def test_ends_of_the_scales(q, flags, ek, ev):
    """All blocks at one end of the range; queries that bring the scores back to an ordinary size."""
    b = Batch([1, 2, 40], [100, 300, 90], d=64, q=q, flags=flags, size=2.0 ** (-7 - ek))
    b.scales["k"].fill_(ek + 127)
    b.scales["v"].fill_(ev + 127)
    b.put()
    b.run()


@kinds
def test_scale_bytes_beyond_the_range(q, flags):
    """Read as the nearest that is inside."""
    b = Batch([1, 2, 40], [100, 300, 90], d=64, q=q, flags=flags, size=2.0 ** 32)
    b.scales["k"].fill_(3)
    b.scales["v"].fill_(250)
    b.put()
    k = dict(b.scales)
    out, lse = b.attend()
    b.scales = {"k": torch.full_like(k["k"], 127 - 40), "v": torch.full_like(k["v"], 127 + 40)}
    b.check(out, lse)


@kinds
@pytest.mark.parametrize("channels", [1, 3])
def test_outlier_channels(q, flags, channels):
    """A few channels of the queries 1000 times the others, which count all the same."""
    b = Batch([1, 2, 40], [100, 300, 90], d=128, q=q, flags=flags)
    b.q[:b.total, :, 5:5 + channels] *= 1000.0
    for page in b.bytes["k"]:
        page[:, :, 5:5 + channels] = 0
    b.put()
    b.run()


@kinds
@pytest.mark.parametrize("scale", [1e-6, 0.3, 40.0])
def test_score_scales(q, flags, scale):
    Batch([1, 2, 40], [100, 300, 90], d=64, q=q, flags=flags, sm_scale=scale, size=0.2).run()


@pytest.mark.parametrize("cap", [1e30, 3e38])
def test_a_cap_that_is_none(cap):
    """Up to the end of fp32: scores far below it stay what they are."""
    b = Batch([1, 2, 40], [100, 300, 90], d=64)
    out, lse = b.attend(softcap=cap)
    assert b.cache.sync_status() == 0
    b.check(out, lse)


@kinds
def test_what_a_row_does_not_see_does_not_touch_it(q, flags):
    """NaN among keys and values that some rows see and others do not: the former are NaN (one channel, for a value), the latter as ever."""
    for new, old in (([1, 1, 1], [10, 200, 300]), ([3, 2, 1], [10, 200, 300]), ([60, 3, 40], [10, 200, 300])):
        for window in (0, 25):
            b = Batch(new, old, hq=4, hkv=2, d=128, P=32, q=q, flags=flags)
            for s, n in enumerate(b.new):
                for what, back, channel in (("k", 0, None), ("v", 1, 77), ("v", 30, 5)):
                    at = b.lens[s] - 1 - back
                    page = int(b.table_cpu[s, at // b.P])
                    if what == "v" or s == 1:                                  # (a key: in the second sequence alone)
                        b.bytes[what][page, :, at % b.P, 9 if channel is None else channel] = 0x7f if s else 0xff
            b.put()
            out, lse = b.attend(window=window)
            assert b.cache.sync_status() == 0
            b.check(out, lse, none=True, window=window)


@pytest.mark.parametrize("what", ["inf", "-inf", "nan"])
@pytest.mark.parametrize("cap", [0.0, 4.0])
def test_queries_that_are_not_finite(what, cap):
    """An infinite score is weight 0 or makes the row NaN, under a cap it is the cap; other rows are as ever."""
    for new, old in (([1, 2], [40, 30]), ([40], [100])):
        b = Batch(new, old, d=64, hq=4, hkv=2, spread=0)
        for x in "kv":
            b.bytes[x][b.bytes[x] == 0x80] = 0
        page = b.bytes["k"]
        page[..., 3] = torch.where(page[..., 3] == 0x7f, page[..., 3], (page[..., 3] & 0x7f) | 8)   # a positive channel
        for r in range(b.total):
            b.q[r, r % 4, 3] = float(what)
        b.put()
        out, lse = b.attend(softcap=cap)
        b.check(out, lse, none=True, softcap=cap)


@kinds
def test_queries_of_any_stride_and_address(q, flags):
    """Queries inside a packed projection; an address and a stride that are no multiples of 16 bytes."""
    b = Batch([1, 3, 50], [100, 40, 9], hq=4, hkv=2, d=64, q=q, flags=flags)
    want, want_lse = b.run()
    wide = torch.zeros(b.total, 7, 64, dtype=b.q_t, device=DEV)
    wide[:, 2:6] = b.qd
    out, lse = b.attend(q=wide[:, 2:6])
    assert torch.equal(out, want) and torch.equal(lse, want_lse)
    for stride, offset in ((261, 0), (256, 1), (264, 3)):
        flat = torch.zeros(b.total * stride + 8, dtype=b.q_t, device=DEV)
        some = flat[offset:].as_strided((b.total, 4, 64), (stride, 64, 1), offset)
        some.copy_(b.qd)
        out, lse = b.attend(q=some)
        b.check(out, lse, kernel=lambda n: "general")


@kinds
def test_rows_behind_the_last_sequence_stay(q, flags):
    b = Batch([1, 40, 0], [50, 7, 3], q=q, flags=flags, extra_rows=5)
    out = torch.full_like(b.qd, 3.0)
    lse = torch.full((b.rows, b.hq), 4.0, device=DEV)
    b.attend(out=out, lse=lse)
    assert (out[b.total:] == 3).all() and (lse[b.total:] == 4).all()
    b.check(out, lse)


@kinds
def test_numbers_that_do_not_fit_are_skipped(q, flags):
    """Lengths below the new tokens or beyond the bound, prefix sums that do not ascend, pages outside the pool (read as zeros)."""
    b = Batch([1, 20, 1, 2], [300, 100, 200, 64], q=q, flags=flags, d=64)
    for lens, cu, skipped in (([301, 19, 201, 66], None, [1]), ([301, 120, 100000, 66], None, [2]), (None, [0, 1, 21, 20, 24], [2, 3])):
        out, lse = torch.full_like(b.qd, 3.0), torch.full((b.rows, b.hq), 4.0, device=DEV)
        b.cache.attend(b.qd, b.cu if cu is None else ints(cu), b.lens_t if lens is None else ints(lens), b.table, b.max_new, b.max_len, out=out, lse=lse)
        assert b.cache.sync_status() == binding.SPLA_ERR_BOUNDS
        b.check(out, lse, seqs=[s for s in range(4) if s not in skipped])
        if cu is None:
            rows = slice(int(b.cu_cpu[skipped[0]]), int(b.cu_cpu[skipped[0] + 1]))
            assert (out[rows] == 3).all() and (lse[rows] == 4).all()
    for bad in (-1, 1 << 30):
        table = b.table_cpu.clone()
        table[1, 0] = bad
        out, lse = b.cache.attend(b.qd, b.cu, b.lens_t, table.to(DEV), b.max_new, b.max_len)
        assert b.cache.sync_status() == binding.SPLA_ERR_BOUNDS
        zero = Batch([1, 20, 1, 2], [300, 100, 200, 64], q=q, flags=flags, d=64)
        page = int(zero.table_cpu[1, 0])
        for x in "kv":
            zero.bytes[x][page] = 0
            zero.scales[x][page] = 127
        zero.check(out, lse)


def test_waits_that_run_out():
    """A bounded wait that ends without its copy: the status is latched, the kernel returns, the next call is as ever."""
    for new in ([1, 2], [150, 40]):
        b = Batch(new, [500, 900], hq=8, hkv=2, d=128)
        want, want_lse = b.run()
        b.cache.debug_wait_hook(1 << 14, 16)
        b.attend()
        assert b.cache.sync_status() == binding.SPLA_ERR_TIMEOUT
        b.cache.debug_wait_hook(0, 0)
        out, lse = b.attend()
        assert b.cache.sync_status() == 0 and torch.equal(out, want) and torch.equal(lse, want_lse)


@kinds
def test_streams_and_graphs(q, flags):
    """Calls on two streams at once and captured calls, replayed with other contents beside an eager one: no scratch is shared."""
    b = Batch([1, 1, 66], [4000, 30, 900], hq=8, hkv=2, d=128, q=q, flags=flags)
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


def test_two_threads():
    import threading
    b = Batch([1, 1, 66], [4000, 30, 900], hq=8, hkv=2, d=128)
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


@kinds
def test_many_sequences(q, flags):
    """More sequences than a launch's table holds; chunks among them; prompts only."""
    b = Batch(torch.randint(20, 60, (400,), generator=torch.Generator().manual_seed(4)).tolist(), [0] * 400, hq=8, hkv=1, d=64, P=16, q=q, flags=flags)
    b.run()
    assert b.wide
    n = 900
    g = torch.Generator().manual_seed(3)
    new = torch.randint(0, 3, (n,), generator=g).tolist()
    new[5], new[700] = 40, 70
    old = torch.randint(0, 40, (n,), generator=g).tolist()
    Batch(new, old, hq=2, hkv=1, d=64, P=16, q=q, flags=flags).run()


@pytest.mark.parametrize("new", [1, 40])
def test_a_long_cache(new):
    """Walks of several hundred tiles: sums that are taken out of the tensor core on the way, and those that never go in."""
    b = Batch([new], [70000], hq=2, hkv=1, d=64, P=128, spread=0)
    for x in "kv":                                                            # equal weights: every token adds a little
        b.bytes[x][:] = torch.where(b.bytes[x] == 0x7f, b.bytes[x], (b.bytes[x] & 0x07) | 0x30)
    b.put()
    b.run()


def test_offsets_past_32_bits():
    """A pool of more than 2^32 bytes, the sequences in its last pages and its first: stored, read and attended to."""
    hkv, P, d = 8, 128, 128
    n_pages = (1 << 32) // (hkv * P * d) + 7
    t = binding.PagedCache.pages(n_pages, hkv, P, d)
    table = torch.tensor([[n_pages - 1, 0, n_pages - 2], [n_pages - 3, n_pages - 4, 5]], dtype=torch.int32)
    g = torch.Generator().manual_seed(2)
    k, v, q = (torch.randn(560, h, d, generator=g).to(torch.bfloat16) for h in (hkv, hkv, 16))
    cu, ln, tb = ints([0, 300, 560]), ints([300, 260]), table.to(DEV)
    cache = binding.PagedCache(n_q_heads=16, **t)
    cache.append(k.to(DEV), v.to(DEV), cu, ln, tb)
    small = binding.PagedCache(n_q_heads=16, **binding.PagedCache.pages(6, hkv, P, d))
    own = torch.arange(6, dtype=torch.int32, device=DEV).view(2, 3)
    small.append(k.to(DEV), v.to(DEV), cu, ln, own)
    assert all(torch.equal(x, y) for x, y in zip(cache.read(cu, ln, tb, 560), small.read(cu, ln, own, 560)))
    for cu_q, n in ((cu, 300), (ints([0, 1, 2]), 1)):
        rows = q[:int(cu_q[-1])].to(DEV)
        assert all(torch.equal(x, y) for x, y in zip(cache.attend(rows, cu_q, ln, tb, n, 300), small.attend(rows, cu_q, ln, own, n, 300)))
    assert cache.sync_status() == 0 and small.sync_status() == 0


@pytest.mark.parametrize("seed", [int(os.environ.get("SPLA_FUZZ_OFFSET", "0")) + i for i in range(80)])
def test_drawn(seed):
    """Anything the documentation allows, at once."""
    r = random.Random(19000 + seed)
    q, flags = r.choice([KINDS[0]] * 5 + KINDS[1:])
    B, hkv, G, d, P = r.choice([1, 2, 3, 7, 20, 33]), r.choice([1, 2, 3]), r.choice([1, 2, 3, 4, 5, 7, 8, 11, 16]), r.choice([64, 128]), r.choice([16, 32, 64, 128])
    few = r.random() < 0.5
    new = [r.choice([0, 1, 1, r.randint(1, 3 if few else 150)]) for _ in range(B)]
    if not sum(new):
        new[0] = 1
    old = [r.choice([0, r.randint(0, 30), r.randint(0, 700), r.randint(0, 3000)]) for _ in range(B)]
    b = Batch(new, old, hq=G * hkv, hkv=hkv, d=d, P=P, q=q, flags=flags, seed=seed, extra_rows=r.choice([0, 3]), extra_cols=r.choice([0, 5]), spread=r.choice([0, 1, 4]))
    kw = {}
    if r.random() < 0.3:
        kw["softcap"] = r.choice([1.0, 5.0, 30.0, 500.0])
    if r.random() < 0.4:
        kw["window"] = r.choice([1, 2, 17, 128, 400])
    if r.random() < 0.3:
        kw["slopes"] = torch.tensor([r.choice([0.0, 0.01, 0.3, 2.0]) for _ in range(G * hkv)])
    if r.random() < 0.3:
        kw["first_key"] = torch.tensor([max(-1, r.choice([0, p, p - r.randint(0, 200), p + 1])) for n, o in zip(new, old) for p in range(o, o + n)] + [0] * (b.rows - b.total),
                                       dtype=torch.int32)
    elif r.random() < 0.5:
        kw["sinks"] = r.choice([1, 4, 100, 300])
    if r.random() < 0.3:
        kw["prefix_lens"] = torch.tensor([r.choice([0, 5, 100, 5000]) for _ in range(B)], dtype=torch.int32)
    bounds = dict(max_new=b.max_new + r.choice([0, 0, 40]), max_len=min(b.max_len + r.choice([0, 0, 300]), b.table.shape[1] * P))
    bounds["max_new"] = min(bounds["max_new"], bounds["max_len"])
    out, lse = b.attend(**kw, **bounds)
    assert b.cache.sync_status() == 0
    b.check(out, lse, **{k: (v[:b.total] if k == "first_key" else v) for k, v in kw.items()})
    again, lse2 = b.attend(**kw, **bounds)
    assert torch.equal(out[:b.total], again[:b.total]) and torch.equal(lse[:b.total], lse2[:b.total])


# ---- storing and reading ----------------------------------------------------------------------------------------------
def fresh_pool(n_pages, hkv, P, d, seed=0):
    """Pages of any bytes and scales of any sizes, as a pool that has been in use."""
    g = torch.Generator().manual_seed(seed)
    held = torch.randint(0, 256, (n_pages, hkv, P, d), generator=g, dtype=torch.uint8)
    held = torch.where(held & 0x7f == 0x7f, held - 1, held)
    return held, torch.randint(120, 134, (n_pages, hkv, P // 16), generator=g, dtype=torch.uint8)


@pytest.mark.parametrize("q", ["bf16", "f32"])
@pytest.mark.parametrize("d,P", [(128, 64), (64, 16), (128, 16), (64, 128)])
@pytest.mark.parametrize("packed,offset", [(False, 0), (True, 0), (False, 1)], ids=["dense", "packed", "unaligned"])
def test_store_bit_for_bit(q, d, P, packed, offset):
    """Blocks begun before, begun anew and grown; every other byte of the pool stays as it was; the values come back as they were stored."""
    new, old = [1, 0, 40, 7, 130, 1, 16, 15], [0, 9, 25, 64, 511, 47, 32, 1]
    total, hkv, hq, t = sum(new), 2, 4, TYPES[q]
    g = torch.Generator().manual_seed(11)
    size = torch.exp2(torch.randint(-6, 7, (total, 1, 1), generator=g).float())
    if packed:
        qkv = (torch.randn(total, hq + 2 * hkv + 1, d, generator=g) * size).to(t).to(DEV)
        qq, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:hq + 2 * hkv]
    else:
        def some(h):
            flat = torch.zeros(total * h * d + 8, dtype=t, device=DEV)
            x = flat[offset:offset + total * h * d].view(total, h, d)
            x.copy_((torch.randn(total, h, d, generator=g) * size).to(t))
            return x
        qq, k, v = some(hq), some(hkv), some(hkv)
    lens = [a + b for a, b in zip(new, old)]
    need = [-(-x // P) for x in lens]
    order = torch.randperm(sum(need) + 2, generator=g)
    table, at = torch.full((len(new), max(need)), -3, dtype=torch.int32), 0
    for b, m in enumerate(need):
        table[b, :m] = order[at:at + m]
        at += m
    pools = {x: fresh_pool(len(order), hkv, P, d, i) for i, x in enumerate("kv")}
    dev = {x: on_device(*(y.clone() for y in pools[x])) for x in "kv"}
    cache = binding.PagedCache(dev["k"][0], dev["v"][0], n_q_heads=hq, q_dtype=q, k_scales=dev["k"][1], v_scales=dev["v"][1])
    cu = ints([0] + torch.tensor(new).cumsum(0).tolist())
    out = cache.append(k, v, cu, ints(lens), table.to(DEV), q=qq)
    assert cache.sync_status() == 0 and torch.equal(out, qq)
    for x, rows in (("k", k), ("v", v)):
        ref8.store(*pools[x], rows.cpu().double(), new, old, table, P)
        assert torch.equal(dev[x][1].view(torch.uint8).cpu(), pools[x][1]), x
        assert torch.equal(dev[x][0].view(torch.uint8).cpu(), pools[x][0]), x
    for dtype in (torch.bfloat16, torch.float32):
        got = cache.read(cu, ints(lens), table.to(DEV), total, dtype=dtype)
        for x, rows in zip("kv", got):
            held = ref8.values(*pools[x])
            at = 0
            for b, (n, o) in enumerate(zip(new, old)):
                j = torch.arange(o, o + n)
                assert torch.equal(rows[at:at + n].cpu().double(), held[table[b].long()[j // P], :, j % P]), x
                at += n


@pytest.mark.parametrize("q", ["bf16", "f32"])
def test_any_cutting_ends_with_the_same_scales(q):
    """Tokens one at a time, in pieces and at once: the same scales; the same bytes too where nothing comes below 2^-6 of a scale."""
    n, hkv, d, P = 77, 2, 64, 16
    g = torch.Generator().manual_seed(5)
    x = ((torch.rand(n, hkv, d, generator=g) + 1) * torch.exp2(torch.randint(0, 5, (n, 1, 1), generator=g).float()) *
         (torch.randint(0, 2, (n, hkv, d), generator=g) * 2 - 1)).to(TYPES[q]).to(DEV)
    found = []
    for pieces in ([n], [1] * n, [5, 11, 1, 30, 30], [15, 2, 60]):
        t = binding.PagedCache.pages(-(-n // P), hkv, P, d)
        cache = binding.PagedCache(n_q_heads=hkv, q_dtype=q, **t)
        at = 0
        for m in pieces:
            cache.append(x[at:at + m], -x[at:at + m], ints([0, m]), ints([at + m]), torch.arange(-(-n // P), dtype=torch.int32, device=DEV)[None])
            at += m
        assert cache.sync_status() == 0
        found.append([y.view(torch.uint8).clone() for y in t.values()])
    for other in found[1:]:
        assert all(torch.equal(a, b) for a, b in zip(found[0], other))


def test_values_at_the_ends():
    """Zeros, the smallest and largest magnitudes, values that are not finite."""
    d, P = 64, 16
    rows = torch.zeros(8 * 16, 1, d)
    rows[16] = 1e-30                                                          # below every scale: zeros
    rows[32] = 448.0                                                          # the largest of scale 1
    rows[48, 0, 0] = 448.0000305                                              # one step of fp32 above: scale 2
    rows[64] = 3e38                                                           # beyond every scale: the largest there is
    rows[80, 0, :4] = torch.tensor([math.inf, -math.inf, math.nan, 2.0])
    rows[96] = 2.0 ** -41
    rows[112, 0, 0] = -0.0
    t = binding.PagedCache.pages(8, 1, P, d)
    cache = binding.PagedCache(n_q_heads=1, q_dtype="f32", **t)
    table = torch.arange(8, dtype=torch.int32, device=DEV)[None]
    k = rows.to(DEV)
    cache.append(k, k, ints([0, 128]), ints([128]), table)
    exps = t["k_scales"].view(torch.uint8).cpu().flatten().long() - 127
    assert exps.tolist() == [-40, -40, 0, 1, 40, -7, -40, -40]
    back, _ = cache.read(ints([0, 128]), ints([128]), table, 128)
    back = back.cpu()
    assert (back[16] == 0).all() and (back[32] == 448).all() and float(back[48, 0, 0]) == 448 and (back[64] == 448 * 2.0 ** 40).all()
    assert torch.isnan(back[80, 0, :3]).all() and float(back[80, 0, 3]) == 2.0 and (back[96] == 2.0 ** -41).all() and cache.sync_status() == 0


@pytest.mark.parametrize("q", ["bf16", "f32"])
def test_what_does_not_fit_is_not_stored(q):
    """Bad lengths and prefix sums are skipped, the tokens of a bad page are not stored, and both are latched; read as in the other calls."""
    hkv, d, P, t = 2, 64, 16, TYPES[q]
    new, old = [3, 20, 2], [5, 0, 30]
    held, scales = fresh_pool(12, hkv, P, d)
    x, qq = torch.randn(25, hkv, d, device=DEV).to(t), torch.randn(25, 4, d, device=DEV).to(t)
    table = torch.tensor([[1, -1], [2, 3], [4, 5]], dtype=torch.int32)
    for lens, cu, tab, served in (([8, 20, 1], [0, 3, 23, 25], table, [0, 1]), ([8, 20, 32], [0, 3, 2, 25], table, [0]), ([8, 20, 32], [0, 3, 23, 25], torch.tensor([[1, -1], [99, 3], [4, 5]], dtype=torch.int32), [0, 1, 2])):
        k, ks = on_device(held.clone(), scales.clone())
        v, vs = on_device(held.clone(), scales.clone())
        cache = binding.PagedCache(k, v, n_q_heads=4, q_dtype=q, k_scales=ks, v_scales=vs)
        out = torch.full_like(qq, 9.0)
        cache.append(x, x, ints(cu), ints(lens), tab.to(DEV), q=qq, q_out=out)
        assert cache.sync_status() == binding.SPLA_ERR_BOUNDS
        want, want_s = held.clone(), scales.clone()
        rows = {0: slice(0, 3), 1: slice(3, 23), 2: slice(23, 25)}
        for s in served:
            one = tab[s:s + 1]
            ref8.store(want, want_s, x[rows[s]].cpu().double(), [new[s]], [old[s]], one, P)
        assert torch.equal(k.view(torch.uint8).cpu(), want) and torch.equal(ks.view(torch.uint8).cpu(), want_s)
        for s in range(3):
            assert torch.equal(out[rows[s]], qq[rows[s]] if s in served else torch.full_like(qq[rows[s]], 9.0))
        back = [torch.full((25, hkv, d), 5.0, dtype=t, device=DEV) for _ in range(2)]
        cache.read(ints(cu), ints(lens), tab.to(DEV), 25, k_out=back[0], v_out=back[1])
        assert cache.sync_status() == binding.SPLA_ERR_BOUNDS
        for s in range(3):
            if s not in served:
                assert (back[0][rows[s]] == 5).all()
        if int(tab[1, 0]) == 99:
            assert (back[1][rows[1]][:16] == 0).all() and (back[1][rows[1]][16:] != 5).any()


@pytest.mark.parametrize("kv", ["bf16", "f32"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_read_of_other_caches(kv, dtype):
    """Pages of 16 and 32 bits are read the same way (and rounded once)."""
    hkv, d, P = 3, 64, 32
    k, v = (torch.randn(5, hkv, P, d, device=DEV).to(TYPES[kv]) for _ in range(2))
    cache = binding.PagedCache(k, v, n_q_heads=3)
    table = ints([[3, 0], [4, 2]])
    rk, rv = cache.read(ints([0, 40, 41]), ints([50, 7]), table, 41, dtype=dtype)
    for rows, pages in ((rk, k), (rv, v)):
        j = torch.arange(10, 50, device=DEV)
        assert torch.equal(rows[:40], pages[table[0].long()[j // P], :, j % P].to(dtype)) and torch.equal(rows[40], pages[4, :, 6].to(dtype))
    assert cache.sync_status() == 0


@pytest.mark.parametrize("kv,q", [("e4m3", "bf16"), ("e4m3", "f32"), ("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32")])
@pytest.mark.parametrize("d,rope", [(128, dict()), (64, dict(rot_dim=32, interleaved=True)), (128, None), (64, dict(rot_dim=6, amplitude=1.2)), (128, dict(scaling="linear", factor=4.0))])
@pytest.mark.parametrize("norm", ["both", "k", "none"])
def test_store_with_norms(kv, q, d, rope, norm):
    """Keys and queries normed, then rotated, then stored: in 8 bits within half a step of the formula, in others as rounded once."""
    new, old, hq, hkv, P, eps = [1, 40, 7, 130], [0, 25, 64, 511], 4, 2, 64, 1e-5
    total, t, qt = sum(new), TYPES["bf16" if kv == "bf16" else q], TYPES[q]
    if kv != "e4m3":
        t = TYPES[kv]
    g = torch.Generator().manual_seed(3)
    k, v, qq = torch.randn(total, hkv, d, generator=g).to(t), torch.randn(total, hkv, d, generator=g).to(t), (3 * torch.randn(total, hq, d, generator=g)).to(qt)
    wq, wk = 1 + 0.3 * torch.randn(d, generator=g), 1 + 0.3 * torch.randn(d, generator=g)
    lens = [a + b for a, b in zip(new, old)]
    need = [-(-x // P) for x in lens]
    table, at = torch.full((len(new), max(need)), -3, dtype=torch.int32), 0
    for b, m in enumerate(need):
        table[b, :m] = torch.arange(at, at + m)
        at += m
    if kv == "e4m3":
        pages = binding.PagedCache.pages(at, hkv, P, d)
        cache = binding.PagedCache(n_q_heads=hq, q_dtype=q, **pages)
    else:
        cache = binding.PagedCache(*(torch.zeros(at, hkv, P, d, dtype=t, device=DEV) for _ in range(2)), n_q_heads=hq, q_dtype=q)
    cu = ints([0] + torch.tensor(new).cumsum(0).tolist())
    r = binding.Rope(d, **rope) if rope is not None else None
    out = cache.append(k.to(DEV), v.to(DEV), cu, ints(lens), table.to(DEV), q=qq.to(DEV), rope=r, eps=eps,
                       q_weight=wq.to(DEV) if norm == "both" else None, k_weight=wk.to(DEV) if norm != "none" else None)
    assert cache.sync_status() == 0
    a = dict(rope or {})
    rot, inter, amp = a.pop("rot_dim", d), a.pop("interleaved", False), a.pop("amplitude", 1.0)
    pos = torch.cat([torch.arange(o, o + n) for n, o in zip(new, old)])

    def wanted(x, w):
        y, rel = x.double(), 0.0
        if w is not None:
            y = y / (y.pow(2).mean(-1, keepdim=True) + eps).sqrt() * w.double()
            rel = (d / 2 + 8) * 2.0 ** -24                                    # the sum of d squares, its root, two products
        if rope is None:
            return y, rel * y.abs()
        z, err = ref.rotate(y, pos, rot, inter, ref.frequencies(rot, **a), amp)
        i = torch.arange(rot // 2)
        ia, ib = (2 * i, 2 * i + 1) if inter else (i, i + rot // 2)
        both = amp * (y[..., ia].abs() + y[..., ib].abs()) * rel
        err[..., ia] += both
        err[..., ib] += both
        err[..., rot:] += rel * y[..., rot:].abs()
        return z, err

    y, err = wanted(qq, wq if norm == "both" else None)
    ref.check(out, y, err, qt, "q")
    y, err = wanted(k, wk if norm != "none" else None)
    rk, rv = cache.read(cu, ints(lens), table.to(DEV), total, dtype=torch.float32)
    if kv != "e4m3":
        ref.check(rk, y, err, t, "k")
        assert torch.equal(rv.cpu(), v.float())
        return
    scales = pages["k_scales"].view(torch.uint8).cpu().long() - 127
    row = 0
    for b, (n, o) in enumerate(zip(new, old)):
        e = scales[table[b].long()[torch.arange(o, o + n) // P], :, torch.arange(o, o + n) % P // 16]       # [n][hkv]
        for block in sorted(set((torch.arange(o, o + n) // 16).tolist())):
            j = [i for i in range(n) if (o + i) // 16 == block]
            some, off = y[row + j[0]:row + j[-1] + 1].abs(), err[row + j[0]:row + j[-1] + 1]
            low, high = ref8.exponent((some - off).amax((0, 2))), ref8.exponent((some + off).amax((0, 2)))
            started = o % 16 != 0 and block == o // 16                        # (begun before: the pool's scale of 1 is kept where it is large enough)
            if started:
                low, high = low.clamp(min=0), high.clamp(min=0)
            assert ((e[j[0]] >= low) & (e[j[0]] <= high)).all()
        step = torch.pow(2.0, e.double())[..., None]
        some, off = y[row:row + n], err[row:row + n]
        bound = off + torch.maximum((some.abs() + off) * 2.0 ** -4, step * 2.0 ** -10)
        assert ((rk[row:row + n].cpu().double() - some).abs() <= bound).all()
        row += n


def test_a_layer():
    """A few steps of one layer as a serving loop takes them: prompts, then single tokens, normed, rotated and stored in 8 bits, then attended to; the same as
    norm, rotation and float64 attention over what the cache says it holds."""
    hq, hkv, d, P, eps = 8, 2, 128, 16, 1e-6
    g = torch.Generator().manual_seed(1)
    wq, wk = 1 + 0.2 * torch.randn(d, generator=g), 1 + 0.2 * torch.randn(d, generator=g)
    rope = binding.Rope(d, base=500000.0)
    t = binding.PagedCache.pages(60, hkv, P, d)
    cache = binding.PagedCache(n_q_heads=hq, **t)
    table = torch.randperm(60, generator=g).to(torch.int32).view(3, 20)
    lens = [0, 0, 0]
    for new in ([130, 40, 1], [1, 1, 1], [1, 0, 1], [1, 17, 1], [1, 1, 1]):
        lens = [a + b for a, b in zip(lens, new)]
        total = sum(new)
        qkv = torch.randn(total, hq + 2 * hkv, d, generator=g).to(torch.bfloat16).to(DEV)
        cu, ln = ints([0] + torch.tensor(new).cumsum(0).tolist()), ints(lens)
        q = cache.append(qkv[:, hq:hq + hkv], qkv[:, hq + hkv:], cu, ln, table.to(DEV), q=qkv[:, :hq], rope=rope, q_weight=wq.to(DEV), k_weight=wk.to(DEV), eps=eps)
        pos = torch.cat([torch.arange(x - n, x) for n, x in zip(new, lens)]).to(torch.int32).to(DEV)
        assert torch.equal(q, rope.norm_apply(pos, qkv[:, :hq], wq.to(DEV), eps=eps))
        out, lse = cache.attend(q, cu, ln, table.to(DEV), max(new), max(lens), window=64, sinks=3)
        assert cache.sync_status() == 0
        k, v = (ref8.values(t[x + "_pages"].view(torch.uint8).cpu(), t[x + "_scales"].view(torch.uint8).cpu()) for x in "kv")
        wide = widened(3, total, hq, hkv, d, max(new), max(lens), window=64, sinks=3)
        o, l, ob, lb = ref8.attend(q.cpu(), k, v, cu.cpu(), lens, table, lambda n: "wide" if wide else "few" if n * 4 <= 16 else "chunk", 4, window=64, sinks=3)
        ref8.check(lse, l, lb, what="lse")
        ref8.check(out, o, ob, torch.bfloat16, "out")


def test_store_in_a_graph():
    """A captured step, replayed: lengths and tokens of each replay; two caches' graphs share nothing."""
    hq, hkv, d, P = 4, 2, 64, 16
    caches, graphs = [], []
    x = torch.randn(3, hq + 2 * hkv, d, device=DEV).to(torch.bfloat16)
    ln, cu, table = ints([1, 20, 5]), ints([0, 1, 2, 3]), torch.arange(12, dtype=torch.int32, device=DEV).view(3, 4)
    for _ in range(2):
        t = binding.PagedCache.pages(12, hkv, P, d)
        c = binding.PagedCache(n_q_heads=hq, **t)
        c.append(x[:, 4:6], x[:, 6:], cu, ln, table, q=x[:, :4])
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            q = c.append(x[:, 4:6], x[:, 6:], cu, ln, table, q=x[:, :4])
            res = c.attend(q, cu, ln, table, 1, 64)
        caches.append((c, t))
        graphs.append((g, res))
    for step in range(8):
        x.copy_(torch.randn_like(x) * 2.0 ** step)
        ln += 1
        for g, _ in graphs:
            g.replay()
    torch.cuda.synchronize()
    a, b = caches[0][1], caches[1][1]
    assert all(torch.equal(a[n].view(torch.uint8), b[n].view(torch.uint8)) for n in a)
    out, lse = caches[0][0].attend(x[:, :4].contiguous(), cu, ln, table, 1, 64)
    assert torch.equal(out, graphs[0][1][0]) and torch.equal(lse, graphs[1][1][1]) and caches[0][0].sync_status() == 0
