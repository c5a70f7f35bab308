"""First tokens that stay visible beside a window, over pages of 16 and 32 bits, against a plain float64 form."""
import pytest
import torch

from paper_2601_22379_b200 import binding
from tests import paged_bytes_reference as ref8
from tests.test_gpu_paged import TYPES, Batch, kinds

pytestmark = pytest.mark.gpu


def check(b, out, lse, **kw):
    """Values of 16 or 32 bits have no scale: the terms of the 8-bit forms that remain are those of the general kernel, and a weight in bf16, half a step of 2^-8."""
    kw["prefix"] = kw.pop("prefix_lens", None)
    o, l, ob, lb = ref8.attend(b.q[:b.total], b.k.double(), b.v.double(), b.cu_cpu, b.lens, b.table_cpu, lambda n: "general", 0, **kw)
    if b.tensor_cores:
        absolute = ref8.attend(b.q[:b.total], b.k.double(), b.v.double().abs(), b.cu_cpu, b.lens, b.table_cpu, lambda n: "general", 0, **kw)[0]
        ob = ob + absolute * 2.0 ** -8
    ref8.check(lse[:b.total], l, lb, what="lse")
    ref8.check(out[:b.total], o, ob, b.q_t, "out")


@kinds
@pytest.mark.parametrize("d,P", [(128, 64), (64, 16)])
@pytest.mark.parametrize("window,sinks", [(1, 1), (37, 4), (100, 128), (130, 129), (64, 700), (5000, 4)])
@pytest.mark.parametrize("new,old", [([1], [0]), ([1, 2, 1], [1000, 37, 700]), ([5, 0, 1, 33], [0, 3, 700, 930]), ([150, 260], [40, 2000])], ids=["one", "few", "ragged", "chunk"])
def test_window_and_sinks(kv, q, flags, d, P, window, sinks, new, old):
    b = Batch(new, old, d=d, P=P, kv=kv, q=q, flags=flags)
    kw = dict(window=window, sinks=sinks)
    out, lse = b.attend(**kw)
    assert b.cache.sync_status() == 0
    check(b, out, lse, **kw)


@kinds
def test_with_the_other_masks(kv, q, flags):
    b = Batch([1, 70, 9, 1, 200], [400, 300, 0, 1065, 331], hq=4, hkv=2, d=64, P=32, kv=kv, q=q, flags=flags)
    kw = dict(softcap=8.0, slopes=torch.tensor([0.01, 0.125, 0.0, 1.0]), window=90, sinks=5, prefix_lens=torch.tensor([390, 350, 7, 0, 60], dtype=torch.int32))
    out, lse = b.attend(**kw)
    assert b.cache.sync_status() == 0
    check(b, out, lse, **kw)


@kinds
def test_without_a_window_sinks_change_nothing(kv, q, flags):
    b = Batch([1, 40], [300, 100], kv=kv, q=q, flags=flags)
    want = b.run()
    assert all(torch.equal(x, y) for x, y in zip(b.attend(sinks=7), want))


def test_sinks_with_documents_are_refused():
    b = Batch([1, 2], [30, 40])
    with pytest.raises(binding.SplaError) as e:
        b.attend(window=10, sinks=2, first_key=torch.zeros(3, dtype=torch.int32))
    assert e.value.status == binding.SPLA_ERR_UNSUPPORTED
    with pytest.raises(binding.SplaError):
        b.attend(window=10, sinks=-1)
    with pytest.raises(ValueError):
        b.attend(window=10, sinks=2 ** 32)


def test_as_many_sinks_as_there_are():
    """The largest number: every key is visible, as without a window."""
    b = Batch([1, 40], [300, 100])
    out, lse = b.attend(window=3, sinks=2 ** 31 - 1)
    assert b.cache.sync_status() == 0
    check(b, out, lse)


@pytest.mark.parametrize("kv", ["bf16", "f32"])
def test_over_an_spla_cache(kv):
    """Its pages read back are what was appended, and sinks beside a window are those of the same tokens in pages of their own."""
    B, hq, hkv, d, T = 3, 8, 2, 128, 300
    cfg = binding.make_config(batch=B, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, block_size=64, top_k=8, max_context=512, kv_dtype=kv, flags=binding.SPLA_NO_RLA)
    cache = binding.SplaCache(cfg, "cuda:0")
    t = TYPES[kv]
    g = torch.Generator(device="cuda:0").manual_seed(2)
    k, v = (torch.randn(B, hkv, T, d, device="cuda:0", generator=g).to(t) for _ in range(2))
    q = torch.randn(B, hq, d, device="cuda:0", generator=g).to(t)
    lens = [300, 1, 129]
    cache.append_tokens(k, v, torch.tensor(lens, dtype=torch.int32, device="cuda:0"))
    pages = binding.PagedCache.of(cache)
    cu = torch.tensor([0, 300, 301, 430], dtype=torch.int32, device="cuda:0")
    kr, vr = pages.read(cu, cache.bufs.seq_lens, pages.table(), 430)
    rows = lambda x: torch.cat([x[b, :, :n].transpose(0, 1) for b, n in enumerate(lens)])  # noqa: E731
    assert torch.equal(kr, rows(k)) and torch.equal(vr, rows(v))

    b = Batch([1, 1, 1], [n - 1 for n in lens], hq=hq, hkv=hkv, d=d, P=64, kv=kv, q=kv)
    own = torch.arange(3, dtype=torch.int32, device="cuda:0")
    b.cache.append(rows(k), rows(v), cu, b.lens_t, b.table)
    kw = dict(window=30, sinks=5)
    cu1 = torch.arange(B + 1, dtype=torch.int32, device="cuda:0")
    got = pages.attend(q, cu1, cache.bufs.seq_lens, pages.table(), 1, 300, **kw)
    want = b.cache.attend(q, cu1, b.lens_t, b.table, 1, 300, **kw)
    assert pages.sync_status() == 0 and b.cache.sync_status() == 0
    assert all(torch.equal(x, y) for x, y in zip(got, want))
