"""First tokens that stay visible beside a window, over pages of 16 and 32 bits, against a plain float64 form."""
import pytest
import torch

from paper_2601_22379_b200 import binding
from tests import paged_bytes_reference as ref8
from tests.test_gpu_paged import Batch, kinds

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
