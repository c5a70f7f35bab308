"""Each kernel of the attention over 8-bit pages: waits that run out, and calls of two threads at once."""
import threading

import pytest
import torch

from paper_2601_22379_b200 import binding
from tests.test_gpu_paged_bytes import Batch

pytestmark = pytest.mark.gpu
# new tokens, cached ones, queries, what serves the sequences
KERNELS = {
    "few-8-rows": ([1, 2], [500, 900], "bf16", {"few"}),
    "few-16-rows": ([4, 3], [500, 900], "bf16", {"few"}),
    "few-f32": ([1, 2], [500, 900], "f32", {"few32"}),
    "few-f32-16-rows": ([4, 3], [4000, 900], "f32", {"few32"}),
    "chunk-32-rows": ([8, 2], [500, 900], "bf16", {"few", "chunk"}),
    "chunk": ([150, 40], [500, 900], "bf16", {"chunk"}),
    "wide": ([150, 40], [0, 30], "bf16", {"wide"}),
}
kernels = pytest.mark.parametrize("new,old,q,how", list(KERNELS.values()), ids=list(KERNELS))


def batch(new, old, q, how, d=128):
    b = Batch(new, old, hq=8, hkv=2, d=d, q=q)
    want = b.run(softcap=20.0)
    assert {b.kernel(n) for n in new} == how
    return b, want


@kernels
@pytest.mark.parametrize("d", [64, 128])
def test_waits_that_run_out(new, old, q, how, d):
    """The status is latched, the kernels return, the next call is as ever."""
    b, want = batch(new, old, q, how, d)
    for _ in range(2):
        b.cache.debug_wait_hook(1 << 14, 16)
        b.attend(softcap=20.0)
        assert b.cache.sync_status() == binding.SPLA_ERR_TIMEOUT
        b.cache.debug_wait_hook(0, 0)
        out = b.attend(softcap=20.0)
        assert b.cache.sync_status() == 0 and all(torch.equal(x, y) for x, y in zip(out, want))


@kernels
def test_two_threads(new, old, q, how):
    b, want = batch(new, old, q, how)
    wrong = []

    def work():
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            for _ in range(40):
                out = b.cache.attend(b.qd, b.cu, b.lens_t, b.table, b.max_new, b.max_len, softcap=20.0)
                stream.synchronize()
                if not all(torch.equal(x, y) for x, y in zip(out, want)):
                    wrong.append(1)

    threads = [threading.Thread(target=work) for _ in range(2)]
    [t.start() for t in threads]
    [t.join() for t in threads]
    assert not wrong and b.cache.sync_status() == 0
