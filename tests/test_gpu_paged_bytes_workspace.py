"""The workspace of attention over 8-bit pages: as much as a call can use (host only, but for the tensor maps that a cache is made with)."""
import ctypes as C

import pytest
import torch

from paper_2601_22379_b200 import binding

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hq,hkv,d", [(32, 8, 128), (16, 16, 64)])
@pytest.mark.parametrize("tokens", [16, 32, 64, 127, 128, 500, 512])
def test_what_the_widened_tokens_may_take(hq, hkv, d, tokens):
    """On a long cache: eight times the queries in two parts where a sequence has 512 rows, four times where it has fewer; besides, what partial results and drained sums of one
    launch take (a CTA's two, 256 rows and 128 rows, on at most 256 SMs)."""
    cache = binding.PagedCache(n_q_heads=hq, **binding.PagedCache.pages(2, hkv, 64, d))
    batch, rest = 300, 2 * 256 * (256 * (d * 4 + 8) + 128 * (d + 1) * 4) + (1 << 20)
    b = binding.SplaPagedBatch(4, 8, 12, batch, batch * tokens * 64, max(tokens * 64, 17), 1 << 24, 1 << 18)
    rows = tokens * 64 * hq // hkv
    n = C.c_size_t()
    assert cache.lib.spla_paged_query_workspace(cache.handle, C.addressof(b), C.byref(n)) == binding.SPLA_OK
    few = binding.SplaPagedBatch(4, 8, 12, batch * 64, batch * tokens * 64, max(tokens * 64, 17), 1 << 24, 1 << 18)   # the same tokens of more sequences
    m = C.c_size_t()
    assert cache.lib.spla_paged_query_workspace(cache.handle, C.addressof(few), C.byref(m)) == binding.SPLA_OK
    parts = batch * tokens * 64 * hq * (2 * d + 1)
    assert rows >= 512 and 8 * parts <= n.value <= 8 * parts + rest
    most = 8 if tokens * hq // hkv >= 512 else 4
    assert most * parts <= m.value <= most * parts + rest
    torch.cuda.synchronize()
