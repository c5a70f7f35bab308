"""What the binding of the paged cache and the rotary positions refuses before it calls the library: tensors on the CPU, no device."""
import pytest
import torch

from paper_2601_22379_b200 import binding


def cache(hq=4, hkv=2, d=64, P=16):
    """A cache without a handle: a call that gets past the checks of its tensors fails in the library."""
    c = binding.PagedCache.__new__(binding.PagedCache)
    c.k_pages = c.v_pages = torch.zeros(3, hkv, P, d)
    c.device, c.index = torch.device("cpu"), 0
    c.page_size, c.n_q_heads, c.n_kv_heads, c.head_dim, c.q_torch_dtype = P, hq, hkv, d, torch.float32
    return c


def sequences(total):
    i = lambda *x: torch.tensor(x, dtype=torch.int32)  # noqa: E731
    return i(0, total), i(total), torch.arange(3, dtype=torch.int32)[None]


def expanded(heads, total=5, d=64):
    """One token, repeated by a stride of 0."""
    return torch.zeros(1, heads, d).expand(total, heads, d)


@pytest.mark.parametrize("bad", ["k", "v", "q", "q_out"])
def test_append_refuses_tokens_that_lie_on_each_other(bad):
    x = dict(k=torch.zeros(5, 2, 64), v=torch.zeros(5, 2, 64), q=torch.zeros(5, 4, 64), q_out=torch.zeros(5, 4, 64))
    x[bad] = expanded(2 if bad in "kv" else 4)
    with pytest.raises(ValueError, match="elements apart"):
        cache().append(x["k"], x["v"], *sequences(5), q=x["q"], q_out=x["q_out"])


def test_attend_refuses_queries_that_lie_on_each_other():
    for q in (expanded(4), torch.zeros(5 * 64 + 4 * 64).as_strided((5, 4, 64), (64, 64, 1))):
        with pytest.raises(ValueError, match="elements apart"):
            cache().attend(q, *sequences(5), 5, 48)


def test_strides_of_tokens():
    c = cache()
    rows = lambda x, heads: c._rows(x, x.shape[0], heads, torch.float32, "x")  # noqa: E731
    assert rows(torch.zeros(5, 4, 64), 4) == 256
    assert rows(torch.zeros(5, 9, 64)[:, 2:6], 4) == 576                      # inside a packed projection
    assert rows(expanded(4, total=1), 4) == 256                               # one token has no neighbour


def test_scales_that_overflow_are_refused():
    """A scale whose product with log2 e is not finite: scores of 0 would be 0 x infinity."""
    import ctypes as C

    from paper_2601_22379_b200 import build
    build.build()
    lib = binding.load()
    for scale, want in ((2.3e38, binding.SPLA_OK), (2.4e38, binding.SPLA_ERR_INVALID_ARG), (3.4e38, binding.SPLA_ERR_INVALID_ARG)):
        h = C.c_void_p()
        cfg = binding.SplaPagedConfig(8, 2, 128, 64, 10, 1, 1, 0, 0, scale, 0)
        assert lib.spla_paged_create(C.byref(cfg), 4096, 8192, 256, C.byref(h)) == want
        lib.spla_paged_destroy(h)


def test_pages_of_an_spla_cache_are_not_appended_to():
    """Its statistics, state and lengths would not know of the tokens.  (`of` without a device: the cache's handle is not made.)"""
    class Spla:
        cfg = binding.make_config(batch=2, n_q_heads=4, n_kv_heads=2, head_dim=64, block_size=16, top_k=2, max_context=48)
        max_blocks = 3

        class bufs:
            k_cache = v_cache = torch.zeros(2, 2, 3, 16, 64)

    class Paged(binding.PagedCache):
        def _create(self, k, v, *args):
            self.__dict__.update(cache().__dict__, k_pages=k, v_pages=v)

    c = Paged.of(Spla)
    assert c.table().tolist() == [[0, 1, 2], [6, 7, 8]]
    with pytest.raises(ValueError, match="SPLA cache"):
        c.append(torch.zeros(5, 2, 64), torch.zeros(5, 2, 64), *sequences(5))


def test_imports_without_torchs_cuda_internals():
    """Host-only use (configurations, argument checks) of a torch that was built without CUDA."""
    import os
    import subprocess
    import sys
    code = ("import torch\n"
            "for name in ('_cuda_getDevice', '_cuda_getCurrentRawStream'):\n"
            "    if hasattr(torch._C, name): delattr(torch._C, name)\n"
            "from paper_2601_22379_b200 import binding\n"
            "binding.make_config(batch=1, n_q_heads=2, n_kv_heads=1, head_dim=64, block_size=16, top_k=1, max_context=16)\n"
            "assert callable(binding._device_now) and callable(binding._stream_now)\n"
            "print('imported')\n")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    done = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True)
    assert done.stdout.strip() == "imported", done.stderr[-500:]


def test_strides_of_axes_of_one():
    """The stride of an axis of length one says nothing: one head, one page."""
    c = cache(hq=1, hkv=1)
    k = torch.zeros(1, 5, 64).transpose(0, 1)                                 # head-major, one head
    assert k.stride(1) == 5 * 64 and c._rows(k, 5, 1, torch.float32, "k") == 64
    table = torch.zeros(1, 2, dtype=torch.int32).T
    cu, lens = torch.zeros(3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    assert table.shape == (2, 1) and table.stride(1) == 2
    packed = binding.SplaPagedBatch.from_buffer_copy(c._batch(5, cu, lens, table, 5, 16))
    assert packed.table_stride == 1 and packed.batch == 2
