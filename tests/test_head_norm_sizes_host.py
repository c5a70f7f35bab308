"""The workspace of the head norms' gradients at the largest sizes: host only."""
import ctypes as C

import pytest

from paper_2601_22379_b200 import binding, build


@pytest.mark.parametrize("dim,heads", [(8, 1), (128, 1), (256, 8192)])
def test_tokens_near_the_end_of_32_bits(dim, heads):
    """As many blocks as fit the GPU at once, whether there are 2^24 tokens or all that an index counts."""
    build.build()
    lib, h, n = binding.load(), C.c_void_p(), C.c_size_t()
    cfg = binding.SplaRopeConfig(dim, 0, 0, 0, 0.0, 0.0, 0.0, 0.0, 0.0, 0.0)
    assert lib.spla_rope_create(C.byref(cfg), C.byref(h)) == binding.SPLA_OK
    sizes = []
    for batch, tokens in ((1, 1 << 24), (1, (1 << 31) - 65), (1, (1 << 31) - 64), (1, (1 << 31) - 1), ((1 << 31) - 1, 1), (3, 715827882), (65535, 32768)):
        assert lib.spla_rope_norm_query_workspace(h, batch, tokens, heads, C.byref(n)) == binding.SPLA_OK
        sizes.append(n.value)
    assert set(sizes) == {sizes[0]} and sizes[0] % (2 * dim * 4) == 0
    assert lib.spla_rope_norm_query_workspace(h, 1 << 16, 1 << 15, heads, C.byref(n)) == binding.SPLA_ERR_UNSUPPORTED
    lib.spla_rope_destroy(h)
