"""Argument checks of the rotary positions and the paged cache: on the host, before anything touches a device."""
import ctypes as C
import math

import pytest

from paper_2601_22379_b200 import binding, build

INVALID, UNSUPPORTED, OK = binding.SPLA_ERR_INVALID_ARG, binding.SPLA_ERR_UNSUPPORTED, binding.SPLA_OK


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load()


ROPE = dict(head_dim=128, rot_dim=64, interleaved=0, scaling=0, base=1e4, factor=1.0, original_len=0.0, ramp_low=0.0, ramp_high=0.0, amplitude=1.0)


def rope(lib, **kw):
    h = C.c_void_p()
    cfg = binding.SplaRopeConfig(*{**ROPE, **kw}.values())
    rc = lib.spla_rope_create(C.byref(cfg), C.byref(h))
    return rc, h


@pytest.mark.parametrize("kw,want", [
    ({}, OK), (dict(rot_dim=0), OK), (dict(base=0.0, factor=0.0, amplitude=0.0), OK), (dict(head_dim=8, rot_dim=2), OK), (dict(head_dim=256, rot_dim=256), OK),
    (dict(rot_dim=63), INVALID), (dict(rot_dim=130), INVALID), (dict(rot_dim=-2), INVALID), (dict(head_dim=0, rot_dim=0), INVALID), (dict(interleaved=2), INVALID),
    (dict(scaling=4), INVALID), (dict(scaling=-1), INVALID), (dict(base=-1.0), INVALID), (dict(base=math.nan), INVALID), (dict(base=math.inf), INVALID),
    (dict(factor=0.5), INVALID), (dict(factor=math.nan), INVALID), (dict(amplitude=math.inf), INVALID), (dict(scaling=2, rot_dim=2), INVALID),
    (dict(scaling=3), INVALID), (dict(scaling=3, original_len=4096.0, ramp_low=4.0, ramp_high=4.0), INVALID), (dict(scaling=3, original_len=4096.0, ramp_high=4.0), OK),
    (dict(scaling=3, original_len=math.nan, ramp_high=4.0), INVALID), (dict(head_dim=100, rot_dim=50), UNSUPPORTED), (dict(head_dim=264, rot_dim=64), UNSUPPORTED)])
def test_rope_config(lib, kw, want):
    rc, h = rope(lib, **kw)
    assert rc == want
    lib.spla_rope_destroy(h)


def test_rope_apply_arguments(lib):
    _, h = rope(lib)

    def call(q=None, k=None, positions=4096, batch=1, n=1, dtype=1, rope_h=h):
        return lib.spla_rope_apply(rope_h, positions, batch, n, C.addressof(q) if q else None, C.addressof(k) if k else None, dtype, 0, None)

    t = lambda **kw: binding.SplaRopeTensor(*{**dict(in_=8192, out=16384, n_heads=1, a=0, b=128, c=128, d=0, e=128, f=128), **kw}.values())  # noqa: E731
    assert call() == INVALID and call(q=t(), rope_h=None) == INVALID and call(q=t(), positions=None) == INVALID and call(q=t(), positions=4098) == INVALID
    assert call(q=t(), batch=0) == INVALID and call(q=t(), n=0) == INVALID and call(q=t(), dtype=2) == INVALID
    assert call(q=t(in_=None)) == INVALID and call(q=t(out=None)) == INVALID and call(q=t(n_heads=0)) == INVALID
    assert call(q=t(in_=8193)) == INVALID and call(q=t(in_=8194), dtype=0) == INVALID
    assert call(q=t(out=8192, e=256)) == INVALID                              # in place with other strides
    assert call(q=t(), k=t(in_=None)) == INVALID
    lib.spla_rope_destroy(h)
    assert lib.spla_rope_destroy(None) == OK
    assert lib.spla_rope_create(None, C.byref(h)) == INVALID


PAGED = dict(n_q_heads=8, n_kv_heads=2, head_dim=128, page_size=64, n_pages=10, kv_dtype=1, q_dtype=1, page_stride=0, head_stride=0, sm_scale=0.0, flags=0)


def paged(lib, k=4096, v=8192, status=256, **kw):
    h = C.c_void_p()
    cfg = binding.SplaPagedConfig(*{**PAGED, **kw}.values())
    return lib.spla_paged_create(C.byref(cfg), k, v, status, C.byref(h)), h


@pytest.mark.parametrize("kw,want", [
    ({}, OK), (dict(kv_dtype=0), OK), (dict(head_dim=64, page_size=16), OK), (dict(n_q_heads=32, n_kv_heads=2), OK), (dict(page_stride=64, head_stride=640), OK),
    (dict(n_q_heads=9), INVALID), (dict(n_q_heads=0), INVALID), (dict(n_kv_heads=0), INVALID), (dict(n_pages=0), INVALID), (dict(kv_dtype=2), INVALID), (dict(q_dtype=-1), INVALID),
    (dict(sm_scale=-1.0), INVALID), (dict(sm_scale=math.nan), INVALID), (dict(sm_scale=math.inf), INVALID), (dict(flags=1), INVALID), (dict(page_stride=-1), INVALID),
    (dict(head_stride=32), INVALID), (dict(page_stride=63, head_stride=640), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(status=None), INVALID),
    (dict(k=4096 + 16), INVALID), (dict(v=8192 + 128), INVALID), (dict(status=258), INVALID),
    (dict(n_q_heads=34, n_kv_heads=2), UNSUPPORTED), (dict(head_dim=96), UNSUPPORTED), (dict(page_size=48), UNSUPPORTED), (dict(page_size=256), UNSUPPORTED)])
def test_paged_config(lib, kw, want):
    rc, h = paged(lib, **kw)
    assert rc == want
    lib.spla_paged_destroy(h)


BATCH = dict(cu_new=256, seq_lens=512, page_table=1024, batch=2, total_new=6, max_new=4, max_len=640, table_stride=10)


def batch(**kw):
    return binding.SplaPagedBatch(*{**BATCH, **kw}.values())


BAD_BATCHES = [(dict(batch=0), INVALID), (dict(total_new=0), INVALID), (dict(max_new=0), INVALID), (dict(max_len=3), INVALID), (dict(table_stride=0), INVALID),
               (dict(max_len=641), INVALID), (dict(table_stride=9), INVALID), (dict(max_len=(1 << 24) + 1, table_stride=1 << 20), UNSUPPORTED)]
BAD_POINTERS = [(dict(cu_new=None), INVALID), (dict(seq_lens=None), INVALID), (dict(page_table=None), INVALID), (dict(cu_new=258), INVALID), (dict(page_table=1025), INVALID)]


@pytest.mark.parametrize("kw,want", BAD_BATCHES + BAD_POINTERS)
def test_batches(lib, kw, want):
    _, h = paged(lib)
    b = batch(**kw)
    assert lib.spla_paged_append(h, C.addressof(b), None, None, 4096, 0, 8192, 0, None, 0, None, 0, None) == want
    assert lib.spla_paged_attend(h, C.addressof(b), 4096, 0, None, 8192, None, None, 0, None) == want
    n = C.c_size_t()
    if (kw, want) in BAD_BATCHES:
        assert lib.spla_paged_query_workspace(h, C.addressof(b), C.byref(n)) == want
    lib.spla_paged_destroy(h)


def test_append_arguments(lib):
    _, h = paged(lib)
    _, r64 = rope(lib, head_dim=64)
    b = batch()

    def call(paged_h=h, rope_h=None, positions=None, k=4096, ks=0, v=8192, vs=0, q=None, qs=0, qo=None, qos=0):
        return lib.spla_paged_append(paged_h, C.addressof(b), rope_h, positions, k, ks, v, vs, q, qs, qo, qos, None)

    assert call(paged_h=None) == INVALID and call(k=None) == INVALID and call(v=None) == INVALID
    assert call(q=4096) == INVALID and call(qo=4096) == INVALID               # queries in without queries out
    assert call(rope_h=r64) == INVALID                                        # a rotation of heads of another size
    assert call(k=4097) == INVALID and call(q=4097, qo=4096) == INVALID and call(positions=4097) == INVALID
    assert call(ks=255) == INVALID and call(vs=-1) == INVALID and call(q=4096, qo=8192, qs=1023) == INVALID
    assert call(q=4096, qo=4096, qs=1024, qos=2048) == INVALID                # in place with another stride
    lib.spla_rope_destroy(r64)
    lib.spla_paged_destroy(h)


def test_attend_arguments(lib):
    _, h = paged(lib)
    b = batch()
    n = C.c_size_t()
    assert lib.spla_paged_query_workspace(h, C.addressof(b), C.byref(n)) == OK
    assert lib.spla_paged_query_workspace(h, C.addressof(b), None) == INVALID and lib.spla_paged_query_workspace(None, C.addressof(b), C.byref(n)) == INVALID
    m = lambda **kw: binding.SplaPagedMask(*{**dict(softcap=0.0, window=0, slopes=None, first_key=None, prefix_lens=None), **kw}.values())  # noqa: E731

    def call(paged_h=h, q=4096, qs=0, mask=None, out=8192, lse=None, ws=1 << 20, nb=1 << 40, bb=b):
        return lib.spla_paged_attend(paged_h, C.addressof(bb), q, qs, C.addressof(mask) if mask else None, out, lse, ws, nb, None)

    assert call(paged_h=None) == INVALID and call(q=None) == INVALID and call(out=None) == INVALID
    assert call(q=4097) == INVALID and call(out=8192 + 8) == INVALID and call(lse=4098) == INVALID and call(qs=1023) == INVALID and call(qs=-1024) == INVALID
    assert call(ws=(1 << 20) + 16) == INVALID
    for bad in (dict(softcap=-1.0), dict(softcap=math.nan), dict(softcap=math.inf), dict(softcap=1e-7), dict(window=-1), dict(slopes=4098), dict(first_key=4097), dict(prefix_lens=4099)):
        assert call(mask=m(**bad)) == INVALID, bad
    long = batch(max_len=1 << 20, table_stride=1 << 14)
    assert lib.spla_paged_query_workspace(h, C.addressof(long), C.byref(n)) == OK and n.value > 0
    assert call(bb=long, ws=None, nb=0) == INVALID and call(bb=long, nb=n.value - 1) == INVALID
    lib.spla_paged_destroy(h)
    assert lib.spla_paged_destroy(None) == OK


def test_wait_hook_arguments(lib):
    _, h = paged(lib)
    hook = lib.spla_paged_debug_wait_hook
    assert hook(None, 0, 0) == INVALID and hook(h, -1, 0) == INVALID and hook(h, 0, 8) == INVALID and hook(h, 0, -16) == INVALID
    assert hook(h, 1000, 16) == OK and hook(h, 0, 0) == OK
    lib.spla_paged_destroy(h)


def test_python_checks():
    with pytest.raises(ValueError, match="scaling"):
        binding.Rope(128, scaling="other")
    with pytest.raises(binding.SplaError):
        binding.Rope(128, rot_dim=3)
