"""Argument checks of the 8-bit cache, the head norms and the sinks: on the host, before anything touches a device."""
import ctypes as C
import math

import pytest
import torch

from paper_2601_22379_b200 import binding, build

OK, INVALID, UNSUPPORTED = binding.SPLA_OK, binding.SPLA_ERR_INVALID_ARG, binding.SPLA_ERR_UNSUPPORTED
PAGED = dict(n_q_heads=8, n_kv_heads=2, head_dim=128, page_size=64, n_pages=10, kv_dtype=binding.SPLA_BF16, q_dtype=binding.SPLA_BF16, page_stride=0, head_stride=0,
             sm_scale=0.0, flags=0)


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load()


def paged(lib, k=4096, v=8192, ks=16384, vs=32768, status=256, **kw):
    h = C.c_void_p()
    cfg = binding.SplaPagedConfig(*{**PAGED, **kw}.values())
    return lib.spla_paged_create_scaled(C.byref(cfg), k, v, ks, vs, status, C.byref(h)), h


def batch(**kw):
    return binding.SplaPagedBatch(*{**dict(cu_new=4, seq_lens=8, page_table=12, batch=2, total_new=5, max_new=3, max_len=128, table_stride=2), **kw}.values())


@pytest.mark.parametrize("kw,want", [
    (dict(), OK), (dict(head_dim=64, page_size=16), OK), (dict(kv_dtype=0, q_dtype=0), OK), (dict(page_stride=128, head_stride=64), OK),
    (dict(ks=None), INVALID), (dict(vs=None), INVALID), (dict(k=None), INVALID), (dict(k=4100), INVALID), (dict(status=None), INVALID),
    (dict(kv_dtype=0), UNSUPPORTED), (dict(q_dtype=0), UNSUPPORTED), (dict(kv_dtype=2, q_dtype=2), INVALID), (dict(page_stride=256), UNSUPPORTED), (dict(head_stride=128), UNSUPPORTED),
    (dict(head_dim=96), UNSUPPORTED), (dict(page_size=8), UNSUPPORTED), (dict(n_q_heads=34), UNSUPPORTED), (dict(n_q_heads=9), INVALID), (dict(flags=1), INVALID),
    (dict(sm_scale=math.inf), INVALID)])
def test_create(lib, kw, want):
    rc, h = paged(lib, **kw)
    assert rc == want
    lib.spla_paged_destroy(h)


def test_append_with_norms(lib):
    _, h = paged(lib)
    b = batch()
    norm = lambda q=4, k=8, eps=1e-6: C.addressof(keep.setdefault((q, k, eps), binding.SplaHeadNorm(q, k, eps)))  # noqa: E731
    keep = {}

    def call(p=h, n=None, k=4096, ks=0, v=8192, vs=0, q=None, qs=0, qo=None, qos=0):
        return lib.spla_paged_append_norm(p, C.addressof(b), None, None, n, k, ks, v, vs, q, qs, qo, qos, None)

    assert call(p=None) == INVALID and call(k=None) == INVALID and call(v=None) == INVALID and call(q=4096) == INVALID
    assert call(n=norm(eps=-1.0)) == INVALID and call(n=norm(eps=math.inf)) == INVALID and call(n=norm(eps=math.nan)) == INVALID and call(n=norm(q=5)) == INVALID and call(n=norm(k=6)) == INVALID
    assert call(k=4097) == INVALID and call(ks=255) == INVALID and call(vs=-1) == INVALID
    assert call(q=4096, qo=4096, qs=1024, qos=2048) == INVALID
    lib.spla_paged_destroy(h)


def test_read(lib):
    _, h = paged(lib)
    b = batch()
    call = lambda p=h, bb=b, k=4096, v=8192, t=1: lib.spla_paged_read(p, C.addressof(bb), k, v, t, None)  # noqa: E731
    assert call(p=None) == INVALID and call(k=None) == INVALID and call(v=None) == INVALID and call(t=2) == INVALID and call(t=-1) == INVALID
    assert call(k=4100) == INVALID and call(v=8200) == INVALID
    assert call(bb=batch(total_new=0)) == INVALID and call(bb=batch(max_len=129)) == INVALID and call(bb=batch(cu_new=None)) == INVALID
    assert call(bb=batch(max_len=(1 << 24) + 1, table_stride=1 << 20)) == UNSUPPORTED
    lib.spla_paged_destroy(h)


def test_attend_and_its_workspace(lib):
    _, h = paged(lib)
    n = C.c_size_t()
    assert lib.spla_paged_query_workspace(h, C.addressof(batch(max_new=3)), C.byref(n)) == OK
    few = n.value
    assert lib.spla_paged_query_workspace(h, C.addressof(batch(total_new=500, max_new=300, max_len=4096, table_stride=64)), C.byref(n)) == OK
    assert n.value >= few + 500 * 8 * (2 * 128 + 1)                           # queries in two parts and their exponents
    b = batch()
    mask = binding.SplaPagedMask(0.0, 10, None, 4, None)
    call = lambda q=4096, m=None, sinks=0, out=8192: lib.spla_paged_attend_sinks(h, C.addressof(b), q, 0, C.addressof(m) if m else None, sinks, out, None, 1 << 20, 1 << 40, None)  # noqa: E731
    assert call(q=None) == INVALID and call(out=None) == INVALID and call(out=8200) == INVALID and call(sinks=-1) == INVALID
    assert call(m=mask, sinks=2) == UNSUPPORTED
    assert lib.spla_paged_attend_sinks(h, C.addressof(batch(total_new=500, max_new=300, max_len=4096, table_stride=64)), 4096, 0, None, 0, 8192, None, 1 << 20, n.value - 1, None) == INVALID
    lib.spla_paged_destroy(h)


def rope(lib, dim=64):
    h = C.c_void_p()
    cfg = binding.SplaRopeConfig(dim, 0, 0, 0, 0.0, 0.0, 0.0, 0.0, 0.0, 0.0)
    assert lib.spla_rope_create(C.byref(cfg), C.byref(h)) == OK
    return h


def test_head_norms(lib):
    h = rope(lib)
    tensor = lambda i=4096, o=8192, n=2: binding.SplaRopeTensor(i, o, n, 0, 128, 64, 0, 128, 64)  # noqa: E731
    norm, only_q = binding.SplaHeadNorm(64, 128, 1e-6), binding.SplaHeadNorm(64, None, 1e-6)
    at = lambda x: None if x is None else C.addressof(x)  # noqa: E731

    def apply(r=h, pos=64, b=1, t=5, q=tensor(), k=None, dtype=1, n=norm):
        return lib.spla_rope_norm_apply(r, pos, b, t, at(q), at(k), dtype, at(n), None)

    assert apply(r=None) == INVALID and apply(pos=None) == INVALID and apply(q=None) == INVALID and apply(n=None) == INVALID and apply(b=0) == INVALID and apply(t=0) == INVALID
    assert apply(dtype=2) == INVALID and apply(k=tensor(), n=only_q) == INVALID and apply(n=binding.SplaHeadNorm(None, 64, 1e-6)) == INVALID
    assert apply(n=binding.SplaHeadNorm(64, 64, -1e-6)) == INVALID and apply(q=tensor(i=4097)) == INVALID and apply(q=tensor(n=0)) == INVALID and apply(q=tensor(o=None)) == INVALID
    assert apply(q=tensor(n=4097)) == UNSUPPORTED and apply(b=1 << 20, t=1 << 20) == UNSUPPORTED
    moved = tensor(o=4096)
    moved.out_token = 256
    assert apply(q=moved) == INVALID                                          # in place with other strides

    n = C.c_size_t()
    query = lib.spla_rope_norm_query_workspace
    assert query(h, 1, 5, 4, C.byref(n)) == OK and n.value > 0
    assert query(None, 1, 5, 4, C.byref(n)) == INVALID and query(h, 0, 5, 4, C.byref(n)) == INVALID and query(h, 1, 5, 0, C.byref(n)) == INVALID and query(h, 1, 5, 4, None) == INVALID
    assert query(h, 1 << 16, 1 << 16, 4, C.byref(n)) == UNSUPPORTED

    def backward(g=tensor(), q=tensor(o=None), gk=None, k=None, dq=64, dk=None, ws=1 << 20, nb=1 << 40, n=norm):
        return lib.spla_rope_norm_backward(h, 64, 1, 5, at(g), at(q), at(gk), at(k), 1, at(n), dq, dk, ws, nb, None)

    assert backward(g=None) == INVALID and backward(q=None) == INVALID and backward(dq=None) == INVALID and backward(ws=None) == INVALID and backward(ws=8) == INVALID and backward(nb=0) == INVALID
    assert backward(k=tensor()) == INVALID and backward(gk=tensor()) == INVALID and backward(gk=tensor(), k=tensor()) == INVALID    # (no dk_weight)
    assert backward(g=tensor(n=3)) == INVALID and backward(g=tensor(o=None)) == INVALID and backward(dq=65) == INVALID
    over = tensor(o=4096)
    over.out_token = 256
    assert backward(g=over) == INVALID
    lib.spla_rope_destroy(h)


# ---- what the binding refuses before it calls the library: tensors on the CPU, no device ------------------------------
def cache(hq=4, hkv=2, d=64, P=16, new=torch.bfloat16):
    c = binding.PagedCache.__new__(binding.PagedCache)
    c.k_pages = c.v_pages = torch.zeros(3, hkv, P, d, dtype=torch.uint8).view(torch.float8_e4m3fn)
    c.device, c.index = torch.device("cpu"), 0
    c.page_size, c.n_q_heads, c.n_kv_heads, c.head_dim, c.q_torch_dtype, c._new_dtype = P, hq, hkv, d, new, new
    return c


def sequences(total):
    i = lambda *x: torch.tensor(x, dtype=torch.int32)  # noqa: E731
    return i(0, total), i(total), torch.arange(3, dtype=torch.int32)[None]


def test_pages_of_other_types_or_shapes_are_refused():
    t = binding.PagedCache.pages(3, 2, 32, 64, device="cpu")
    assert t["k_pages"].shape == (3, 2, 32, 64) and t["k_scales"].shape == (3, 2, 2) and (t["v_scales"].float() == 1).all()
    for bad in (dict(), dict(k_scales=None), dict(k_pages=torch.zeros(3, 2, 32, 64)), dict(v_scales=t["v_scales"][:, :, :1])):   # (the first: on the CPU)
        with pytest.raises(ValueError, match="8_e4m3fn"):
            binding.PagedCache(**{**t, **bad}, n_q_heads=2)


def test_tokens_and_weights_of_other_types_are_refused():
    x, q = torch.zeros(5, 2, 64, dtype=torch.bfloat16), torch.zeros(5, 4, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="k "):
        cache().append(x.float(), x, *sequences(5), q=q)
    with pytest.raises(ValueError, match="q "):
        cache().append(x, x, *sequences(5), q=q.float())
    for w in (torch.ones(64, dtype=torch.bfloat16), torch.ones(32), torch.ones(128)[::2]):
        with pytest.raises(ValueError, match="weight"):
            cache().append(x, x, *sequences(5), q=q, k_weight=w)
    with pytest.raises(ValueError, match="read as"):
        cache().read(*sequences(5), 5, dtype=torch.float16)
    with pytest.raises(ValueError, match="k_out"):
        cache().read(*sequences(5), 5, k_out=torch.zeros(5, 2, 32, dtype=torch.bfloat16))


def test_head_norm_arguments():
    class R(binding.Rope):
        def __init__(self):
            self.head_dim = 64
    r = R()
    x, w, pos = torch.zeros(5, 2, 64), torch.ones(64), torch.zeros(5, dtype=torch.int32)
    with pytest.raises(ValueError, match="together"):
        r.norm_apply(pos, x, w, k=x)
    with pytest.raises(ValueError, match="together"):
        r.norm_backward(pos, x, x, w, k=x, k_weight=w)
    with pytest.raises(ValueError, match="positions"):
        r.norm_apply(pos.long(), x, w)
    with pytest.raises(ValueError, match="of the positions' batch and device"):
        r.norm_apply(pos, x, w)                                               # (a tensor on the CPU)
