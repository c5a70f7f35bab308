"""Thin ctypes binding of libspla.so: the same entry points as include/spla.h, argument marshalling only.

Every step of the decode path runs inside the CUDA library.  PyTorch is used here for device memory and
streams and nothing else; there is no CPU or eager fallback: if the shared library is missing or fails to load,
`load()` raises.
"""
from __future__ import annotations

import ctypes as C
import os
import struct
from dataclasses import dataclass

import torch

SPLA_OK, SPLA_ERR_INVALID_ARG, SPLA_ERR_CAPACITY, SPLA_ERR_CUDA, SPLA_ERR_UNSUPPORTED = 0, -1, -2, -3, -4
SPLA_ERR_TIMEOUT, SPLA_ERR_BOUNDS = -5, -6
SPLA_F32, SPLA_BF16 = 0, 1
SPLA_ADOPT_CONTENTS, SPLA_FIRST_ORDER, SPLA_NO_RLA, SPLA_GENERAL_KERNELS, SPLA_STATS_BF16, SPLA_DEBUG_BOUNDS = 1, 2, 4, 8, 16, 32

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libspla.so")

EXPORTS = ["spla_query_sizes", "spla_init_cache", "spla_append_tokens", "spla_decode", "spla_decode_selected",
           "spla_select_blocks_noalloc", "spla_select", "spla_append_decode", "spla_prefill",
           "spla_query_prefill_workspace",
           "spla_copy_scores", "spla_sync_status", "spla_set_length_bound", "spla_debug_wait_hook", "spla_destroy_cache",
           "spla_rope_create", "spla_rope_destroy", "spla_rope_apply", "spla_rope_norm_apply", "spla_rope_norm_backward",
           "spla_rope_norm_query_workspace", "spla_paged_create", "spla_paged_create_scaled", "spla_paged_destroy",
           "spla_paged_append", "spla_paged_append_norm", "spla_paged_read", "spla_paged_query_workspace", "spla_paged_attend",
           "spla_paged_attend_sinks", "spla_paged_sync_status", "spla_paged_debug_wait_hook",
           "spla_launch_count", "spla_status_string", "spla_last_cuda_error"]


class SplaConfig(C.Structure):
    _fields_ = [("batch", C.c_int32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32),
                ("block_size", C.c_int32), ("top_k", C.c_int32), ("max_context", C.c_int32),
                ("n_sink_blocks", C.c_int32), ("n_local_blocks", C.c_int32), ("kv_dtype", C.c_int32),
                ("q_dtype", C.c_int32), ("sm_scale", C.c_float), ("phi_scale", C.c_float), ("rms_eps", C.c_float),
                ("flags", C.c_uint32), ("window_size", C.c_int32), ("window_stride", C.c_int32)]

    @property
    def n_windows(self) -> int:
        """Selection windows per block (1 without strided windows)."""
        return (self.block_size - self.window_size) // self.window_stride + 1 if self.window_size > 0 else 1


class SplaBuffers(C.Structure):
    _fields_ = [("k_cache", C.c_void_p), ("v_cache", C.c_void_p), ("stats", C.c_void_p), ("rla_state", C.c_void_p),
                ("tok_lse", C.c_void_p), ("seq_lens", C.c_void_p), ("workspace", C.c_void_p),
                ("workspace_bytes", C.c_size_t)]


class SplaSizes(C.Structure):
    _fields_ = [(n, C.c_size_t) for n in ("k_cache", "v_cache", "stats", "rla_state", "tok_lse", "seq_lens",
                                          "workspace")]


class SplaRopeConfig(C.Structure):
    _fields_ = [("head_dim", C.c_int32), ("rot_dim", C.c_int32), ("interleaved", C.c_int32), ("scaling", C.c_int32),
                ("base", C.c_double), ("factor", C.c_double), ("original_len", C.c_double), ("ramp_low", C.c_double),
                ("ramp_high", C.c_double), ("amplitude", C.c_double)]


class SplaRopeTensor(C.Structure):
    _fields_ = [("in_", C.c_void_p), ("out", C.c_void_p), ("n_heads", C.c_int32),
                ("in_batch", C.c_int64), ("in_token", C.c_int64), ("in_head", C.c_int64),
                ("out_batch", C.c_int64), ("out_token", C.c_int64), ("out_head", C.c_int64)]


class SplaHeadNorm(C.Structure):
    _fields_ = [("q_weight", C.c_void_p), ("k_weight", C.c_void_p), ("eps", C.c_float)]


class SplaPagedConfig(C.Structure):
    _fields_ = [("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("page_size", C.c_int32),
                ("n_pages", C.c_int32), ("kv_dtype", C.c_int32), ("q_dtype", C.c_int32), ("page_stride", C.c_int64),
                ("head_stride", C.c_int64), ("sm_scale", C.c_float), ("flags", C.c_uint32)]


class SplaPagedBatch(C.Structure):
    _fields_ = [("cu_new", C.c_void_p), ("seq_lens", C.c_void_p), ("page_table", C.c_void_p), ("batch", C.c_int32),
                ("total_new", C.c_int32), ("max_new", C.c_int32), ("max_len", C.c_int32), ("table_stride", C.c_int32)]


class SplaPagedMask(C.Structure):
    _fields_ = [("softcap", C.c_float), ("window", C.c_int32), ("slopes", C.c_void_p), ("first_key", C.c_void_p),
                ("prefix_lens", C.c_void_p)]


_lib = None


def load(path: str | None = None) -> C.CDLL:
    """Loads the shared library (once).  Raises if it is absent: there is nothing to fall back to."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    p = path or LIB_PATH
    if not os.path.exists(p):
        raise RuntimeError(f"{p} not found: build it with `python -m paper_2601_22379_b200.build` "
                           "(the SPLA path has no fallback implementation)")
    lib = C.CDLL(p)
    vp, i32 = C.c_void_p, C.c_int32
    lib.spla_query_sizes.argtypes = [C.POINTER(SplaConfig), C.POINTER(SplaSizes)]
    lib.spla_init_cache.argtypes = [C.POINTER(SplaConfig), C.POINTER(SplaBuffers), vp, C.POINTER(vp)]
    lib.spla_append_tokens.argtypes = [vp, vp, vp, vp, i32, vp]
    lib.spla_decode.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp]
    lib.spla_decode_selected.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp]
    lib.spla_select.argtypes = [vp, vp, vp, vp]
    lib.spla_append_decode.argtypes = [vp, vp, vp, vp, i32, vp, vp, vp, vp, vp, vp, vp]
    lib.spla_select_blocks_noalloc.argtypes = [C.POINTER(SplaConfig), vp, vp, vp, vp, vp, vp, vp]
    lib.spla_prefill.argtypes = [vp, vp, vp, vp, i32, vp, vp, vp, vp, C.c_size_t, vp]
    lib.spla_query_prefill_workspace.argtypes = [C.POINTER(SplaConfig), i32, C.POINTER(C.c_size_t), C.POINTER(C.c_size_t)]
    lib.spla_copy_scores.argtypes = [vp, vp, vp]
    lib.spla_debug_wait_hook.argtypes = [vp, i32, i32]
    lib.spla_sync_status.argtypes = [vp, vp]
    lib.spla_set_length_bound.argtypes = [vp, i32]
    lib.spla_destroy_cache.argtypes = [vp]
    i64 = C.c_int64
    lib.spla_rope_create.argtypes = [C.POINTER(SplaRopeConfig), C.POINTER(vp)]
    lib.spla_rope_destroy.argtypes = [vp]
    lib.spla_rope_apply.argtypes = [vp, vp, i32, i32, vp, vp, i32, i32, vp]
    lib.spla_paged_create.argtypes = [C.POINTER(SplaPagedConfig), vp, vp, vp, C.POINTER(vp)]
    lib.spla_rope_norm_apply.argtypes = [vp, vp, i32, i32, vp, vp, i32, vp, vp]
    lib.spla_rope_norm_backward.argtypes = [vp, vp, i32, i32, vp, vp, vp, vp, i32, vp, vp, vp, vp, C.c_size_t, vp]
    lib.spla_rope_norm_query_workspace.argtypes = [vp, i32, i32, i32, C.POINTER(C.c_size_t)]
    lib.spla_paged_create_scaled.argtypes = [C.POINTER(SplaPagedConfig), vp, vp, vp, vp, vp, C.POINTER(vp)]
    lib.spla_paged_append_norm.argtypes = [vp, vp, vp, vp, vp, vp, i64, vp, i64, vp, i64, vp, i64, vp]
    lib.spla_paged_read.argtypes = [vp, vp, vp, vp, i32, vp]
    lib.spla_paged_attend_sinks.argtypes = [vp, vp, vp, i64, vp, i32, vp, vp, vp, C.c_size_t, vp]
    lib.spla_paged_destroy.argtypes = [vp]
    lib.spla_paged_append.argtypes = [vp, vp, vp, vp, vp, i64, vp, i64, vp, i64, vp, i64, vp]
    lib.spla_paged_query_workspace.argtypes = [vp, vp, C.POINTER(C.c_size_t)]
    lib.spla_paged_attend.argtypes = [vp, vp, vp, i64, vp, vp, vp, vp, C.c_size_t, vp]
    lib.spla_paged_sync_status.argtypes = [vp, vp]
    lib.spla_paged_debug_wait_hook.argtypes = [vp, i32, i32]
    for name in EXPORTS[:-3]:
        getattr(lib, name).restype = C.c_int
    lib.spla_launch_count.argtypes = []
    lib.spla_launch_count.restype = C.c_ulonglong
    lib.spla_status_string.argtypes = [C.c_int]
    lib.spla_status_string.restype = C.c_char_p
    lib.spla_last_cuda_error.argtypes = []
    lib.spla_last_cuda_error.restype = C.c_char_p
    if path is None:
        _lib = lib
    return lib


class SplaError(RuntimeError):
    def __init__(self, status: int, where: str):
        lib = load()
        msg = lib.spla_status_string(status).decode()
        extra = lib.spla_last_cuda_error().decode() if status == SPLA_ERR_CUDA else ""
        super().__init__(f"{where}: {msg} ({status}) {extra}".strip())
        self.status = status


def _check(status: int, where: str):
    if status != SPLA_OK:
        raise SplaError(status, where)


def _ptr(t) -> int | None:
    return None if t is None else t.data_ptr()


def _stream() -> int:
    return torch.cuda.current_stream().cuda_stream


def make_config(*, batch, n_q_heads, n_kv_heads, head_dim, block_size, top_k, max_context, n_sink_blocks=1,
                n_local_blocks=4, kv_dtype="bf16", q_dtype=None, sm_scale=0.0, phi_scale=0.0, rms_eps=0.0,
                flags=0, window_size=0, window_stride=0) -> SplaConfig:
    code = {"bf16": SPLA_BF16, "f32": SPLA_F32}
    return SplaConfig(batch, n_q_heads, n_kv_heads, head_dim, block_size, top_k, max_context, n_sink_blocks,
                      n_local_blocks, code[kv_dtype], code[q_dtype or kv_dtype], sm_scale, phi_scale, rms_eps, flags,
                      window_size, window_stride)


def query_sizes(cfg: SplaConfig) -> SplaSizes:
    sz = SplaSizes()
    _check(load().spla_query_sizes(C.byref(cfg), C.byref(sz)), "spla_query_sizes")
    return sz


@dataclass
class _Bufs:
    k_cache: torch.Tensor
    v_cache: torch.Tensor
    stats: torch.Tensor
    rla_state: torch.Tensor
    tok_lse: torch.Tensor
    seq_lens: torch.Tensor
    workspace: torch.Tensor


NOALLOC_SCRATCH_BYTES = 4 << 20


def select_blocks_noalloc(cfg: SplaConfig, stats: torch.Tensor, seq_lens: torch.Tensor, q: torch.Tensor,
                          sel_idx: torch.Tensor, scores_out: torch.Tensor | None = None,
                          status_out: torch.Tensor | None = None) -> int:
    """Score + select for callers that may not allocate on the device: every tensor is passed in, the kernel's
    scratch is a fixed array inside the library.  Returns the status code (0 = ok) instead of raising, so that a
    caller can fall back to `SplaCache.decode` when the configuration exceeds the fixed scratch.  Calls share
    that scratch: never let two of them overlap on the GPU."""
    assert stats.is_cuda and stats.dtype == torch.float32 and stats.is_contiguous()
    assert seq_lens.dtype == torch.int32 and sel_idx.dtype == torch.int32 and q.is_contiguous()
    with torch.cuda.device(stats.device):
        return load().spla_select_blocks_noalloc(C.byref(cfg), stats.data_ptr(), seq_lens.data_ptr(), q.data_ptr(),
                                                 sel_idx.data_ptr(), _ptr(scores_out), _ptr(status_out), _stream())


def launch_count() -> int:
    """Kernels the library has launched (or recorded into a graph capture) from this thread so far."""
    return int(load().spla_launch_count())


class SplaCache:
    """Owns the device buffers (as torch tensors) of one cache and forwards to the C ABI.

    Shapes follow include/spla.h: k_cache/v_cache [batch, H_kv, max_blocks, B, d], stats
    [batch, H_kv, max_blocks, 2, d] (with strided windows [batch, H_kv, max_blocks, NW, 2, d]; fp32, or bfloat16
    with SPLA_STATS_BF16), rla_state
    [batch, H_kv, d, d], tok_lse [batch, H_kv, max_blocks * B].
    """

    def __init__(self, cfg: SplaConfig, device="cuda:0"):
        self.lib = load()
        self.cfg = cfg
        self.device = torch.device(device)
        sz = query_sizes(cfg)
        self.sizes = sz
        B, d = cfg.block_size, cfg.head_dim
        self.max_blocks = (cfg.max_context + B - 1) // B
        kv_t = torch.bfloat16 if cfg.kv_dtype == SPLA_BF16 else torch.float32
        self.kv_torch_dtype = kv_t
        self.q_torch_dtype = torch.bfloat16 if cfg.q_dtype == SPLA_BF16 else torch.float32
        shp = (cfg.batch, cfg.n_kv_heads, self.max_blocks)
        dev = self.device
        self.bufs = _Bufs(
            k_cache=torch.empty(*shp, B, d, dtype=kv_t, device=dev),
            v_cache=torch.empty(*shp, B, d, dtype=kv_t, device=dev),
            stats=torch.empty(*shp, *((cfg.n_windows,) if cfg.window_size > 0 else ()), 2, d, device=dev,
                              dtype=torch.bfloat16 if cfg.flags & SPLA_STATS_BF16 else torch.float32),
            rla_state=torch.empty(cfg.batch, cfg.n_kv_heads, d, d, dtype=torch.float32, device=dev),
            tok_lse=torch.empty(cfg.batch, cfg.n_kv_heads, self.max_blocks * B, dtype=torch.float32, device=dev),
            seq_lens=torch.empty(cfg.batch, dtype=torch.int32, device=dev),
            workspace=torch.empty(sz.workspace, dtype=torch.uint8, device=dev),
        )
        b = self.bufs
        assert b.k_cache.numel() * b.k_cache.element_size() == sz.k_cache
        assert b.stats.numel() * b.stats.element_size() == sz.stats and b.tok_lse.numel() * 4 == sz.tok_lse
        cb = SplaBuffers(b.k_cache.data_ptr(), b.v_cache.data_ptr(), b.stats.data_ptr(), b.rla_state.data_ptr(),
                         b.tok_lse.data_ptr(), b.seq_lens.data_ptr(), b.workspace.data_ptr(), sz.workspace)
        self.handle = C.c_void_p()
        with torch.cuda.device(self.device):
            _check(self.lib.spla_init_cache(C.byref(cfg), C.byref(cb), _stream(), C.byref(self.handle)),
                   "spla_init_cache")

    # -- the three calls of the path -------------------------------------------------------------------
    def append_tokens(self, k_new: torch.Tensor, v_new: torch.Tensor, n_new: torch.Tensor | None = None):
        """k_new, v_new: [batch, H_kv, max_new, d] contiguous device tensors of the cache dtype."""
        cfg = self.cfg
        assert k_new.is_cuda and k_new.is_contiguous() and v_new.is_contiguous()
        assert k_new.dtype == self.kv_torch_dtype and v_new.dtype == self.kv_torch_dtype
        assert k_new.shape == v_new.shape and k_new.shape[0] == cfg.batch and k_new.shape[1] == cfg.n_kv_heads
        assert k_new.shape[3] == cfg.head_dim
        if n_new is not None:
            assert n_new.dtype == torch.int32 and n_new.is_cuda and n_new.numel() == cfg.batch
        with torch.cuda.device(self.device):
            _check(self.lib.spla_append_tokens(self.handle, k_new.data_ptr(), v_new.data_ptr(), _ptr(n_new),
                                               k_new.shape[2], _stream()), "spla_append_tokens")

    def decode(self, q: torch.Tensor, rms_weight: torch.Tensor | None, out: torch.Tensor | None = None,
               sel_idx: torch.Tensor | None = None, dbg_o_sparse=None, dbg_o_rla=None) -> torch.Tensor:
        """q: [batch, H_q, d] of the query dtype; returns out [batch, H_q, d] fp32."""
        cfg = self.cfg
        assert q.is_cuda and q.is_contiguous() and q.dtype == self.q_torch_dtype
        assert tuple(q.shape) == (cfg.batch, cfg.n_q_heads, cfg.head_dim)
        if out is None:
            out = torch.empty(cfg.batch, cfg.n_q_heads, cfg.head_dim, dtype=torch.float32, device=self.device)
        with torch.cuda.device(self.device):
            _check(self.lib.spla_decode(self.handle, q.data_ptr(), _ptr(rms_weight), out.data_ptr(), _ptr(sel_idx),
                                        _ptr(dbg_o_sparse), _ptr(dbg_o_rla), _stream()), "spla_decode")
        return out

    def append_decode(self, k_new: torch.Tensor, v_new: torch.Tensor, q: torch.Tensor, rms_weight, out=None,
                      n_new: torch.Tensor | None = None, sel_idx=None, dbg_o_sparse=None, dbg_o_rla=None) -> torch.Tensor:
        """One step: `append_tokens(k_new, v_new, n_new)` then `decode(q, ...)`, as one call."""
        cfg = self.cfg
        assert k_new.is_cuda and k_new.is_contiguous() and v_new.is_contiguous() and k_new.shape == v_new.shape
        assert k_new.dtype == self.kv_torch_dtype and v_new.dtype == self.kv_torch_dtype
        assert tuple(k_new.shape[:2]) == (cfg.batch, cfg.n_kv_heads) and k_new.shape[3] == cfg.head_dim
        assert q.is_cuda and q.is_contiguous() and q.dtype == self.q_torch_dtype
        assert tuple(q.shape) == (cfg.batch, cfg.n_q_heads, cfg.head_dim)
        if n_new is not None:
            assert n_new.dtype == torch.int32 and n_new.is_cuda and n_new.numel() == cfg.batch
        if out is None:
            out = torch.empty(cfg.batch, cfg.n_q_heads, cfg.head_dim, dtype=torch.float32, device=self.device)
        with torch.cuda.device(self.device):
            _check(self.lib.spla_append_decode(self.handle, k_new.data_ptr(), v_new.data_ptr(), _ptr(n_new),
                                               k_new.shape[2], q.data_ptr(), _ptr(rms_weight), out.data_ptr(),
                                               _ptr(sel_idx), _ptr(dbg_o_sparse), _ptr(dbg_o_rla), _stream()),
                   "spla_append_decode")
        return out

    def prefill(self, k_new: torch.Tensor, v_new: torch.Tensor, q: torch.Tensor, rms_weight, out=None, sel_idx=None,
                workspace_bytes: int | None = None) -> torch.Tensor:
        """Prefill-shaped forward: appends T tokens per sequence and returns the output of every position.
        k_new, v_new [batch, H_kv, T, d]; q [batch, T, H_q, d]; out [batch, T, H_q, d] fp32;
        sel_idx (optional) [batch, T, H_kv, top_k] int32.  `workspace_bytes`: scratch to use (default: the size the
        library recommends; at least the minimum it reports)."""
        cfg = self.cfg
        T = k_new.shape[2]
        assert k_new.is_cuda and k_new.is_contiguous() and v_new.is_contiguous() and k_new.shape == v_new.shape
        assert k_new.dtype == self.kv_torch_dtype and tuple(k_new.shape[:2]) == (cfg.batch, cfg.n_kv_heads)
        assert q.is_contiguous() and q.dtype == self.q_torch_dtype and tuple(q.shape) == (cfg.batch, T, cfg.n_q_heads, cfg.head_dim)
        lo, good = C.c_size_t(), C.c_size_t()
        _check(self.lib.spla_query_prefill_workspace(C.byref(cfg), T, C.byref(lo), C.byref(good)), "spla_query_prefill_workspace")
        nbytes = good.value if workspace_bytes is None else max(int(workspace_bytes), lo.value)
        ws = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        if out is None:
            out = torch.empty(cfg.batch, T, cfg.n_q_heads, cfg.head_dim, dtype=torch.float32, device=self.device)
        with torch.cuda.device(self.device):
            _check(self.lib.spla_prefill(self.handle, k_new.data_ptr(), v_new.data_ptr(), q.data_ptr(), T, _ptr(rms_weight),
                                         out.data_ptr(), _ptr(sel_idx), ws.data_ptr(), nbytes, _stream()), "spla_prefill")
        self._prefill_ws = ws                                  # keep the scratch alive until the stream has used it
        return out

    def select(self, q: torch.Tensor, sel_idx: torch.Tensor | None = None) -> torch.Tensor:
        """Block scores + top-k only; returns sel_idx [batch, H_kv, top_k] int32."""
        assert q.is_cuda and q.is_contiguous() and q.dtype == self.q_torch_dtype
        if sel_idx is None:
            sel_idx = self.new_sel_buffer()
        with torch.cuda.device(self.device):
            _check(self.lib.spla_select(self.handle, q.data_ptr(), sel_idx.data_ptr(), _stream()), "spla_select")
        return sel_idx

    def decode_selected(self, q, rms_weight, sel_in: torch.Tensor, out=None, dbg_o_sparse=None, dbg_o_rla=None):
        cfg = self.cfg
        assert q.is_cuda and q.is_contiguous() and q.dtype == self.q_torch_dtype
        assert sel_in.dtype == torch.int32 and sel_in.is_contiguous()
        assert tuple(sel_in.shape) == (cfg.batch, cfg.n_kv_heads, cfg.top_k)
        if out is None:
            out = torch.empty(cfg.batch, cfg.n_q_heads, cfg.head_dim, dtype=torch.float32, device=self.device)
        with torch.cuda.device(self.device):
            _check(self.lib.spla_decode_selected(self.handle, q.data_ptr(), _ptr(rms_weight), sel_in.data_ptr(),
                                                 out.data_ptr(), _ptr(dbg_o_sparse), _ptr(dbg_o_rla), _stream()),
                   "spla_decode_selected")
        return out

    # -- helpers ------------------------------------------------------------------------------------------
    def scores(self) -> torch.Tensor:
        out = torch.empty(self.cfg.batch, self.cfg.n_kv_heads, self.max_blocks, dtype=torch.float32,
                          device=self.device)
        with torch.cuda.device(self.device):
            _check(self.lib.spla_copy_scores(self.handle, out.data_ptr(), _stream()), "spla_copy_scores")
        return out

    def sync_status(self) -> int:
        with torch.cuda.device(self.device):
            return self.lib.spla_sync_status(self.handle, _stream())

    def debug_wait_hook(self, max_wait_polls: int, extra_expected_bytes: int):
        """Test hook: wait limit of the kernels' copy barriers (decode, prefill, bulk append) and bytes they expect in excess (see spla.h)."""
        _check(self.lib.spla_debug_wait_hook(self.handle, max_wait_polls, extra_expected_bytes), "spla_debug_wait_hook")

    def set_length_bound(self, n: int):
        _check(self.lib.spla_set_length_bound(self.handle, n), "spla_set_length_bound")

    def new_sel_buffer(self) -> torch.Tensor:
        return torch.empty(self.cfg.batch, self.cfg.n_kv_heads, self.cfg.top_k, dtype=torch.int32, device=self.device)

    def close(self):
        if getattr(self, "handle", None) is not None and self.handle.value:
            self.lib.spla_destroy_cache(self.handle)
            self.handle = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# ---- rotary positions and the paged cache ---------------------------------------------------------------------------
_TYPE_CODE = {torch.bfloat16: SPLA_BF16, torch.float32: SPLA_F32}
# The structures of the calls of a step, packed in one go: a ctypes.Structure takes 0.1 us per field
_pack_rope_tensor = struct.Struct("@PPi6q").pack
_pack_batch = struct.Struct("@PPP5i4x").pack
_pack_mask = struct.Struct("@fiPPP").pack
_pack_norm = struct.Struct("@PPf4x").pack
# (torch's own short ways to the current device and stream, 0.1 us each, where there are any: a torch without CUDA has none)
_device_now = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
_stream_now = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)
assert struct.calcsize("@PPi6q") == C.sizeof(SplaRopeTensor) and struct.calcsize("@PPP5i4x") == C.sizeof(SplaPagedBatch)
assert struct.calcsize("@fiPPP") == C.sizeof(SplaPagedMask) and struct.calcsize("@PPf4x") == C.sizeof(SplaHeadNorm)


def _on(index: int, fn, *args) -> int:
    """fn(*args, stream) with device `index` the current one and its current stream as the last argument."""
    before = _device_now()
    if before == index:
        return fn(*args, _stream_now(index))
    torch.cuda.set_device(index)
    try:
        return fn(*args, _stream_now(index))
    finally:
        torch.cuda.set_device(before)


def _norm_weight(w: torch.Tensor, head_dim: int, device) -> int:
    """Address of a norm's weight."""
    if not (w.dtype is torch.float32 and w.shape == (head_dim,) and w.device == device and w.is_contiguous()):
        raise ValueError("head norm: a weight fp32 [head_dim] on the device of what it weighs, contiguous")
    return w.data_ptr()


class Rope:
    """Rotary positions: the frequencies of one configuration, for all layers and steps (`spla_rope_create`).

    `rot_dim` channels of every head are rotated (default: all), channel i with i + rot_dim / 2, or 2 i with 2 i + 1 where
    `interleaved`.  `scaling`: "none", "linear", "base" or "ramp" (see spla_rope_scaling_t); `ramp` = (low, high)."""

    SCALING = {"none": 0, "linear": 1, "base": 2, "ramp": 3}

    def __init__(self, head_dim: int, rot_dim: int = 0, base: float = 10000.0, interleaved: bool = False, scaling: str = "none",
                 factor: float = 1.0, original_len: float = 0.0, ramp=(1.0, 32.0), amplitude: float = 1.0):
        if scaling not in self.SCALING:
            raise ValueError(f"rope: scaling must be one of {sorted(self.SCALING)}")
        self.lib = load()
        self.head_dim = head_dim
        self._norm_bytes = (None, 0)
        cfg = SplaRopeConfig(head_dim, rot_dim, int(interleaved), self.SCALING[scaling], base, factor, original_len, ramp[0], ramp[1], amplitude)
        self.handle = C.c_void_p()
        _check(self.lib.spla_rope_create(C.byref(cfg), C.byref(self.handle)), "spla_rope_create")

    def _tensor(self, x: torch.Tensor, out: torch.Tensor | None, shape, dtype, device):
        """`out` and the packed descriptor of x -> out, for positions of `shape`."""
        xshape, xs = x.shape, x.stride()
        if not (xshape[:-2] == shape and xshape[-1] == self.head_dim and xs[-1] == 1 and x.dtype is dtype and x.device == device and x.is_cuda):
            raise ValueError("rope: tensors [batch, tokens, heads, head_dim] or [tokens, heads, head_dim] of the positions' batch and device, "
                             "of one type, bf16 or fp32, channels contiguous")
        if out is None:
            out = torch.empty_like(x)                                        # (the strides of x where they are dense)
            ys = out.stride()
            if ys[-1] != 1:
                out = x.new_empty(xshape)
                ys = out.stride()
        else:
            ys = out.stride()
            if not (out.shape == xshape and out.dtype is dtype and out.device == device and ys[-1] == 1):
                raise ValueError("rope: an output like its input, channels contiguous")
            if 0 in ys and any(y == 0 and n > 1 for y, n in zip(ys, xshape)):
                raise ValueError("rope: an output whose elements lie on each other")
        if len(xs) == 3:
            return out, _pack_rope_tensor(x.data_ptr(), out.data_ptr(), xshape[1], 0, xs[0], xs[1], 0, ys[0], ys[1])
        return out, _pack_rope_tensor(x.data_ptr(), out.data_ptr(), xshape[2], xs[0], xs[1], xs[2], ys[0], ys[1], ys[2])

    def apply(self, positions: torch.Tensor, q: torch.Tensor, k: torch.Tensor | None = None, q_out: torch.Tensor | None = None,
              k_out: torch.Tensor | None = None, transpose: bool = False):
        """Rotates q (and k) to `positions` (int32 [batch, tokens] or [tokens]); any strides, channels contiguous.  `q_out=q`
        works in place.  `transpose`: the gradient of the rotation.  Returns q_out, or (q_out, k_out)."""
        shape, dtype, device = positions.shape, q.dtype, positions.device
        if not (positions.dtype is torch.int32 and positions.is_contiguous() and 1 <= len(shape) <= 2 and dtype in _TYPE_CODE):
            raise ValueError("rope: positions int32 [batch, tokens] or [tokens], contiguous; q bf16 or fp32")
        q_out, tq = self._tensor(q, q_out, shape, dtype, device)
        tk = None
        if k is not None:
            k_out, tk = self._tensor(k, k_out, shape, dtype, device)
        n = shape[-1]
        batch = shape[0] if len(shape) == 2 else 1
        if n and batch:
            rc = _on(device.index, self.lib.spla_rope_apply, self.handle, positions.data_ptr(), batch, n, tq, tk, _TYPE_CODE[dtype], 1 if transpose else 0)
            if rc != SPLA_OK:
                raise SplaError(rc, "spla_rope_apply")
        return q_out if k is None else (q_out, k_out)

    def _places(self, positions, q):
        shape, dtype, device = positions.shape, q.dtype, positions.device
        if not (positions.dtype is torch.int32 and positions.is_contiguous() and 1 <= len(shape) <= 2 and dtype in _TYPE_CODE):
            raise ValueError("rope: positions int32 [batch, tokens] or [tokens], contiguous; q bf16 or fp32")
        return shape, dtype, device, shape[0] if len(shape) == 2 else 1, shape[-1]

    def norm_apply(self, positions: torch.Tensor, q: torch.Tensor, q_weight: torch.Tensor, k: torch.Tensor | None = None,
                   k_weight: torch.Tensor | None = None, eps: float = 1e-6, q_out: torch.Tensor | None = None, k_out: torch.Tensor | None = None):
        """Norms every head of q (and k) over its channels, times the weight (fp32 [head_dim]), and rotates it to `positions`, in one pass:
        `apply(x / sqrt(mean(x^2) + eps) * weight)`.  Tensors as for `apply`.  Returns q_out, or (q_out, k_out)."""
        shape, dtype, device, batch, n = self._places(positions, q)
        if (k is None) != (k_weight is None):
            raise ValueError("head norm: k and k_weight go together")
        q_out, tq = self._tensor(q, q_out, shape, dtype, device)
        tk = None
        if k is not None:
            k_out, tk = self._tensor(k, k_out, shape, dtype, device)
        norm = _pack_norm(_norm_weight(q_weight, self.head_dim, device), 0 if k is None else _norm_weight(k_weight, self.head_dim, device), eps)
        if n and batch:
            rc = _on(device.index, self.lib.spla_rope_norm_apply, self.handle, positions.data_ptr(), batch, n, tq, tk, _TYPE_CODE[dtype], norm)
            if rc != SPLA_OK:
                raise SplaError(rc, "spla_rope_norm_apply")
        return q_out if k is None else (q_out, k_out)

    def norm_backward(self, positions: torch.Tensor, dq_out: torch.Tensor, q: torch.Tensor, q_weight: torch.Tensor, dk_out: torch.Tensor | None = None,
                      k: torch.Tensor | None = None, k_weight: torch.Tensor | None = None, eps: float = 1e-6, dq: torch.Tensor | None = None,
                      dk: torch.Tensor | None = None):
        """The gradients of `norm_apply(positions, q, q_weight, k, k_weight, eps)` for dq_out, dk_out of its outputs: (dq, dq_weight), or
        (dq, dq_weight, dk, dk_weight); those of the weights in fp32.  `dq=dq_out` works in place."""
        shape, dtype, device, batch, n = self._places(positions, q)
        if not (k is None) == (k_weight is None) == (dk_out is None):
            raise ValueError("head norm: k, k_weight and dk_out go together")
        _, xq = self._input(q, shape, dtype, device)
        if dq_out.shape != q.shape or (k is not None and dk_out.shape != k.shape):
            raise ValueError("head norm: gradients like their tensors")
        dq, tq = self._tensor(dq_out, dq, shape, dtype, device)
        xk = tk = dk_weight = None
        heads, wk = q.shape[-2], 0
        if k is not None:
            _, xk = self._input(k, shape, dtype, device)
            dk, tk = self._tensor(dk_out, dk, shape, dtype, device)
            heads += k.shape[-2]
            wk = _norm_weight(k_weight, self.head_dim, device)
        norm = _pack_norm(_norm_weight(q_weight, self.head_dim, device), wk, eps)
        if n and batch:
            sizes, nbytes = self._norm_bytes                                 # (of the last call: a training loop asks for the same again and again)
            if sizes != (batch, n, heads, device.index):
                out = C.c_size_t()
                rc = _on(device.index, lambda *a: self.lib.spla_rope_norm_query_workspace(*a[:-1]), self.handle, batch, n, heads, C.byref(out))
                if rc != SPLA_OK:
                    raise SplaError(rc, "spla_rope_norm_query_workspace")
                nbytes = out.value
                self._norm_bytes = (batch, n, heads, device.index), nbytes
            # the weights' gradients and the call's own scratch, from the stream's pool
            dq_weight = torch.empty(self.head_dim, dtype=torch.float32, device=device)
            if k is not None:
                dk_weight = torch.empty(self.head_dim, dtype=torch.float32, device=device)
            ws = torch.empty(nbytes, dtype=torch.uint8, device=device)
            rc = _on(device.index, self.lib.spla_rope_norm_backward, self.handle, positions.data_ptr(), batch, n, tq, xq, tk, xk, _TYPE_CODE[dtype], norm,
                     dq_weight.data_ptr(), _ptr(dk_weight), ws.data_ptr(), nbytes)
            if rc != SPLA_OK:
                raise SplaError(rc, "spla_rope_norm_backward")
        else:
            dq_weight = torch.zeros(self.head_dim, dtype=torch.float32, device=device)
            dk_weight = None if k is None else torch.zeros(self.head_dim, dtype=torch.float32, device=device)
        return (dq, dq_weight) if k is None else (dq, dq_weight, dk, dk_weight)

    def _input(self, x, shape, dtype, device):
        """The packed descriptor of an input alone (its strides may be 0)."""
        xshape, xs = x.shape, x.stride()
        if not (xshape[:-2] == shape and xshape[-1] == self.head_dim and xs[-1] == 1 and x.dtype is dtype and x.device == device and x.is_cuda):
            raise ValueError("rope: tensors [batch, tokens, heads, head_dim] or [tokens, heads, head_dim] of the positions' batch and device, "
                             "of one type, bf16 or fp32, channels contiguous")
        s = (0, *xs) if len(xs) == 3 else xs
        return None, _pack_rope_tensor(x.data_ptr(), x.data_ptr(), xshape[-2], s[0], s[1], s[2], s[0], s[1], s[2])

    def close(self):
        if getattr(self, "handle", None) is not None and self.handle.value:
            self.lib.spla_rope_destroy(self.handle)
            self.handle = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class PagedCache:
    """K/V in pages (`spla_paged_create`): k_pages, v_pages [n_pages, H_kv, P, d], bf16 or fp32, kept by the caller's tensors.

    Or in 8 bits (`spla_paged_create_scaled`): k_pages, v_pages torch.float8_e4m3fn with k_scales, v_scales torch.float8_e8m0fnu
    [n_pages, H_kv, P / 16], a power of two for every 16 tokens of a head; new tokens and queries have the type `q_dtype`.  `PagedCache.pages`
    makes the tensors.

    New tokens of all sequences come as one list of rows: cu_new int32 [batch + 1] says which rows are whose, seq_lens int32 [batch]
    how many tokens a sequence has with them, page_table int32 [batch, columns] where they lie."""

    _of_spla = False
    _new_dtype = None                                                        # of new tokens, where it is not the pages'

    def __init__(self, k_pages: torch.Tensor, v_pages: torch.Tensor, n_q_heads: int, q_dtype: str | None = None, sm_scale: float = 0.0, flags: int = 0,
                 k_scales: torch.Tensor | None = None, v_scales: torch.Tensor | None = None):
        if k_scales is not None or v_scales is not None:
            self._create_scaled(k_pages, v_pages, n_q_heads, q_dtype or "bf16", sm_scale, flags, k_scales, v_scales)
            return
        if not (k_pages.is_cuda and k_pages.dim() == 4 and k_pages.is_contiguous() and v_pages.is_contiguous() and k_pages.dtype in _TYPE_CODE
                and v_pages.shape == k_pages.shape and v_pages.dtype == k_pages.dtype and v_pages.device == k_pages.device):
            raise ValueError("paged cache: contiguous k_pages, v_pages [n_pages, H_kv, P, d] of one type and device")
        n_pages, hkv, P, d = k_pages.shape
        self._create(k_pages, v_pages, n_pages, hkv, P, d, 0, 0, n_q_heads, q_dtype, sm_scale, flags)

    def _create_scaled(self, k, v, n_q_heads, q_dtype, sm_scale, flags, ks, vs):
        e4m3, e8m0 = torch.float8_e4m3fn, torch.float8_e8m0fnu
        if not (k.is_cuda and k.dim() == 4 and k.dtype == v.dtype == e4m3 and v.shape == k.shape and ks is not None and vs is not None
                and ks.dtype == vs.dtype == e8m0 and ks.shape == vs.shape == (k.shape[0], k.shape[1], k.shape[2] // 16)
                and all(x.is_contiguous() and x.device == k.device for x in (k, v, ks, vs))):
            raise ValueError("paged cache: contiguous float8_e4m3fn k_pages, v_pages [n_pages, H_kv, P, d] and float8_e8m0fnu k_scales, v_scales "
                             "[n_pages, H_kv, P / 16] of one device")
        n_pages, hkv, P, d = k.shape
        self.k_scales, self.v_scales = ks, vs
        self._new_dtype = {"bf16": torch.bfloat16, "f32": torch.float32}[q_dtype]
        self._create(k, v, n_pages, hkv, P, d, 0, 0, n_q_heads, q_dtype, sm_scale, flags)

    @staticmethod
    def pages(n_pages: int, n_kv_heads: int, page_size: int, head_dim: int, device="cuda") -> dict:
        """The tensors of an 8-bit cache without tokens, as `PagedCache(**PagedCache.pages(...), n_q_heads=...)` takes them."""
        values = lambda: torch.zeros(n_pages, n_kv_heads, page_size, head_dim, dtype=torch.uint8, device=device).view(torch.float8_e4m3fn)  # noqa: E731
        scales = lambda: torch.full((n_pages, n_kv_heads, page_size // 16), 127, dtype=torch.uint8, device=device).view(torch.float8_e8m0fnu)  # noqa: E731
        return dict(k_pages=values(), v_pages=values(), k_scales=scales(), v_scales=scales())

    @classmethod
    def of(cls, cache: SplaCache, sm_scale: float | None = None, flags: int = 0) -> "PagedCache":
        """The K/V of an SPLA cache as pages (its blocks), for dense attention over it: `table()` names the pages.  Read only: tokens are appended by
        the SPLA cache, whose statistics, state and lengths go with them."""
        cfg, self = cache.cfg, cls.__new__(cls)
        hkv, B, mb = cfg.n_kv_heads, cfg.block_size, cache.max_blocks
        n_pages = (cfg.batch - 1) * hkv * mb + mb
        self._create(cache.bufs.k_cache, cache.bufs.v_cache, n_pages, hkv, B, cfg.head_dim, B, mb * B, cfg.n_q_heads,
                     "bf16" if cfg.q_dtype == SPLA_BF16 else "f32", cfg.sm_scale if sm_scale is None else sm_scale, flags)
        self._of_spla = True
        self._table = (torch.arange(cfg.batch, dtype=torch.int32, device=self.device)[:, None] * (hkv * mb)
                       + torch.arange(mb, dtype=torch.int32, device=self.device))
        return self

    def table(self) -> torch.Tensor:
        """Page table of the SPLA cache that these pages are the blocks of."""
        return self._table

    def _create(self, k, v, n_pages, hkv, P, d, page_stride, head_stride, n_q_heads, q_dtype, sm_scale, flags):
        self.lib = load()
        self.k_pages, self.v_pages, self.device = k, v, k.device
        self.page_size, self.n_q_heads, self.n_kv_heads, self.head_dim = P, n_q_heads, hkv, d
        self.q_torch_dtype = {"bf16": torch.bfloat16, "f32": torch.float32, None: k.dtype}[q_dtype]
        new = self._new_dtype
        self.status = torch.zeros(1, dtype=torch.int32, device=self.device)
        cfg = SplaPagedConfig(n_q_heads, hkv, d, P, n_pages, _TYPE_CODE[new or k.dtype], _TYPE_CODE[self.q_torch_dtype], page_stride, head_stride, sm_scale, flags)
        self.index = k.get_device()
        self.handle = C.c_void_p()
        create, scales = self.lib.spla_paged_create, ()
        if new is not None:
            create, scales = self.lib.spla_paged_create_scaled, (self.k_scales.data_ptr(), self.v_scales.data_ptr())
        _check(_on(self.index, lambda *a: create(*a[:-1]), C.byref(cfg), k.data_ptr(), v.data_ptr(), *scales, self.status.data_ptr(),
                   C.byref(self.handle)), create.__name__)

    def _batch(self, total, cu_new, seq_lens, page_table, max_new, max_len):
        """The packed spla_paged_batch_t."""
        shape, ts, n, dev, i32 = page_table.shape, page_table.stride(), seq_lens.shape[0], self.device, torch.int32
        if not (cu_new.dtype is i32 and seq_lens.dtype is i32 and page_table.dtype is i32 and cu_new.device == dev and seq_lens.device == dev
                and page_table.device == dev and cu_new.is_contiguous() and seq_lens.is_contiguous() and len(shape) == 2 and (ts[1] == 1 or shape[1] == 1)
                and cu_new.shape[0] == n + 1 and shape[0] == n):
            raise ValueError("paged cache: int32 cu_new [batch + 1], seq_lens [batch], page_table [batch, columns] on the cache's device")
        # (the table's columns bound max_len; its rows may be further apart)
        if max_len > shape[1] * self.page_size:
            raise ValueError("paged cache: max_len is more than the page table's columns hold")
        return _pack_batch(cu_new.data_ptr(), seq_lens.data_ptr(), page_table.data_ptr(), n, total, max_new, max_len, ts[0] if n > 1 else shape[1])

    def _rows(self, x, total, heads, dtype, what):
        """Elements between the tokens of x [total, heads, d]."""
        d, xs = self.head_dim, x.stride()
        if not (x.shape == (total, heads, d) and x.dtype is dtype and x.device == self.device and xs[2] == 1 and (xs[1] == d or heads == 1)):
            raise ValueError(f"paged cache: {what} [tokens, {heads}, {d}] of its type, heads contiguous")
        if total <= 1:
            return heads * d
        if xs[0] < heads * d:                                                # (0, an expanded tensor's, would mean "dense" to the library)
            raise ValueError(f"paged cache: {what} whose tokens are at least {heads * d} elements apart")
        return xs[0]

    def append(self, k: torch.Tensor, v: torch.Tensor, cu_new: torch.Tensor, seq_lens: torch.Tensor, page_table: torch.Tensor,
               q: torch.Tensor | None = None, rope: Rope | None = None, positions: torch.Tensor | None = None, q_out: torch.Tensor | None = None,
               q_weight: torch.Tensor | None = None, k_weight: torch.Tensor | None = None, eps: float = 1e-6):
        """Stores k, v [total, H_kv, d] at the last n_b positions of every sequence, keys rotated by `rope`; rotates q [total, H_q, d]
        beside them and returns it (None without q).  Tokens may be any stride apart that keeps them off each other (no expanded tensors);
        `q_out=q` works in place.  With `k_weight`, `q_weight` (fp32 [d]) keys and queries are normed head by head before (`Rope.norm_apply`)."""
        if self._of_spla:
            raise ValueError("paged cache: the pages of an SPLA cache are read only; append to the SPLA cache")
        total, hkv, kt = k.shape[0], self.n_kv_heads, self._new_dtype or self.k_pages.dtype
        ks = self._rows(k, total, hkv, kt, "k")
        vs = self._rows(v, total, hkv, kt, "v")
        qs = os_ = 0
        qp = op = None
        if q is not None:
            qs = self._rows(q, total, self.n_q_heads, self.q_torch_dtype, "q")
            if q_out is None:
                q_out = torch.empty_like(q, memory_format=torch.contiguous_format)
            os_ = self._rows(q_out, total, self.n_q_heads, self.q_torch_dtype, "q_out")
            qp, op = q.data_ptr(), q_out.data_ptr()
        if positions is not None and not (positions.dtype == torch.int32 and positions.is_contiguous() and positions.numel() == total
                                          and positions.device == self.device):
            raise ValueError("paged cache: positions int32 [total]")
        if total:
            # the store needs no bounds of its own: a sequence may be as long as the table has columns
            most = min(page_table.shape[1] * self.page_size, 1 << 24)
            b = self._batch(total, cu_new, seq_lens, page_table, min(total, most), most)
            norm = None
            if q_weight is not None or k_weight is not None:
                norm = _pack_norm(*(0 if w is None else _norm_weight(w, self.head_dim, self.device) for w in (q_weight, k_weight)), eps)
            rc = _on(self.index, self.lib.spla_paged_append_norm, self.handle, b, None if rope is None else rope.handle, _ptr(positions), norm,
                     k.data_ptr(), ks, v.data_ptr(), vs, qp, qs, op, os_)
            if rc != SPLA_OK:
                raise SplaError(rc, "spla_paged_append")
        return q_out

    def read(self, cu_new: torch.Tensor, seq_lens: torch.Tensor, page_table: torch.Tensor, total: int, dtype: torch.dtype | None = None,
             k_out: torch.Tensor | None = None, v_out: torch.Tensor | None = None):
        """The last n_b cached tokens of every sequence as rows k, v [total, H_kv, d], where `append` took them from: in `dtype` (bf16 or fp32;
        default: that of the queries).  Rows of no sequence are not written."""
        shape = (total, self.n_kv_heads, self.head_dim)
        if dtype is None:
            dtype = self.q_torch_dtype if k_out is None else k_out.dtype
        if dtype not in _TYPE_CODE:
            raise ValueError("paged cache: tokens are read as bf16 or fp32")
        rows = []
        for x in (k_out, v_out):
            if x is None:
                x = torch.empty(shape, dtype=dtype, device=self.device)
            elif not (x.shape == shape and x.dtype is dtype and x.device == self.device and x.is_contiguous()):
                raise ValueError("paged cache: contiguous k_out, v_out [total, H_kv, d] of one type")
            rows.append(x)
        if total:
            most = min(page_table.shape[1] * self.page_size, 1 << 24)
            b = self._batch(total, cu_new, seq_lens, page_table, min(total, most), most)
            rc = _on(self.index, self.lib.spla_paged_read, self.handle, b, rows[0].data_ptr(), rows[1].data_ptr(), _TYPE_CODE[dtype])
            if rc != SPLA_OK:
                raise SplaError(rc, "spla_paged_read")
        return rows[0], rows[1]

    def attend(self, q: torch.Tensor, cu_new: torch.Tensor, seq_lens: torch.Tensor, page_table: torch.Tensor, max_new: int, max_len: int,
               out: torch.Tensor | None = None, lse: torch.Tensor | None = None, softcap: float = 0.0, window: int = 0,
               slopes: torch.Tensor | None = None, first_key: torch.Tensor | None = None, prefix_lens: torch.Tensor | None = None, sinks: int = 0):
        """Attention of the new tokens' queries q [total, H_q, d] over the cache, which holds their keys already; max_new and max_len
        bound the new tokens and the length of any sequence.  Returns out [total, H_q, d] and lse fp32 [total, H_q].  See
        spla_paged_mask_t for the mask; `sinks` first tokens stay visible beside a window (`spla_paged_attend_sinks`)."""
        if sinks > 0x7fffffff:
            raise ValueError("paged cache: sinks is an int32")
        total, hq, dev = q.shape[0], self.n_q_heads, self.device
        qs = self._rows(q, total, hq, self.q_torch_dtype, "q")
        if out is None:
            out = torch.empty_like(q, memory_format=torch.contiguous_format)
        elif not (out.shape == q.shape and out.dtype == q.dtype and out.device == dev and out.is_contiguous()):
            raise ValueError("paged cache: a contiguous out like q")
        if lse is None:
            lse = torch.empty((total, hq), dtype=torch.float32, device=dev)
        elif not (lse.shape == (total, hq) and lse.dtype == torch.float32 and lse.device == dev and lse.is_contiguous()):
            raise ValueError("paged cache: lse fp32 [total, H_q]")
        if slopes is not None or first_key is not None or prefix_lens is not None:
            for x, n, t, what in ((slopes, hq, torch.float32, "slopes fp32 [H_q]"), (first_key, total, torch.int32, "first_key int32 [total]"),
                                  (prefix_lens, seq_lens.shape[0], torch.int32, "prefix_lens int32 [batch]")):
                if x is not None and not (x.dtype is t and x.numel() == n and x.is_contiguous() and x.device == dev):
                    raise ValueError(f"paged cache: {what}")
        if total:
            b = self._batch(total, cu_new, seq_lens, page_table, max_new, max_len)
            mask = _pack_mask(softcap, window, _ptr(slopes) or 0, _ptr(first_key) or 0, _ptr(prefix_lens) or 0)
            nbytes = C.c_size_t()
            # (what the call refuses it refuses below too, with its name)
            self.lib.spla_paged_query_workspace(self.handle, b, C.byref(nbytes))
            n = nbytes.value
            # a scratch of the call's own, from the stream's pool: calls on other streams and captured graphs share nothing
            ws = torch.empty(n, dtype=torch.uint8, device=dev) if n else None
            rc = _on(self.index, self.lib.spla_paged_attend_sinks, self.handle, b, q.data_ptr(), qs, mask, sinks, out.data_ptr(), lse.data_ptr(),
                     None if ws is None else ws.data_ptr(), n)
            if rc != SPLA_OK:
                raise SplaError(rc, "spla_paged_attend")
        return out, lse

    def sync_status(self) -> int:
        return _on(self.index, self.lib.spla_paged_sync_status, self.handle)

    def debug_wait_hook(self, max_wait_polls: int, extra_expected_bytes: int):
        """Test hook, as SplaCache.debug_wait_hook: waits of the tensor-core attention that run out."""
        _check(self.lib.spla_paged_debug_wait_hook(self.handle, max_wait_polls, extra_expected_bytes), "spla_paged_debug_wait_hook")

    def close(self):
        if getattr(self, "handle", None) is not None and self.handle.value:
            self.lib.spla_paged_destroy(self.handle)
            self.handle = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
