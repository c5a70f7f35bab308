"""Rotary positions against the formula in float64: pairings, parts of a head, scalings, strides, in place, gradients."""
import itertools
import math

import pytest
import torch

from paper_2601_22379_b200 import binding
from tests import paged_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _rand(*shape, dtype, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return torch.randn(*shape, device=DEV, generator=g).to(dtype)


def _check(rope_args, positions, x, y, transpose=False):
    a = dict(rope_args)
    d = a.pop("head_dim")
    rot, inter, amp = a.pop("rot_dim", 0) or d, a.pop("interleaved", False), a.pop("amplitude", 1.0)
    want, err = ref.rotate(x, positions, rot, inter, ref.frequencies(rot, **a), amp, transpose)
    ref.check(y, want, err, x.dtype)
    assert torch.equal(y[..., rot:].cpu(), x[..., rot:].cpu())               # channels beyond the rotated part: copied


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,rot,heads,tokens", [(128, 0, (32, 8), 8), (128, 64, (5, 1), 1), (64, 16, (3, 3), 301), (64, 6, (4, 2), 33), (256, 0, (2, 1), 5),
                                                (8, 2, (7, 1), 70), (72, 0, (1, 1), 9), (128, 128, (1, 1), 4097), (96, 48, (12, 4), 77), (16, 16, (40, 8), 3),
                                                (128, 0, (1, 1), 20011), (64, 4, (4096, 4096), 3), (8, 2, (4096, 4095), 700)])
def test_rotation(dtype, interleaved, d, rot, heads, tokens):
    args = dict(head_dim=d, rot_dim=rot, interleaved=interleaved)
    pos = (torch.arange(tokens, dtype=torch.int32) * 131 % 100003).to(DEV)
    q, k = _rand(tokens, heads[0], d, dtype=TYPES[dtype], seed=1), _rand(tokens, heads[1], d, dtype=TYPES[dtype], seed=2)
    r = binding.Rope(**args)
    yq, yk = r.apply(pos, q, k)
    _check(args, pos, q, yq)
    _check(args, pos, k, yk)
    assert torch.equal(r.apply(pos, q), yq)                                   # alone, and the same bits again


@pytest.mark.parametrize("scaling", [dict(scaling="linear", factor=4.0), dict(scaling="base", factor=8.0), dict(scaling="ramp", factor=8.0, original_len=8192.0),
                                     dict(scaling="ramp", factor=32.0, original_len=4096.0, ramp=(1.0, 4.0), amplitude=1.25), dict(base=500000.0)])
@pytest.mark.parametrize("top", [0, 1, 131072, 2 ** 24, 2 ** 31 - 1])
def test_scalings_and_far_positions(scaling, top):
    args = dict(head_dim=128, **scaling)
    pos = torch.tensor([max(0, top - i) for i in range(7)], dtype=torch.int32, device=DEV)
    x = _rand(7, 3, 128, dtype=torch.float32)
    _check(args, pos, x, binding.Rope(**args).apply(pos, x))


def test_negative_positions_turn_back():
    pos = torch.tensor([-1, -70000, 5], dtype=torch.int32, device=DEV)
    x = _rand(3, 2, 64, dtype=torch.float32)
    _check(dict(head_dim=64), pos, x, binding.Rope(64).apply(pos, x))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("offset", [0, 1])
def test_strides(dtype, offset):
    """Queries inside a packed projection, keys head-major as the SPLA cache takes them; `offset` breaks the 16-byte alignment."""
    B, T, hq, hkv, d = 3, 21, 6, 2, 64
    t = TYPES[dtype]
    flat = _rand(B * T * (hq + 2 * hkv) * d + 8, dtype=t)
    qkv = flat[offset:offset + B * T * (hq + 2 * hkv) * d].view(B, T, hq + 2 * hkv, d)
    q = qkv[:, :, :hq]
    k = _rand(B, hkv, T, d, dtype=t, seed=5).transpose(1, 2)
    pos = torch.randint(0, 4000, (B, T), dtype=torch.int32, device=DEV)
    args = dict(head_dim=d, rot_dim=32)
    yq, yk = binding.Rope(**args).apply(pos, q, k)
    assert yk.stride() == k.stride()
    _check(args, pos, q, yq)
    _check(args, pos, k, yk)
    rest = qkv[:, :, hq:].clone()
    before = q.clone()
    binding.Rope(**args).apply(pos, q, q_out=q)                               # in place, between other heads
    assert torch.equal(q, yq) and torch.equal(qkv[:, :, hq:], rest)
    _check(args, pos, before, q)


@pytest.mark.parametrize("interleaved", [False, True])
def test_gradient(interleaved):
    """The transposed rotation: of the formula's gradient, and against differences."""
    args = dict(head_dim=64, rot_dim=48, interleaved=interleaved, scaling="ramp", factor=4.0, original_len=1000.0, amplitude=1.1)
    r = binding.Rope(**args)
    pos = torch.randint(0, 30000, (2, 17), dtype=torch.int32, device=DEV)
    x, g = _rand(2, 17, 3, 64, dtype=torch.float32), _rand(2, 17, 3, 64, dtype=torch.float32, seed=9)
    gx = r.apply(pos, g, transpose=True)
    _check(args, pos, g, gx, transpose=True)
    x64 = x.double().cpu().requires_grad_()
    f = ref.frequencies(48, scaling="ramp", factor=4.0, original_len=1000.0)
    y, _ = ref.rotate(x64.detach(), pos, 48, interleaved, f, 1.1)
    # the rotation is linear: <g, R dx> = <R^T g, dx> for any step dx
    dx = _rand(2, 17, 3, 64, dtype=torch.float32, seed=11)
    y2, _ = ref.rotate(x64.detach() + dx.double().cpu(), pos, 48, interleaved, f, 1.1)
    left, right = float((g.double().cpu() * (y2 - y)).sum()), float((gx.double().cpu() * dx.double().cpu()).sum())
    # each of the gradient's 6528 values is off by 1.1 x 2 x |g| x 10 x 2^-24 at most; their products' sum by as much in all
    assert abs(left - right) <= float((g.abs() * dx.abs()).sum()) * 2 * 1.1 * 2 * 12 * 2.0 ** -24


def test_other_stream_and_graph():
    r = binding.Rope(128)
    pos = torch.arange(64, dtype=torch.int32, device=DEV)
    q, k = _rand(64, 8, 128, dtype=torch.bfloat16), _rand(64, 2, 128, dtype=torch.bfloat16, seed=1)
    want = r.apply(pos, q, k)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = r.apply(pos, q, k)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = r.apply(pos, q, k)
    q2 = _rand(64, 8, 128, dtype=torch.bfloat16, seed=7)
    q.copy_(q2)
    pos.add_(1000)
    graph.replay()
    torch.cuda.synchronize()
    want = r.apply(pos, q, k)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_before_the_spla_cache():
    """Rotated queries and keys through a decode step: with every block selected the step is dense attention of them."""
    B, hq, hkv, d, T = 2, 4, 2, 64, 100
    cfg = binding.make_config(batch=B, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, block_size=32, top_k=8, max_context=128, kv_dtype="f32",
                              flags=binding.SPLA_NO_RLA)
    cache, r = binding.SplaCache(cfg, DEV), binding.Rope(d)
    k, v = _rand(B, hkv, T, d, dtype=torch.float32, seed=1), _rand(B, hkv, T, d, dtype=torch.float32, seed=2)
    q = _rand(B, 1, hq, d, dtype=torch.float32, seed=3)
    pos = torch.arange(T, dtype=torch.int32, device=DEV).expand(B, T).contiguous()
    rk = r.apply(pos, k.transpose(1, 2)).transpose(1, 2)
    assert rk.is_contiguous()
    cache.append_tokens(rk, v)
    out = cache.decode(r.apply(pos[:, -1:].contiguous(), q).view(B, hq, d), None)
    f = ref.frequencies(d)
    k64, _ = ref.rotate(k.transpose(1, 2), pos, d, False, f)
    q64, _ = ref.rotate(q, pos[:, -1:], d, False, f)
    kk = k64.transpose(1, 2).repeat_interleave(hq // hkv, 1)
    w = torch.softmax(torch.einsum("bhd,bhtd->bht", q64[:, 0], kk) / math.sqrt(d), -1)
    want = torch.einsum("bht,bhtd->bhd", w, v.double().cpu().repeat_interleave(hq // hkv, 1))
    # scores of magnitude up to about 10 whose 64 terms are off by some 2^-22 each way: 1e-5 of the values' magnitudes
    assert float((out.double().cpu() - want).abs().max()) < 1e-4
