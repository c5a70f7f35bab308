"""Head norms with the rotation in the same pass, and their gradients, against the formulas in float64 and against differences."""
import pytest
import torch

from paper_2601_22379_b200 import binding
from tests import paged_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
U = 2.0 ** -24                                                                # a rounding of fp32


def rand(*shape, dtype=torch.float32, seed=0, size=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (size * torch.randn(*shape, device=DEV, generator=g)).to(dtype)


def pairs(rot, interleaved):
    i = torch.arange(rot // 2)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)


def turn(y, err, positions, rot, interleaved, f, amplitude, back=False):
    """paged_reference.rotate of values that are themselves off by `err`."""
    z, e = ref.rotate(y, positions, rot, interleaved, f, amplitude, back)
    ia, ib = pairs(rot, interleaved)
    both = amplitude * (err[..., ia] + err[..., ib])
    e[..., ia] += both
    e[..., ib] += both
    e[..., rot:] += err[..., rot:]
    return z, e


def root(x, eps):
    """1 / sqrt(mean x^2 + eps) and its relative error: half that of a sum of d squares, the root's 2 units, the product and sum before it."""
    return 1.0 / (x.pow(2).mean(-1, keepdim=True) + eps).sqrt(), (x.shape[-1] / 2 + 6) * U


def forward(x, w, eps, positions, rot, interleaved, f, amplitude):
    x, w = x.double().cpu(), w.double().cpu()
    r, rel = root(x, eps)
    n = x * r * w
    return turn(n, n.abs() * (rel + 2 * U), positions, rot, interleaved, f, amplitude)


def backward(dy, x, w, eps, positions, rot, interleaved, f, amplitude):
    """dx, dw and bounds of their errors before the last rounding."""
    dy, x, w = dy.double().cpu(), x.double().cpu(), w.double().cpu()
    d = x.shape[-1]
    u, eu = turn(dy, torch.zeros_like(dy), positions, rot, interleaved, f, amplitude, back=True)
    r, rel = root(x, eps)
    t = u * x * r
    dims = tuple(range(x.dim() - 1))
    n = x.numel() // d
    dw, dw_e = t.sum(dims), (eu * x.abs() * r + t.abs() * (rel + (n + 2) * U)).sum(dims)   # (n rows added, in whatever order)
    g = u * w
    mean = (g * x).mean(-1, keepdim=True)
    mean_e = ((eu * w.abs() + 3 * U * g.abs()) * x.abs() + d * U * (g * x).abs()).mean(-1, keepdim=True)
    back = x * r * r * mean
    dx = r * (g - back)
    dx_e = r * (eu * w.abs() + U * g.abs() + x.abs() * r * r * (mean_e + mean.abs() * (2 * rel + 4 * U)) + 2 * U * (g - back).abs()) + dx.abs() * (rel + U)
    return dx, dx_e, dw, dw_e


SHAPES = [(128, 0, (32, 8), 8), (128, 64, (5, 1), 1), (64, 16, (3, 3), 301), (64, 6, (4, 2), 33), (256, 0, (2, 1), 5), (8, 2, (7, 1), 70), (72, 0, (1, 1), 9),
          (128, 128, (1, 1), 4097), (96, 48, (12, 4), 77), (16, 16, (40, 8), 3), (80, 16, (3, 1), 50), (64, 4, (4096, 4096), 2), (128, 0, (16, 4), 700), (256, 32, (3, 2), 40)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,rot,heads,tokens", SHAPES)
def test_forward_and_gradients(dtype, interleaved, d, rot, heads, tokens):
    args = dict(rot_dim=rot, interleaved=interleaved, amplitude=1.2 if tokens == 33 else 1.0)
    r, t, eps = binding.Rope(d, **args), TYPES[dtype], 1e-5
    pos = (torch.arange(tokens, dtype=torch.int32) * 131 % 100003).to(DEV)
    q, k = rand(tokens, heads[0], d, dtype=t, seed=1, size=1.7), rand(tokens, heads[1], d, dtype=t, seed=2, size=0.3)
    gq, gk = rand(tokens, heads[0], d, dtype=t, seed=3), rand(tokens, heads[1], d, dtype=t, seed=4)
    wq, wk = 1 + 0.3 * rand(d, seed=5), 1 + 0.3 * rand(d, seed=6)
    a = (eps, pos, rot or d, interleaved, ref.frequencies(rot or d), args["amplitude"])
    yq, yk = r.norm_apply(pos, q, wq, k, wk, eps=eps)
    for y, x, w in ((yq, q, wq), (yk, k, wk)):
        want, err = forward(x, w, *a)
        ref.check(y, want, err, t, "y")
    assert torch.equal(r.norm_apply(pos, q, wq, eps=eps), yq)                 # alone, and the same bits again
    dq, dwq, dk, dwk = r.norm_backward(pos, gq, q, wq, gk, k, wk, eps=eps)
    for got, got_w, x, w, g in ((dq, dwq, q, wq, gq), (dk, dwk, k, wk, gk)):
        dx, dx_e, dw, dw_e = backward(g, x, w, *a)
        ref.check(got, dx, dx_e, t, "dx")
        ref.check(got_w, dw, dw_e, torch.float32, "dw")
    again = r.norm_backward(pos, gq, q, wq, gk, k, wk, eps=eps)
    assert all(torch.equal(x, y) for x, y in zip((dq, dwq, dk, dwk), again))
    alone, alone_w = r.norm_backward(pos, gq, q, wq, eps=eps)
    assert torch.equal(alone, dq)
    _, _, dw, dw_e = backward(gq, q, wq, *a)
    ref.check(alone_w, dw, dw_e, torch.float32, "dw alone")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("offset", [0, 1])
def test_strides(dtype, offset):
    """Inside a packed projection, head-major gradients, batches; `offset` breaks the 16-byte alignment; in place."""
    B, T, hq, hkv, d, eps, t = 3, 21, 6, 2, 64, 1e-6, TYPES[dtype]
    flat = rand(B * T * (hq + 2 * hkv) * d + 8, dtype=t)
    qkv = flat[offset:offset + B * T * (hq + 2 * hkv) * d].view(B, T, hq + 2 * hkv, d)
    q, k = qkv[:, :, :hq], qkv[:, :, hq:hq + hkv]
    gq, gk = rand(B, hq, T, d, dtype=t, seed=1).transpose(1, 2), rand(B, hkv, T, d, dtype=t, seed=2).transpose(1, 2)
    wq, wk = 1 + 0.3 * rand(d, seed=5), 1 + 0.3 * rand(d, seed=6)
    pos = torch.randint(0, 5000, (B, T), dtype=torch.int32, device=DEV)
    r = binding.Rope(d)
    a = (eps, pos, d, False, ref.frequencies(d), 1.0)
    yq, yk = r.norm_apply(pos, q, wq, k, wk, eps=eps)
    dq, dwq, dk, dwk = r.norm_backward(pos, gq, q, wq, gk, k, wk, eps=eps)
    for y, x, w, g, dx, dw in ((yq, q, wq, gq, dq, dwq), (yk, k, wk, gk, dk, dwk)):
        want, err = forward(x, w, *a)
        ref.check(y, want, err, t, "y")
        ex, ex_e, ew, ew_e = backward(g, x, w, *a)
        ref.check(dx, ex, ex_e, t, "dx")
        ref.check(dw, ew, ew_e, torch.float32, "dw")
    keep = qkv.clone()
    r.norm_apply(pos, q, wq, k, wk, eps=eps, q_out=q, k_out=k)                # in place: the values beside stay
    assert torch.equal(q, yq) and torch.equal(k, yk) and torch.equal(qkv[:, :, hq + hkv:], keep[:, :, hq + hkv:])
    ex, ex_e, _, _ = backward(gq, keep[:, :, :hq], wq, *a)
    g2 = gq.clone()
    dq2, _ = r.norm_backward(pos, g2, keep[:, :, :hq], wq, eps=eps, dq=g2)
    assert dq2 is g2
    x2 = keep[:, :, :hq].clone()
    r.norm_backward(pos, gq, x2, wq, eps=eps, dq=x2)                          # over x
    for dx in (g2, x2):
        ref.check(dx, ex, ex_e, t, "dx in place")


def test_gradients_of_expanded_inputs():
    """One token's queries for all of a batch (a stride of 0): a gradient for each use."""
    B, T, h, d = 4, 9, 3, 64
    q = rand(1, 1, h, d).expand(B, T, h, d)
    g, w, pos = rand(B, T, h, d, seed=1), 1 + 0.3 * rand(d, seed=2), torch.arange(B * T, dtype=torch.int32, device=DEV).view(B, T)
    dq, dw = binding.Rope(d).norm_backward(pos, g, q, w)
    dx, dx_e, dw_, dw_e = backward(g, q, w, 1e-6, pos, d, False, ref.frequencies(d), 1.0)
    ref.check(dq, dx, dx_e, torch.float32, "dx")
    ref.check(dw, dw_, dw_e, torch.float32, "dw")


def test_gradients_against_differences():
    """(L(x + h v) - L(x - h v)) / 2 h of the kernel's forward pass, L = sum y g: off by the errors of its outputs over h, and by what the same difference in
    float64 is off by."""
    T, h, d, eps, step = 5, 2, 32, 1e-3, 2.0 ** -5
    r, pos = binding.Rope(d, rot_dim=16, interleaved=True), torch.arange(T, dtype=torch.int32, device=DEV) * 7
    x, g, w = rand(T, h, d, seed=1), rand(T, h, d, seed=2), 1 + 0.3 * rand(d, seed=3)
    a = (eps, pos, 16, True, ref.frequencies(16), 1.0)
    dx, dw = r.norm_backward(pos, g, x, w, eps=eps)
    for what, v in (("x", rand(T, h, d, seed=4)), ("w", rand(d, seed=5))):
        ends, exact, off = [], [], 0.0
        for s in (step, -step):
            xs, ws = (x + s * v, w) if what == "x" else (x, w + s * v)
            y = r.norm_apply(pos, xs, ws, eps=eps)
            want, err = forward(xs, ws, *a)
            ends.append(float((y.double().cpu() * g.double().cpu()).sum()))
            exact.append(float((want * g.double().cpu()).sum()))
            off += float((ref.rounded(want, err, torch.float32) * g.double().cpu().abs()).sum())
        ex, ex_e, ew, ew_e = backward(g, x, w, *a)
        vv = v.double().cpu()
        mine = float(((dx if what == "x" else dw).double().cpu() * vv).sum())
        true, true_e = (float((ex * vv).sum()), float((ref.rounded(ex, ex_e, torch.float32) * vv.abs()).sum())) if what == "x" else (
            float((ew * vv).sum()), float((ref.rounded(ew, ew_e, torch.float32) * vv.abs()).sum()))
        # (x + h v is rounded too, by the same amount on either side's own: the float64 difference sees the same points)
        by_kernel, by_formula = (ends[0] - ends[1]) / (2 * step), (exact[0] - exact[1]) / (2 * step)
        assert abs(by_kernel - mine) <= off / (2 * step) + abs(by_formula - true) + true_e, (what, by_kernel, mine)
        assert abs(by_formula - true) < 0.05 * abs(true) + 0.05               # the difference says something


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_of_zeros_and_large_ones(dtype):
    """eps alone under the root; magnitudes whose squares fit; eps = 0."""
    d, t = 64, TYPES[dtype]
    x = torch.zeros(4, 1, d, device=DEV, dtype=t)
    x[1], x[2], x[3] = 1e-12, 1e15, 1.0
    w, pos, r = torch.full((d,), 2.0, device=DEV), torch.zeros(4, dtype=torch.int32, device=DEV), binding.Rope(d)
    for eps in (1e-6, 0.0):
        y = r.norm_apply(pos[1:], x[1:], w, eps=eps)
        want, err = forward(x[1:], w, eps, pos[1:], d, False, ref.frequencies(d), 1.0)
        ref.check(y, want, err + 2.0 ** -100, t)
    assert (r.norm_apply(pos, x, w, eps=1e-6)[0] == 0).all()
    g = torch.ones_like(x)
    dq, dw = r.norm_backward(pos[:1], g[:1], x[:1], w, eps=1e-6)
    assert float((dq.float() - 2000).abs().max()) <= 2000 * (torch.finfo(t).eps / 2 + 2.0 ** -20) and (dw == 0).all()


def test_graphs_and_streams():
    """Captured and replayed beside eager calls of the same tensors: each has a scratch of its own."""
    T, d, t = 500, 128, torch.bfloat16
    r, pos = binding.Rope(d), torch.arange(T, dtype=torch.int32, device=DEV)
    q, k, gq, gk = rand(T, 8, d, dtype=t), rand(T, 2, d, dtype=t, seed=1), rand(T, 8, d, dtype=t, seed=2), rand(T, 2, d, dtype=t, seed=3)
    wq, wk = 1 + 0.3 * rand(d, seed=5), 1 + 0.3 * rand(d, seed=6)
    want = r.norm_backward(pos, gq, q, wq, gk, k, wk)
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            res = (*r.norm_apply(pos, q, wq, k, wk), *r.norm_backward(pos, gq, q, wq, gk, k, wk))
        graphs.append((g, res))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        with torch.cuda.stream(side):
            graphs[0][0].replay()
            other = r.norm_backward(pos, gq, q, wq, gk, k, wk)
        graphs[1][0].replay()
    torch.cuda.synchronize()
    fwd = r.norm_apply(pos, q, wq, k, wk)
    for res in (graphs[0][1], graphs[1][1]):
        assert all(torch.equal(x, y) for x, y in zip(res, (*fwd, *want)))
    assert all(torch.equal(x, y) for x, y in zip(other, want))


def test_no_tokens():
    r, w = binding.Rope(64), torch.ones(64, device=DEV)
    x, pos = torch.zeros(0, 2, 64, device=DEV), torch.zeros(0, dtype=torch.int32, device=DEV)
    assert r.norm_apply(pos, x, w).shape == x.shape
    dx, dw = r.norm_backward(pos, x, x, w)
    assert dx.shape == x.shape and (dw == 0).all()
