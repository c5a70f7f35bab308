"""Plain float64 forms of the rotary positions, the append to a paged cache and the attention over it, one sequence and head
at a time, with bounds of what a kernel's roundings may add."""
import math

import torch


def frequencies(rot, base=10000.0, scaling="none", factor=1.0, original_len=0.0, ramp=(1.0, 32.0)):
    if scaling == "base":
        base = base * factor ** (rot / (rot - 2))
    f = torch.tensor([base ** (-2.0 * i / rot) for i in range(rot // 2)], dtype=torch.float64)
    if scaling == "linear":
        f = f / factor
    if scaling == "ramp":
        w = ((original_len * f / (2 * math.pi) - ramp[0]) / (ramp[1] - ramp[0])).clamp(0, 1)
        f = w * f + (1 - w) * f / factor
    return f


def rotate(x, positions, rot, interleaved, f, amplitude=1.0, transpose=False):
    """x [..., tokens, heads, d], positions [..., tokens].  Returns y and a bound of its fp32 error before the last rounding:
    the angle is off by pi 2^-24 (its float) and the sine and cosine by 2 units in the last place, a product and a sum by one each."""
    x = x.double().cpu()
    a = positions.double().cpu()[..., None] * f
    c, s = amplitude * torch.cos(a)[..., None, :], amplitude * torch.sin(a)[..., None, :]
    if transpose:
        s = -s
    y, err = x.clone(), torch.zeros_like(x)
    i = torch.arange(rot // 2)
    ia, ib = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
    xa, xb = x[..., ia], x[..., ib]
    y[..., ia], y[..., ib] = xa * c - xb * s, xb * c + xa * s
    # positions up to 2^24 and more: the frequency itself is a double, a few 2^-53 relative
    far = float(positions.abs().max()) * 2.0 ** -51 if positions.numel() else 0.0
    e = amplitude * (xa.abs() + xb.abs()) * (math.pi * 2.0 ** -24 + 4 * 2.0 ** -24 + 3 * 2.0 ** -24 + far)
    err[..., ia], err[..., ib] = e, e
    return y, err


def rounded(y, err, dtype):
    """Bound of |kernel - y| after one rounding to dtype."""
    return err * (1 + 2.0 ** -6) + (y.abs() + err) * torch.finfo(dtype).eps / 2


def gather(pages, table_row, L, h):
    """Rows of KV head h of a sequence's first L tokens."""
    P = pages.shape[2]
    n = -(-L // P)
    return pages[table_row[:n].long(), h].reshape(-1, pages.shape[3])[:L]


def attend(q, k_pages, v_pages, cu, lens, table, sm_scale=None, softcap=0.0, window=0, slopes=None, first_key=None, prefix=None, tensor_cores=False,
           seqs=None):
    """All arguments on the CPU.  Returns out, lse and the bounds of their errors; rows of sequences not in `seqs` are left NaN.

    The bounds: a score is a dot product of d terms in fp32, off by (d + 8) 2^-24 of the sum of the terms' magnitudes; the cap adds
    2^-21 of itself (its argument, exponential, reciprocal and product), the distance 2^-23 of its term; each e^s is off by the score's error and 2^-20 (base change,
    exponential, sums of up to 2^15 terms in parts); on the tensor cores a probability is rounded to bf16, half a step, 2^-8."""
    total, hq, d = q.shape
    hkv = k_pages.shape[1]
    G = hq // hkv
    sc = sm_scale or 1.0 / math.sqrt(d)
    out = torch.full((total, hq, d), math.nan, dtype=torch.float64)
    lse = torch.full((total, hq), math.nan, dtype=torch.float64)
    out_b, lse_b = torch.zeros_like(out), torch.zeros_like(lse)
    for b in range(len(lens)) if seqs is None else seqs:
        r0, r1, L = int(cu[b]), int(cu[b + 1]), int(lens[b])
        n = r1 - r0
        if n == 0:
            continue
        pos = torch.arange(L - n, L)
        j = torch.arange(L)
        lo = torch.zeros(n, dtype=torch.long) if not window else (pos - window + 1).clamp(min=0)
        if first_key is not None:
            lo = torch.maximum(lo, first_key[r0:r1].long())
        hi = pos + 1
        if prefix is not None:
            hi = torch.maximum(hi, torch.full_like(hi, int(prefix[b]))).clamp(max=L)
        seen = (j >= lo[:, None]) & (j < hi[:, None])
        for h in range(hkv):
            k, v = gather(k_pages, table[b], L, h).double(), gather(v_pages, table[b], L, h).double()
            for m in range(h * G, h * G + G):
                x = q[r0:r1, m].double()
                s = sc * (x @ k.T)
                e = sc * (x.abs() @ k.abs().T) * (d + 8) * 2.0 ** -24
                if softcap:
                    s = softcap * torch.tanh(s / softcap)
                    e = e + softcap * 2.0 ** -21
                if slopes is not None:
                    far = slopes[m].double() * (pos[:, None] - j).abs()
                    s, e = s - far, e + far * 2.0 ** -23 + s.abs() * 2.0 ** -24
                s = torch.where(seen, s, -math.inf)
                e = torch.where(seen, e, torch.zeros_like(e))
                top = s.amax(-1, keepdim=True)
                top = torch.where(top == -math.inf, torch.zeros_like(top), top)
                p = torch.where(seen, torch.exp(s - top), torch.zeros_like(s))
                z = p.sum(-1, keepdim=True)
                w = p / torch.where(z == 0, torch.ones_like(z), z)
                ws = torch.where(seen[..., None], w[..., None] * v, torch.zeros(1, dtype=torch.float64)) if not torch.isfinite(v).all() else None
                o = w @ v if ws is None else ws.sum(1)
                e = e + 2.0 ** -20 + e * e
                mass = (w @ v.abs().nan_to_num(posinf=0.0))
                lse_e = (w * e).sum(-1)
                out[r0:r1, m] = o
                lse[r0:r1, m] = torch.where(z[:, 0] == 0, torch.full_like(top[:, 0], -math.inf), top[:, 0] + torch.log(z[:, 0]))
                rel = (2.0 ** -8 if tensor_cores else 0.0)
                out_b[r0:r1, m] = (w * e) @ v.abs().nan_to_num(posinf=0.0) + lse_e[:, None] * mass + rel * mass
                lse_b[r0:r1, m] = lse_e + 2.0 ** -22 * (1 + lse[r0:r1, m].abs().nan_to_num(posinf=0.0, neginf=0.0))
    return out, lse, out_b, lse_b


def check(got, want, bound, dtype=None, what=""):
    got, want = got.double().cpu(), want.double()
    left_out = torch.isnan(want)
    fine = torch.isfinite(want)
    assert torch.equal(got[~fine & ~left_out], want[~fine & ~left_out]), f"{what}: values that are not finite"
    lim = bound if dtype is None else rounded(want, bound, dtype)
    off = (got - want).abs()[fine]
    bad = ~(off <= lim[fine])
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off by more than their bound, worst {float((off / lim[fine])[bad].max()):.3g} times, {float(off[bad].max()):.3g}"
