"""Plain forms of the 8-bit pages and of the attention over them, in float64 and bit for bit where the result is one of rounding alone."""
import math

import torch

from tests import paged_reference as ref

BLOCK = 16


def exponent(top):
    """Least e in [-40, 40] with top <= 448 2^e, of magnitudes in float64 (exact: 448 = 7/8 2^9)."""
    m, x = torch.frexp(top)
    e = (x - 9 + (m > 0.875)).clamp(-40, 40)
    return torch.where(top > 0, e, torch.full_like(e, -40)).long()


def finite_top(x, dims):
    return torch.where(torch.isfinite(x), x.abs(), torch.zeros((), dtype=x.dtype)).amax(dims)


def e4m3(x):
    """float64 / float32 -> the nearest e4m3, ties to even, beyond 448: 448, not finite: NaN."""
    x = torch.where(torch.isfinite(x), x.clamp(-448, 448), torch.full_like(x, math.nan))
    return x.float().to(torch.float8_e4m3fn)


def values(pages, scales):
    """What pages [n, h, P, d] and scale bytes [n, h, P / 16] stand for, float64."""
    e = (scales.view(torch.uint8).long() - 127).clamp(-40, 40)
    return pages.view(torch.float8_e4m3fn).double() * torch.pow(2.0, e.double()).repeat_interleave(BLOCK, 2)[..., None]


def store(pages, scales, x, new, old, table, P):
    """Appends rows x [total, h, d] (float64 values as they are quantised) to CPU pages and scale bytes, run by run, bit for bit."""
    at = 0
    for b, (n, o) in enumerate(zip(new, old)):
        here = o
        while here < o + n:
            end = min(o + n, (here // BLOCK + 1) * BLOCK)
            page, row, off = int(table[b, here // P]), here % P - here % BLOCK, here % BLOCK
            some = x[at:at + end - here]
            at += end - here
            here = end
            if not 0 <= page < pages.shape[0]:
                continue
            e = exponent(finite_top(some, (0, 2)))
            if off:
                was = (scales[page, :, row // BLOCK].long() - 127).clamp(-40, 40)
                e = torch.maximum(e, was)
                held = pages[page, :, row:row + off].view(torch.float8_e4m3fn).double()
                again = e4m3(held * torch.pow(2.0, (was - e).double())[:, None, None]).view(torch.uint8)
                pages[page, :, row:row + off] = torch.where((e > was)[:, None, None], again, pages[page, :, row:row + off])
            scales[page, :, row // BLOCK] = (e + 127).to(torch.uint8)
            q = e4m3(some * torch.pow(2.0, -e.double())[:, None])
            pages[page, :, row + off:row + off + some.shape[0]] = q.view(torch.uint8).transpose(0, 1)


def attend(q, k, v, cu, lens, table, kernel, exps, sm_scale=None, softcap=0.0, window=0, slopes=None, first_key=None, prefix=None, sinks=0, seqs=None):
    """k, v: float64 pages (values).  kernel(n): "general", "few", "few32", "chunk" or "wide", what serves a sequence of n new tokens.  exps: largest exponent of a block of V
    anywhere (for the weights that fp16 cannot hold).  Returns out, lse and bounds as paged_reference.attend, whose terms hold here too; besides:

    few: queries in fp16 below 2^15 of the row's largest channel are off by 2^-39 of it at most; chunk: what e4m3 and e5m2 leave is at most 2^-21 of it.
    Weights are rounded to fp16, half a step, 2^-11; those it cannot hold are off by 2^-25 of a scale where the largest is at least 2^14 (few) or 2^11 (chunk).
    few32: queries below 2^15 in two parts of fp16 are off by 2^-9 where the largest channel is 2^14 at least; weights in two parts by 2^-22 of themselves or 2^-25 of
    that scale, and the tensor core cuts off less than 2^-23 of a sum at each of the four additions of 16 tokens (of two parts each).
    wide: keys and values in bf16, which is exact; weights rounded to bf16, half a step, 2^-8.
    chunk, wide: the tensor core cuts off less than 2^-23 of a sum at each addition of 16 tokens, over 128 tiles at most."""
    total, hq, d = q.shape
    hkv = k.shape[1]
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
        how = kernel(n)
        pos, j = torch.arange(L - n, L), torch.arange(L)
        lo = torch.zeros(n, dtype=torch.long) if not window else (pos - window + 1).clamp(min=0)
        if first_key is not None:
            lo = torch.maximum(lo, first_key[r0:r1].long())
        hi = pos + 1
        if prefix is not None:
            hi = torch.maximum(hi, torch.full_like(hi, int(prefix[b]))).clamp(max=L)
        seen = ((j >= lo[:, None]) | (j < (sinks if window else 0))) & (j < hi[:, None])
        for h in range(hkv):
            kk, vv = ref.gather(k, table[b], L, h), ref.gather(v, table[b], L, h)
            va = vv.abs().nan_to_num(nan=0.0)
            for m in range(h * G, h * G + G):
                x = q[r0:r1, m].double()
                xa = torch.where(torch.isfinite(x), x.abs(), torch.zeros(()))   # (a score that is infinite, or the cap for it, is off by nothing)
                top_q = xa.amax(-1, keepdim=True)
                s = sc * (x @ kk.T)
                sums = sc * kk.abs().nan_to_num(nan=0.0).sum(-1)[None]
                e = sc * (xa @ kk.abs().nan_to_num(nan=0.0).T) * (d + 8) * 2.0 ** -24
                e = e + {"general": 0.0, "few": 2.0 ** -39, "few32": 2.0 ** -23, "chunk": 2.0 ** -21, "wide": 0.0}[how] * top_q * sums
                if softcap:
                    s = torch.where(torch.isnan(s), s, softcap * torch.tanh(s / softcap))
                    e = e + softcap * 2.0 ** -21
                if slopes is not None:
                    far = slopes[m].double() * (pos[:, None] - j).abs()
                    s, e = s - far, e + far * 2.0 ** -23 + s.abs() * 2.0 ** -24
                s = torch.where(seen, s, -math.inf)
                e = torch.where(seen, e, torch.zeros(()).double()).nan_to_num(nan=0.0)
                top = s.amax(-1, keepdim=True)
                top = torch.where(top == -math.inf, torch.zeros_like(top), top)
                p = torch.where(seen, torch.exp(s - top), torch.zeros_like(s))
                z = p.sum(-1, keepdim=True)
                w = p / torch.where(z == 0, torch.ones_like(z), z)
                o = w @ vv if torch.isfinite(vv).all() else torch.where(seen[..., None], w[..., None] * vv, torch.zeros(1, dtype=torch.float64)).sum(1)
                # beside the base change and the exponential (2^-20) the exponents of the scales are added to the score in base 2
                e = e + 2.0 ** -20 + 2.0 ** -23 * (s.abs().nan_to_num(posinf=0.0, neginf=0.0, nan=0.0) + 90) + e * e
                mass, lse_e = w @ va, (w * e).sum(-1)
                cut = min(L / 16 + 8, 1024) * 2.0 ** -23
                rel = {"general": 0.0, "few": 2.0 ** -11, "few32": 2.0 ** -22 + 2.0 ** -21, "chunk": 2.0 ** -11 + cut, "wide": 2.0 ** -8 + cut}[how]
                least = {"general": 0.0, "few": 2.0 ** -39, "few32": 2.0 ** -39, "chunk": 2.0 ** -36, "wide": 0.0}[how] * L * 448 * 2.0 ** exps * w.amax(-1, keepdim=True)
                out[r0:r1, m] = o
                lse[r0:r1, m] = torch.where(z[:, 0] == 0, torch.full_like(top[:, 0], -math.inf), top[:, 0] + torch.log(z[:, 0]))
                out_b[r0:r1, m] = (w * e) @ va + lse_e[:, None] * mass + rel * mass + least
                lse_b[r0:r1, m] = lse_e + 2.0 ** -22 * (1 + lse[r0:r1, m].abs().nan_to_num(posinf=0.0, neginf=0.0))
    return out, lse, out_b, lse_b


def check(got, want, bound, dtype=None, what="", none=False):
    """As paged_reference.check; with `none` every NaN that is wanted has to be there."""
    if none:
        assert torch.equal(torch.isnan(got.double().cpu()), torch.isnan(want)), f"{what}: NaN in other places"
    ref.check(got, want, bound, dtype, what)
