"""The division of the paged attention's work among the CTAs, on the CPU: every key tile of every unit is walked by exactly one CTA, however
many tiles there are (the device functions as they are, see paged_division_host.cpp)."""
import ctypes as C
import os
import random
import shutil
import subprocess

import numpy as np
import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2601_22379_b200", "csrc")


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    cuda = os.path.join(os.path.dirname(os.path.dirname(shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc")), "include")
    so = str(tmp_path_factory.mktemp("division") / "division.so")
    subprocess.run(["g++", "-std=c++17", "-O2", "-w", "-shared", "-fPIC", "-I", cuda, "-I", CSRC, "-o", so, os.path.join(HERE, "paged_division_host.cpp")], check=True)
    return C.CDLL(so)


class Division:
    """A launch: its plan (as the host makes it for that many CTAs), its sequences, and what the device makes of them."""

    def __init__(self, lib, cu, lens, kernel="mma", G=4, hkv=2, few=False, ctas=148, window=0, prefix=None, first_key=None, total_new=None, max_new=None, max_len=None,
                 narrow=-1, by_unit=0, first=0):
        self.lib, self.cu, self.lens, self.hkv, self.G = lib, cu, lens, hkv, G
        R = (32 if few else 128) if kernel == "mma" else (4 if few else 64)
        self.ppos = R // G
        self.upos = self.ppos * (2 if kernel == "mma" and not few else 1)
        self.log_tk = 7 if kernel == "mma" else 6
        self.extra = (1 if few else 2) if kernel == "mma" else 0
        self.ctas, self.by_unit, self.window, self.prefix = ctas, by_unit, window, prefix
        B = len(lens) - first
        total_new = cu[-1] if total_new is None else total_new
        max_new = max(b - a for a, b in zip(cu, cu[1:])) if max_new is None else max_new
        arr = lambda x: None if x is None else (C.c_int * len(x))(*x)  # noqa: E731
        plan = arr([self.ppos, self.upos, self.log_tk, by_unit, ctas, 1 if by_unit or (kernel != "mma" and not few) else 2, self.extra, hkv, G, total_new, max_new,
                    max(lens) if max_len is None else max_len, window, narrow, first])
        out, pre, n = (C.c_longlong * 4)(), (C.c_longlong * (B + 1))(), (C.c_int * B)()
        self.keep = (arr(cu), arr(lens), arr(prefix), arr(first_key))              # (the walks read them)
        lib.division_fill(plan, B, *self.keep, out, pre, n)
        self.total, self.share, self.status, self.narrow = out
        self.pre, self.n = list(pre), list(n)

    def walk(self, cta, room=1 << 16):
        seg, cut = (C.c_longlong * (8 * room))(), (C.c_int * 4)()
        count = self.lib.division_walk(C.c_int(cta), room, seg, cut)
        assert count < room
        return [tuple(seg[8 * i:8 * i + 8]) for i in range(count)], tuple(cut)

    def spans(self, b):
        """Of sequence b: [units] first and last key tile that a unit may walk (without documents), in 64 bits."""
        n, L = self.n[b], self.lens[b]
        if n == 0:
            return np.zeros(0, np.int64), np.zeros(0, np.int64)
        u = np.arange(1 if n <= self.ppos else -(-n // self.upos), dtype=np.int64)
        p0, p1 = L - n + u * self.upos, L - n + np.minimum(n, (u + 1) * self.upos) - 1
        lo = np.maximum(0, p0 - self.window + 1) if self.window else np.zeros_like(u)
        hi = np.minimum(L, np.maximum(p1 + 1, self.prefix[b] if self.prefix else 0))
        return lo >> self.log_tk, (hi + (1 << self.log_tk) - 1) >> self.log_tk

    def counts(self, b):
        t0, t1 = self.spans(b)
        return np.ones_like(t0) if self.by_unit else t1 - t0 + self.extra

    def check_totals(self):
        want = [0]
        for b in range(len(self.lens)):
            want.append(want[-1] + int(self.counts(b).sum()) * self.hkv)
        assert self.pre == want and self.total == want[-1]
        assert self.share * self.ctas >= self.total

    def check_walk(self, cta):
        """The segments of one share, found again from the sums before."""
        segs, _ = self.walk(cta)
        at, end = cta * self.share, min((cta + 1) * self.share, self.total)
        want = []
        for b in range(len(self.lens)):
            per = self.counts(b)
            t0, t1 = self.spans(b)
            if not len(per) or self.pre[b + 1] <= at or self.pre[b] >= end:
                continue
            before = np.concatenate([[0], np.cumsum(per)])
            for h in range(self.hkv):
                base = self.pre[b] + h * int(before[-1])
                first = max(0, int(np.searchsorted(before, at - base, side="right")) - 1)
                for u in range(first, len(per)):
                    a = base + int(before[u])
                    if a >= end:
                        break
                    e = a + int(per[u])
                    if e <= at:
                        continue
                    if self.by_unit:
                        want.append((b, h, u, int(t0[u]), int(t1[u])))
                        continue
                    lo = int(t0[u]) + max(0, max(at, a) - a - self.extra)
                    hi = int(t0[u]) + max(0, min(end, e) - a - self.extra)
                    if lo < hi:
                        want.append((b, h, u, lo, hi))
        assert [s[:5] for s in segs] == want
        for b, h, u, x0, x1, head, tail, _ in segs:
            t0, t1 = self.spans(b)
            assert bool(head) == (x0 == t0[u]) and bool(tail) == (x1 == t1[u])


@pytest.mark.parametrize("narrow", [-1, 0], ids=["as-planned", "wide"])
@pytest.mark.parametrize("seed", range(20))
def test_small(lib, seed, narrow):
    """Every share of drawn batches."""
    r = random.Random(seed)
    few = r.random() < 0.4
    B = r.choice([1, 2, 7, 31, 33, 70])
    new = [r.choice([0, 1, r.randint(1, 3 if few else 700)]) for _ in range(B)]
    new[0] = new[0] or 1
    lens = [n + r.choice([0, r.randint(0, 100), r.randint(0, 5000)]) for n in new]
    cu = [int(x) for x in np.concatenate([[0], np.cumsum(new)])]
    d = Division(lib, cu, lens, kernel=r.choice(["mma", "general"]), G=r.choice([1, 3, 4]), hkv=r.choice([1, 2, 5]), few=few, ctas=r.choice([3, 37, 148]),
                 window=r.choice([0, 0, 300]), prefix=r.choice([None, [r.randint(0, 6000) for _ in range(B)]]), narrow=narrow, by_unit=int(r.random() < 0.2))
    d.check_totals()
    assert d.status == 0 and (narrow or not d.narrow)
    for cta in range(d.ctas):
        d.check_walk(cta)


@pytest.mark.parametrize("kernel,new,old,G,hkv", [("general", 40000, (1 << 24) - 40000, 16, 1), ("general", 40001, (1 << 24) - 50000, 16, 3), ("general", 1200000, 0, 16, 1),
                                                  ("mma", 300000, (1 << 24) - 300000, 16, 1), ("general", 300000, 1 << 20, 16, 3)])
def test_tiles_past_32_bits(lib, kernel, new, old, G, hkv):
    """One sequence whose tiles pass 2^31 in a single head, or in its heads together, with another before and behind it."""
    cu = [0, 70, 70 + new, 75 + new]
    d = Division(lib, cu, [100, new + old, 9], kernel=kernel, G=G, hkv=hkv, ctas=296)
    assert not d.narrow and int(d.counts(1).sum()) * hkv > (1 << 31)
    d.check_totals()
    for cta in (101, 295) if new > 1000000 else (0, 1, 101, 294, 295):
        d.check_walk(cta)


def _sound(cu, lens, total, max_new, max_len):
    """The sequences whose own numbers fit, and those that a call serves: no earlier prefix sum inside [0, total] is above their first row."""
    own, served, top = [], [], -1
    for b, L in enumerate(lens):
        r0, r1 = cu[b], cu[b + 1]
        own.append(0 <= r0 <= r1 <= total and r1 - r0 <= max_new and r1 - r0 <= L <= max_len)
        served.append(own[-1] and r0 >= top)
        if 0 <= r0 <= total:
            top = max(top, r0)
    return own, served


def _spoilt(r, B, kind):
    """Prefix sums with mistakes in them."""
    new = [r.choice([0, 1, 2, r.randint(0, 9)]) for _ in range(B)]
    cu = [0]
    for n in new:
        cu.append(cu[-1] + n)
    total = cu[-1] + r.choice([0, 3])
    if kind == "alternating":
        cu = [0 if i % 2 == 0 else total for i in range(B + 1)]
    elif kind == "one":
        cu[r.randrange(B + 1)] = r.randint(0, total)
    elif kind == "far":
        cu[r.randrange(B + 1)] = r.choice([-5, total + 1, 1 << 30, -(1 << 31)])
    elif kind == "several":
        for _ in range(r.randint(1, B)):
            cu[r.randrange(B + 1)] = r.choice([r.randint(0, total), r.randint(0, total), -1, total + 7])
    elif kind == "shuffled":
        r.shuffle(cu)
    return cu, max(total, 1)


@pytest.mark.parametrize("kind", ["sound", "one", "far", "several", "shuffled", "alternating"])
@pytest.mark.parametrize("seed", range(8))
def test_every_row_has_one_owner(lib, kind, seed):
    """Prefix sums that do not ascend: the sequences that are served own rows of their own, and the append finds the same ones."""
    r = random.Random(100 * seed + len(kind))
    B = r.choice([1, 3, 8, 31, 32, 33, 64, 97])
    cu, total = _spoilt(r, B, kind)
    max_new, max_len = r.choice([4, 12, total]), 500
    lens = [r.choice([0, 3, 20, 500, 500, 500, 501]) for _ in range(B)]
    own, want = _sound(cu, lens, total, max_new, max_len)
    launches = [(0, B)] if r.random() < 0.5 else [(0, B // 2), (B // 2, B)]
    got = []
    for first, end in launches:
        if first == end:
            continue
        d = Division(lib, cu[:end + 1], lens[:end], hkv=2, G=4, few=True, total_new=total, max_new=max_new, max_len=max_len, first=first)
        got += d.n
        assert d.pre[-1] == d.total and d.total >= 0
        assert (d.status != 0) == (not all(own[first:end]))
    if not all(want):
        assert not all(own)                                                   # (some sequence before reports it)
    assert [n > 0 for n in got] == [w and cu[b + 1] > cu[b] for b, w in enumerate(want)]
    rows = [None] * total
    for b, w in enumerate(want):
        if w:
            for row in range(cu[b], cu[b + 1]):
                assert rows[row] is None
                rows[row] = b
    d = Division(lib, cu, lens, few=True, total_new=total, max_new=max_new, max_len=max_len)
    out = (C.c_int * 4)()
    step = 8
    for base in range(0, total, 4 * step):
        for w in range(step):
            lib.division_owner(C.c_int(base + w), C.c_int(step), out)
            for k in range(4):
                row, b = base + w + k * step, out[k]
                if row < total:
                    there = b >= 0 and own[b] and cu[b] <= row < cu[b + 1]
                    assert (b if there else None) == rows[row]
