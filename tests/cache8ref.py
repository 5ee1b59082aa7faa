"""Plain forms of the 8-bit cache's calls on the CPU, written from their
definitions: e4m3 codes from a table of their values, scales, bounds, block
scores in exact rational arithmetic where it matters, pages page by page.

Codes, scales and bounds are compared bit for bit, given the rotated keys as
BF16 numbers: x / 2^e is exact and one rounding follows.  Attention is compared
with attnref's bounds over the values that the codes stand for: these are BF16
numbers exactly, so the bounds for a BF16 cache hold as they are."""
from __future__ import annotations

import math

import torch


def _values():
    """Value of each of the 256 codes: sign, 4 exponent bits (bias 7), 3 of mantissa."""
    out = []
    for c in range(256):
        s, e, m = c >> 7, c >> 3 & 15, c & 7
        v = math.nan if e == 15 and m == 7 else math.ldexp(m, -9) if e == 0 else math.ldexp(8 + m, e - 10)
        out.append(-v if s else v)
    return torch.tensor(out, dtype=torch.float64)


VALUES = _values()
_POSITIVE = VALUES[:127]
_MIDDLE = (_POSITIVE[1:] + _POSITIVE[:-1]) / 2


def to_codes(x):
    """x (float64) to the nearest code, ties to the even one; past 448 the largest, NaN 0x7F or 0xFF."""
    mag = x.abs().nan_to_num(0.0)
    up = torch.searchsorted(_MIDDLE, mag, right=True)    # middles count as above
    down = torch.searchsorted(_MIDDLE, mag, right=False)  # middles count as below
    c = torch.where(up == down, up, torch.where(up % 2 == 0, up, down))
    c = torch.where(torch.isnan(x), 0x7F, c)
    return (c + 128 * torch.signbit(x).long()).to(torch.uint8)


def same_codes(a, b):
    """Equal bytes; any NaN equals any NaN."""
    return (a == b) | (((a & 0x7F) == 0x7F) & ((b & 0x7F) == 0x7F))


def values(codes, scale):
    """codes [..., D], scale [...]: what they stand for, in 64 bits."""
    return VALUES[codes.long()] * scale.double().unsqueeze(-1)


def scale_of(m):
    """The smallest 2^e, e in [-100, 119], with m <= 448 2^e."""
    e = -100
    while e < 119 and m > math.ldexp(448.0, e):
        e += 1
    return math.ldexp(1.0, e)


def append(codes, scales, bounds, row_pages, page_size, block, start, x, keep=None):
    """Tokens x [n, H, D] (BF16) of a row become tokens start.. of its pages:
    codes [pages, H, ps, D], scales [pages, H, ps / block], bounds [pages, H, ps /
    block, 2, D] or None, all on the CPU and changed in place.  keep [n]: tokens
    that are stored (None: all)."""
    n, H, D = x.shape
    x = x.double()
    t = start
    while t < start + n:
        end = min(start + n, t // block * block + block)
        ids = [i for i in range(t, end) if keep is None or keep[i - start]]
        page, off = row_pages[t // page_size], t % page_size
        sub, begin = off // block, off // block * block
        if ids and 0 <= page < codes.shape[0]:
            for h in range(H):
                new = x[[i - start for i in ids], h]
                finite = new[torch.isfinite(new)].abs()
                s = scale_of(float(finite.max()) if finite.numel() else 0.0)
                if off > begin:
                    old = float(scales[page, h, sub])
                    if s > old:
                        held = codes[page, h, begin:off]
                        codes[page, h, begin:off] = to_codes(VALUES[held.long()] * old / s)
                    s = max(s, old)
                scales[page, h, sub] = s
                for i in ids:
                    codes[page, h, i % page_size] = to_codes(x[i - start, h] / s)
                if bounds is not None:
                    lo = new.nan_to_num(nan=math.inf, posinf=math.inf, neginf=-math.inf).amin(0)
                    hi = new.nan_to_num(nan=-math.inf, posinf=math.inf, neginf=-math.inf).amax(0)
                    if off > begin:
                        lo, hi = torch.fmin(lo, bounds[page, h, sub, 0].double()), torch.fmax(hi, bounds[page, h, sub, 1].double())
                    bounds[page, h, sub, 0], bounds[page, h, sub, 1] = lo.to(torch.bfloat16), hi.to(torch.bfloat16)
        t = end


def select(q, bounds, n0, budget, first, last):
    """q [R, D], bounds [n, 2, D] of a row's blocks n0.., a None in a list of
    bounds for a block without a page: the chosen blocks' numbers, then -1."""
    n = len(bounds)
    ids = list(range(n))
    if n > budget:
        score = []
        for x in bounds:
            s = -math.inf
            if x is not None:
                d = q.double()
                p = torch.where(d > 0, d * x[1].double(), torch.where(d < 0, d * x[0].double(), d)).flatten().tolist()
                s = math.fsum(p) if all(math.isfinite(v) for v in p) else sum(p)  # fsum: exact, rounded once
                s = -math.inf if math.isnan(s) else s
            score.append(s)
        middle = sorted(range(first, n - last), key=lambda i: (-score[i], i))[:budget - first - last]
        ids = sorted(list(range(first)) + middle + list(range(n - last, n)))
    return [n0 + i for i in ids] + [-1] * (budget - len(ids))


class Pool:
    """Rows and free pages, page by page."""

    def __init__(self, table, lens, free, n_free, page_size):
        self.table, self.lens, self.free, self.n, self.ps = [list(r) for r in table], list(lens), list(free), n_free, page_size

    def pages(self, n):
        return -(-n // self.ps)

    def resize(self, targets, room):
        """result, cu_new, slots, positions; room: entries of these (None: not asked for)."""
        most = (len(self.table[0]) if self.table else 0) * self.ps
        gained = [max(t - n, 0) for t, n in zip(targets, self.lens)]
        flags = 0
        good = [0 <= n <= most and 0 <= t <= most for n, t in zip(self.lens, targets)]
        if not all(good):
            flags |= 2
        gained = [g if ok else 0 for g, ok in zip(gained, good)]
        have = [self.pages(n) if ok else 0 for n, ok in zip(self.lens, good)]
        want = [self.pages(t) if ok else 0 for t, ok in zip(targets, good)]
        freed = sum(max(a - b, 0) for a, b in zip(have, want))
        left = self.n + freed - sum(max(b - a, 0) for a, b in zip(have, want))
        if left < 0:
            flags |= 1
        if sum(gained) > (2 ** 31 - 1 if room is None else room):
            flags |= 4
        if not 0 <= self.n <= len(self.free) or self.n + freed > len(self.free):
            flags |= 8
        result = [flags, max(-left, 0), min(sum(gained), 2 ** 31 - 1), self.n if flags else left]
        cu, slots, positions = [0] * (len(targets) + 1), [], []
        if not flags:
            for b, (a, z) in enumerate(zip(have, want)):
                for p in range(z, a):
                    self.free[self.n] = self.table[b][p]
                    self.table[b][p] = -1
                    self.n += 1
            for b, (a, z) in enumerate(zip(have, want)):
                for p in range(a, z):
                    self.n -= 1
                    self.table[b][p] = self.free[self.n]
            for b, t in enumerate(targets):
                if room is not None:
                    for i in range(self.lens[b], t):
                        slots.append(self.table[b][i // self.ps] * self.ps + i % self.ps)
                        positions.append(i)
                cu[b + 1] = cu[b] + gained[b]
            self.lens = list(targets)
        fill = [-1] * ((room or 0) - len(slots))
        return result, cu, slots + fill, positions + fill
