"""Plain 64-bit implementations on the CPU of the latent cache's operators and of the pages under the
caches, written from their definitions in include/cospec.h."""
import math

import torch

ROT = 64
BF16_HALF_STEP = 2.0 ** -8
F32_HALF_STEP = 2.0 ** -24


def positions_of(row, P):
    """(page, slot) of every position of a table row."""
    return [(int(e), s) for e in row for s in range(P)]


class Latents:
    """A host copy of a latent cache, as values: c [n, P, dc], r [n, P, 64], scale [n, P] or None."""

    def __init__(self, cache):
        self.c = cache.c.detach().cpu().to(torch.float64) if cache.c.dtype == torch.bfloat16 else \
            cache.c.detach().cpu().float().to(torch.float64)
        self.r = cache.r.detach().cpu().double()
        self.scale = None if cache.scale is None else cache.scale.detach().cpu().double()
        self.page = cache.page

    def sequence(self, row):
        """Latents, keys and which positions there are, in order: [T P, dc], [T P, 64], [T P]."""
        n = self.c.shape[0]
        ids = row.long()
        there = ((ids >= 0) & (ids < n)).repeat_interleave(self.page)
        ids = ids.clamp(0, n - 1)
        c = self.c[ids]
        if self.scale is not None:
            c = c * self.scale[ids][..., None]
        return c.reshape(-1, c.shape[-1]), self.r[ids].reshape(-1, ROT), there


def hybrid_sees(ctx, q_start, K, n, room):
    """[n, room] truth values, from the rule."""
    lc = max(int(ctx), 0)
    end = min(lc + 2 * K + 3, room)
    lc = min(lc, end)
    sees = torch.zeros(n, room, dtype=torch.bool)
    for i in range(n):
        p = int(q_start) + i
        if 0 <= p < end:
            sees[i, :(p + 1 if p < lc else end)] = True
    return sees


def tree_sees(ctx, parent, room):
    N = len(parent)
    lc = max(int(ctx), 0)
    sees = torch.zeros(N, room, dtype=torch.bool)
    above = []
    for i, p in enumerate(parent.tolist()):
        above.append((set(above[p]) if 0 <= p < i else set()) | {i})
        if lc + i >= room:
            continue
        sees[i, :min(lc, room)] = True
        for j in above[i]:
            if lc + j < room:
                sees[i, lc + j] = True
    return sees


def attend(q, c, r, sees, scale):
    """q [n, Hq, dc + 64], keys' latents and rotated parts, sees [n, keys] -> out [n, Hq, dc] and how far a
    kernel's may be off: its own rounding, that of every weight to bf16, and 32-bit scores."""
    n, Hq, d = q.shape
    dc = c.shape[1]
    out = torch.zeros(n, Hq, dc, dtype=torch.float64)
    off = torch.zeros(n, Hq, dc, dtype=torch.float64)
    key = torch.cat((c, r), 1)
    for i in range(n):
        at = sees[i].nonzero()[:, 0]
        if len(at) == 0:
            continue
        k, v = key[at], c[at]
        s = q[i].double() @ k.t() * scale
        w = torch.softmax(s, -1)
        out[i] = w @ v
        # a sum of d products in 32 bits, in any order, and two more roundings of the score
        rough = (q[i].double().abs() @ k.abs().t()).amax(-1) * abs(scale)
        slack = (d + 2) * F32_HALF_STEP * rough * 2 + 1e-6
        # (sums of weights and products in 32 bits: far below, within the 1.1)
        off[i] = 1.1 * (BF16_HALF_STEP * out[i].abs() + (BF16_HALF_STEP + 2 * slack)[:, None] * (w @ v.abs())) + 1e-30
    return out, off


def rotated(x, positions, inv_freq, interleaved):
    """x [..., 64] at positions [...] (a pair of dimensions fewer), in 64 bits."""
    x = x.double().clone()
    half = len(inv_freq)
    a = positions.double()[..., None] * inv_freq.double()
    cos, sin = a.cos(), a.sin()
    i1 = torch.arange(half) * 2 if interleaved else torch.arange(half)
    i2 = i1 + 1 if interleaved else i1 + half
    x1, x2 = x[..., i1].clone(), x[..., i2].clone()
    while cos.dim() < x1.dim():
        cos, sin = cos.unsqueeze(-2), sin.unsqueeze(-2)
    x[..., i1], x[..., i2] = x1 * cos - x2 * sin, x2 * cos + x1 * sin
    return x


def normalised(c, weight, eps):
    c = c.double()
    if weight is None:
        return c
    return c / (c.square().mean(-1, keepdim=True) + eps).sqrt() * weight.double()


def power_for(row):
    """The smallest power of two s >= 2^-100 with |x| <= 448 s for the finite values of a row."""
    fin = row[torch.isfinite(row)].abs()
    top = float(fin.max()) if len(fin) else 0.0
    s = 2.0 ** -100
    if top > 0:
        m, e = math.frexp(top)                               # top = m 2^e, 448 = 0.875 * 2^9
        s = max(2.0 ** (e - 9 if m <= 0.875 else e - 8), s)
    return s


# ------------------------------------------------------------------ pages

class Pool:
    """Counts and tables as lists, by the rules."""

    def __init__(self, refs, page):
        self.refs, self.page = list(refs), page

    def _page(self, e):
        return 0 <= e < len(self.refs)

    def fork(self, table, row, length):
        out = []
        for src, n in zip(row, length):
            T = len(table[0])
            new = [-1] * T
            if 0 <= src < len(table):
                for j in range(min(T, -(-max(n, 0) // self.page))):
                    if self._page(table[src][j]):
                        new[j] = table[src][j]
                        self.refs[new[j]] += 1
            out.append(new)
        return out

    def reserve(self, table, start, count):
        """Changes table; returns copies and how many pages are lacking."""
        P, T = self.page, len(table[0]) if table else 0
        wanted, copies = [], [(-1, -1)] * len(table)
        for b, row in enumerate(table):
            lo, hi = max(start[b], 0), min(start[b] + count[b], T * P)
            if lo >= hi:
                continue
            for j in range(lo // P, (hi - 1) // P + 1):
                if not self._page(row[j]) or self.refs[row[j]] > 1:
                    wanted.append((b, j, j == lo // P and lo % P > 0))
        free = [p for p, n in enumerate(self.refs) if n == 0]
        if len(free) < len(wanted):
            return copies, len(wanted) - len(free)
        for (b, j, inside), page in zip(wanted, free):
            old = table[b][j]
            if self._page(old):
                self.refs[old] -= 1
                if inside:
                    copies[b] = (old, page)
            self.refs[page] = 1
            table[b][j] = page
        return copies, 0

    def release(self, table, keep):
        for row, n in zip(table, keep):
            for j in range(-(-max(n, 0) // self.page), len(row)):
                if self._page(row[j]):
                    self.refs[row[j]] -= 1
                row[j] = -1

    def compact(self, table):
        used = sum(n > 0 for n in self.refs)
        behind = [p for p, n in enumerate(self.refs) if n > 0 and p >= used]
        holes = [p for p, n in enumerate(self.refs) if n <= 0 and p < used]
        to = dict(zip(behind, holes))
        for old, new in to.items():
            self.refs[new], self.refs[old] = self.refs[old], 0
        for row in table:
            for j, e in enumerate(row):
                row[j] = to.get(e, e)
        return list(to.items())
