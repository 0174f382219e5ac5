"""Plain 64-bit implementations of the paged cache's operators, on the CPU, for its tests."""
import math

import torch

F8 = torch.float8_e4m3fn


def make_table(B, T, seed, spare=3):
    """A table [B, T] of distinct pages in random order, and the number of pages (some unused)."""
    g = torch.Generator().manual_seed(seed)
    n = B * T + spare
    return torch.randperm(n, generator=g)[:B * T].reshape(B, T).int(), n


def scale_for(amax):
    """The smallest power of two s >= 2^-100 with amax <= 448 s."""
    if amax == 0:
        return 2.0 ** -100
    e = math.ceil(math.log2(amax / 448))
    while 448 * 2.0 ** (e - 1) >= amax:
        e -= 1
    while 448 * 2.0 ** e < amax:
        e += 1
    return 2.0 ** max(e, -100)


def rotate(x, position, inv_freq, interleaved):
    """One token [H, D], in 64 bits."""
    x = x.double().clone()
    half = inv_freq.numel()
    for i in range(half):
        a = float(position) * float(inv_freq[i])
        p1, p2 = (2 * i, 2 * i + 1) if interleaved else (i, half + i)
        x1, x2 = x[:, p1].clone(), x[:, p2].clone()
        x[:, p1] = x1 * math.cos(a) - x2 * math.sin(a)
        x[:, p2] = x2 * math.cos(a) + x1 * math.sin(a)
    return x


class Pages:
    """A host copy of a cache's pages: keys and values both as [n, H, P, D]."""

    def __init__(self, k, v, k_scale=None, v_scale=None):
        self.raw = {"k": k.cpu().clone(), "v": v.cpu().transpose(2, 3).contiguous()}
        self.scale = {"k": k_scale, "v": v_scale}
        self.scale = {s: None if t is None else t.cpu().clone() for s, t in self.scale.items()}
        self.P = k.shape[2]

    def values(self, side):
        x = self.raw[side].double()
        s = self.scale[side]
        return x if s is None else x * s.double()[:, :, None, None]

    def of(self, side, table_row, length):
        """[H, length, D] of a sequence; positions on no page are NaN."""
        x = self.values(side)
        n, H, P, D = x.shape
        out = torch.full((H, length, D), math.nan, dtype=torch.float64)
        for p in range(length):
            pid = int(table_row[p // P])
            if 0 <= pid < n:
                out[:, p] = x[pid, :, p % P]
        return out


def requantised(raw, factor):
    """e4m3 elements times factor (64-bit), rounded anew."""
    return (raw.double() * factor).float().to(F8)


def append(pages, table, start, k, v, count, inv_freq, positions, interleaved):
    """Appends to `pages` (scales, and earlier values of a page whose scale grows); returns
    {side: [(page, place, values [H, D])]} of the new places, unrounded."""
    B, n = k.shape[:2]
    P, T = pages.P, table.shape[1]
    news = {"k": [], "v": []}
    for b in range(B):
        c = n if count is None else min(max(int(count[b]), 0), n)
        at = {}
        for i in range(c):
            p = int(start[b]) + i
            if p < 0 or p >= T * P or not 0 <= int(table[b, p // P]) < pages.raw["k"].shape[0]:
                continue
            place = int(positions[b, i]) if positions is not None else p
            x = rotate(k[b, i], place, inv_freq, interleaved) if inv_freq is not None else k[b, i].double()
            at.setdefault(p // P, []).append((p % P, {"k": x, "v": v[b, i].double()}))
        for j, tokens in at.items():
            pid = int(table[b, j])
            held = tokens[0][0]
            for side in ("k", "v"):
                s = pages.scale[side]
                if s is not None:
                    for h in range(s.shape[1]):
                        x = torch.stack([t[1][side][h] for t in tokens])
                        x = x[torch.isfinite(x)]
                        new = scale_for(float(x.abs().max()) if x.numel() else 0.0)
                        if held:
                            old = float(s[pid, h])
                            new = max(new, old)
                            if new != old:
                                pages.raw[side][pid, h, :held] = requantised(pages.raw[side][pid, h, :held], old / new)
                        s[pid, h] = new
                news[side] += [(pid, place, x[side]) for place, x in tokens]
    return news


def keep(pages, table, ctx, path):
    """Moves the paths' nodes; returns the touched pages' ids."""
    B, N = path.shape
    P, T = pages.P, table.shape[1]
    n = pages.raw["k"].shape[0]
    touched = set()
    for b in range(B):
        c = max(int(ctx[b]), 0)
        ids = []
        for x in path[b].tolist():
            if not 0 <= x < N:
                break
            ids.append(x)
        for side in ("k", "v"):
            raw, s = pages.raw[side], pages.scale[side]
            H = raw.shape[1]
            before, scales = raw.clone(), None if s is None else s.clone()
            for j in sorted({(c + i) // P for i in range(len(ids))}):
                if j >= T or not 0 <= int(table[b, j]) < n:
                    continue
                pid = int(table[b, j])
                moves = []
                for i, x in enumerate(ids):
                    f = c + x
                    if (c + i) // P == j and f // P < T and 0 <= int(table[b, f // P]) < n:
                        moves.append((i, x, int(table[b, f // P]), f % P))
                if all(i == x for i, x, _, _ in moves):
                    continue
                touched.add(pid)
                held = max(c - j * P, 0)
                for h in range(H):
                    if s is None:
                        for i, _, fp, fs in moves:
                            raw[pid, h, (c + i) % P] = before[fp, h, fs]
                        continue
                    new = max(float(scales[fp, h]) for _, _, fp, _ in moves)
                    if held:
                        new = max(new, float(scales[pid, h]))
                        raw[pid, h, :held] = requantised(before[pid, h, :held], float(scales[pid, h]) / new)
                    for i, _, fp, fs in moves:
                        raw[pid, h, (c + i) % P] = requantised(before[fp, h, fs], float(scales[fp, h]) / new)
                    s[pid, h] = new
    return touched


def hybrid_sees(ctx, q_start, n_q, K, room):
    """For each query, the number of leading keys it sees (0: no position of the input)."""
    lc = max(ctx, 0)
    end = min(lc + 2 * K + 3, room)
    out = []
    for i in range(n_q):
        p = q_start + i
        out.append(0 if p < 0 or p >= end else p + 1 if p < lc else end)
    return out


def ancestors(parent):
    """[N][N] booleans: node n's ancestors and itself."""
    N = len(parent)
    sees = torch.zeros(N, N, dtype=torch.bool)
    for n in range(N):
        if 0 <= parent[n] < n:
            sees[n] = sees[parent[n]]
        sees[n, n] = True
    return sees


def attention(q, keys, values, mask, scale):
    """q [n, Hq, D], keys and values [H, L, D], mask [n, L] -> softmax(q k^T scale) v and
    sum(w |v|), in 64 bits; positions on no page (NaN keys) are not attended."""
    n, Hq, D = q.shape
    H = keys.shape[0]
    out = torch.zeros(n, Hq, D, dtype=torch.float64)
    size = torch.zeros(n, Hq, D, dtype=torch.float64)
    for h in range(Hq):
        k, v = keys[h // (Hq // H)], values[h // (Hq // H)]
        real = ~torch.isnan(k).any(1)
        m = mask & real
        s = (q[:, h].double() @ torch.where(real[:, None], k, 0.0).T * scale).masked_fill(~m, -math.inf)
        some = m.any(1)
        w = torch.softmax(s[some], -1)
        v = torch.where(real[:, None], v, 0.0)
        out[some, h] = w @ v
        size[some, h] = w @ v.abs()
    return out, size
