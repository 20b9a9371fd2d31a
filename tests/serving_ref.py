"""Plain 64-bit forms of the serving operators (numpy on the host), one head vector, block of tokens or row at a time."""
import numpy as np


def norm_rotate(x, w, eps, table, positions, adjacent):
    """x [T, H, dh], w [dh] or None, table [P, rot] or None."""
    x = np.asarray(x, np.float64)
    if w is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * np.asarray(w, np.float64)
    if table is None or table.shape[1] == 0:
        return x
    rot = table.shape[1]
    y = x.copy()
    for t, p in enumerate(positions):
        row = np.asarray(table[p], np.float64) if 0 <= p < len(table) else np.full(rot, np.nan)
        for i in range(rot // 2):
            a, b = (2 * i, 2 * i + 1) if adjacent else (i, i + rot // 2)
            c, s = row[i], row[rot // 2 + i]
            y[t, :, a], y[t, :, b] = x[t, :, a] * c - x[t, :, b] * s, x[t, :, b] * c + x[t, :, a] * s
    return y


def padded(dh):
    return next(p for p in (32, 64, 96, 128, 192, 256) if p >= dh)


class Cache:
    """Views of a cache's bytes (a copy on the host): k [page, head, token, dp], v [page, head, token / 16, dp, 16], kg, vg [page, head, block, 2]."""

    def __init__(self, data, heads, dh, pt, st):
        self.data, self.heads, self.dh, self.pt, self.st = np.ascontiguousarray(data).copy(), heads, dh, pt, st
        n, dp = len(self.data), padded(dh)
        lev, gr = heads * pt * dp, heads * (pt // st) * 8
        assert self.data.shape[1] == -(-(2 * lev + 2 * gr) // 256) * 256
        self.k = np.lib.stride_tricks.as_strided(self.data, (n, heads, pt, dp), (self.data.strides[0], pt * dp, dp, 1))
        self.v = np.lib.stride_tricks.as_strided(self.data[:, lev:], (n, heads, pt // 16, dp, 16), (self.data.strides[0], pt * dp, 16 * dp, 16, 1))
        f = self.data.view(np.float32)
        self.kg, self.vg = (np.lib.stride_tricks.as_strided(f[:, at // 4:], (n, heads, pt // st, 2), (f.strides[0], pt // st * 8, 8, 4)) for at in (2 * lev, 2 * lev + gr))

    def grid(self, kv):
        return self.kg if kv == "k" else self.vg

    def levels(self, kv, page, off):
        """Writable view [heads, dh] of one token."""
        return self.k[page, :, off, :self.dh] if kv == "k" else self.v[page, :, off // 16, :self.dh, off % 16]

    def values(self, kv, page, off):
        g = self.grid(kv)[page, :, off // self.st].astype(np.float64)
        with np.errstate(invalid="ignore"):
            return g[:, :1] * (self.levels(kv, page, off).astype(np.float64) - g[:, 1:])


def append(cache, starts, lens, pages, k, v, n_rows):
    """k (rotated), v [rows, heads, dh] in 64 bits, into the host cache."""
    st, pt = cache.st, cache.pt
    for b in range(len(lens)):
        n = starts[b + 1] - starts[b]
        p0, end = max(lens[b] - n, 0), min(lens[b], pages.shape[1] * pt)
        row0 = starts[b] + n - lens[b]
        for q0 in range(p0 // st * st, end, st):
            page = pages[b, q0 // pt]
            if not 0 <= page < len(cache.data):
                continue
            a, e = max(q0, p0), min(q0 + st, end)
            if a >= e:
                continue
            for kv, x in (("k", k), ("v", v)):
                for h in range(cache.heads):
                    new = np.asarray(x[row0 + a:row0 + e, h], np.float64)
                    lo, hi = min(new.min(), 0.0), max(new.max(), 0.0)
                    g = cache.grid(kv)[page, h, q0 % pt // st]
                    s0, z0 = np.float64(g[0]), np.float64(g[1])
                    had, grown = a > q0, False
                    if not np.isfinite(new).all() or (had and not (np.isfinite(s0) and np.isfinite(z0))):
                        s1, z1 = np.nan, 0.0
                    else:
                        bottom, top = -z0 * s0, (255 - z0) * s0
                        if had and lo >= bottom - 0.5625 * s0 and hi <= top + 0.5625 * s0:
                            s1, z1 = s0, z0
                        else:
                            grown = had
                            if had:
                                lo, hi = min(lo, bottom), max(hi, top)
                            if lo == hi:
                                lo, hi = -1.0, 1.0
                            s1 = max(np.float64(np.float32((hi - lo) / 255)), 2.0 ** -126)
                            z1 = np.rint(-lo / s1)
                    for p in range(q0, e):
                        if p < a and not grown:
                            continue
                        lev = cache.levels(kv, page, p % pt)
                        if p < a:
                            lev[h] = np.clip(np.rint((lev[h].astype(np.float64) - z0) * s0 / s1) + z1, 0, 255)
                        else:
                            lev[h] = 0 if np.isnan(s1) else np.clip(np.rint(np.asarray(x[row0 + p, h], np.float64) / s1) + z1, 0, 255)
                    cache.grid(kv)[page, h, q0 % pt // st] = s1, z1


def attention(cache, starts, lens, pages, q, scale, window):
    """q [rows, Hq, dh] -> outputs in 64 bits (NaN rows of no sequence), the sums of A |v| and the largest scale sum |q| |k| of each row and head (for error bounds)."""
    q = np.asarray(q, np.float64)
    rep = q.shape[1] // cache.heads
    out = np.full(q.shape, np.nan)
    size = np.zeros(q.shape)
    most = np.zeros(q.shape[:2])
    for b in range(len(lens)):
        n, end = starts[b + 1] - starts[b], min(lens[b], pages.shape[1] * cache.pt)
        if n == 0:
            continue
        there = np.array([0 <= pages[b, p // cache.pt] < len(cache.data) for p in range(end)], bool)
        zero = np.zeros((cache.heads, cache.dh))
        key = np.array([cache.values("k", pages[b, p // cache.pt], p % cache.pt) if there[p] else zero for p in range(end)]).reshape(end, cache.heads, cache.dh)
        val = np.array([cache.values("v", pages[b, p // cache.pt], p % cache.pt) if there[p] else zero for p in range(end)]).reshape(end, cache.heads, cache.dh)
        for i in range(n):
            pos = lens[b] - n + i
            seen = np.arange(end) <= pos
            if window:
                seen &= np.arange(end) > pos - window
            seen = np.nonzero(seen & there)[0]
            for h in range(q.shape[1]):
                r = starts[b] + i
                if not len(seen):
                    out[r, h] = 0
                    continue
                kk, vv = key[seen, h // rep], val[seen, h // rep]
                x = scale * (kk @ q[r, h])
                with np.errstate(invalid="ignore"):
                    a = np.exp(x - x.max())
                a /= a.sum()
                out[r, h], size[r, h], most[r, h] = a @ vv, a @ np.abs(vv), scale * (np.abs(kk) @ np.abs(q[r, h])).max()
    return out, size, most
