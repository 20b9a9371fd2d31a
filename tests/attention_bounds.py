"""tboa_kv_cache_attention in 64 bits (torch on the host) and the bound of its error, row by row: nothing in a row's bound comes from tokens that the row does not see, or from other rows."""
import numpy as np
import torch

F64 = torch.float64


def attention(cache, starts, lens, pages, q, scale, window):
    """Per row and head: output (NaN for rows of no sequence), sums of A |v| per channel, the largest scale sum |q| |k|, the largest A times scale of V, tokens seen."""
    q = q.double().cpu()
    rows, hq, dh = q.shape
    rep, pt, st = hq // cache.heads, cache.pt, cache.st
    out, size = torch.full((rows, hq, dh), float("nan"), dtype=F64), torch.zeros(rows, hq, dh, dtype=F64)
    most, top, count = (torch.zeros(rows, hq, dtype=F64) for _ in range(3))
    for b in range(len(lens)):
        n, end = int(starts[b + 1] - starts[b]), min(int(lens[b]), pages.shape[1] * pt)
        if n == 0:
            continue
        p = np.arange(end)
        page = np.asarray(pages[b])[p // pt]
        there = (page >= 0) & (page < len(cache.data))
        page = np.where(there, page, 0)
        kg, vg = (torch.tensor(np.where(there[:, None, None], g[page, :, p % pt // st], 0.0), dtype=F64) for g in (cache.kg, cache.vg))
        key = (torch.tensor(cache.k[page, :, p % pt, :dh], dtype=F64) - kg[..., 1:]) * kg[..., :1]
        val = (torch.tensor(cache.v[page, :, p % pt // 16, :dh, p % 16], dtype=F64) - vg[..., 1:]) * vg[..., :1]
        place = torch.arange(int(lens[b]) - n, int(lens[b]))[:, None]
        t = torch.arange(end)[None]
        seen = (t <= place) & torch.tensor(there)[None]
        if window:
            seen &= t > place - window
        r = slice(int(starts[b]), int(starts[b]) + n)
        for h in range(hq):
            g = h // rep
            x = (scale * (q[r, h] @ key[:, g].T)).masked_fill(~seen, -torch.inf)
            none = ~seen.any(1, keepdim=True)
            a = torch.softmax(x, 1).masked_fill(none, 0.0) if end else torch.zeros(n, 0, dtype=F64)
            a = torch.where(seen, a, 0.0)
            v = torch.where(torch.isfinite(val[:, g]), val[:, g], 0.0)
            lost = (seen & ~torch.isfinite(vg[:, g, 0])[None]).any(1, keepdim=True)      # sees a scale that is no number
            out[r, h] = torch.where(lost, torch.nan, a @ v)
            size[r, h] = a @ v.abs()
            if end:
                k = key[:, g].abs().nan_to_num()
                most[r, h] = (scale * (q[r, h].abs() @ k.T)).masked_fill(~seen, 0.0).amax(1)
                top[r, h] = (a * vg[:, g, 0].nan_to_num()[None]).amax(1)
            count[r, h] = seen.sum(1).double()[:]
    return out, size, most, top, count


def bound(want, size, most, top, count, dtype, dh, many):
    """Of an output's error, per element; X: `most`, n: tokens that the row sees.  many: the kernel for many rows.
      scores          dh + 4 fp32 operations on terms that add up to X at most, and fp32 queries in two half terms (2^-22 of them): e = (dh + 4 + [8 for fp32]) 2^-24 X
      probabilities   2 e + 2^-22 + 2 * 2^-24 X, in numerator and sum; held in two halves, 2^-22, or by the kernel for many rows in one, 2^-11
      sums            (n + 8) 2^-24, twice
      next to nothing a half below 2^-14 is off by 2^-25 whatever it is.  The largest probability times scale of the row is at least 2^14 as half (2^-1 for many rows): 2^-39 (2^-24) of it for every
                      token, times at most 255 levels
      output          half a step of the type"""
    n = count[..., None]
    e = (dh + 4 + 8 * (dtype == torch.float32)) * 2.0 ** -24 * most[..., None]
    rel = 2 * (2 * e + 2.0 ** -22 + 2 * 2.0 ** -24 * most[..., None]) + 2.0 ** (-11 if many else -22) + 2 * (n + 8) * 2.0 ** -24
    low = n * 255 * 2.0 ** (-24 if many else -39) * top[..., None]
    return torch.finfo(dtype).eps / 2 * want.abs() + 1.01 * (rel * size + low) + 2.0 ** -133


def check(got, cache, starts, lens, pages, q, scale, window, many=False, rows=None, telling=0.9):
    """rows: a mask [rows, heads] of what is compared (all that belong to sequences).  `telling`: at least this share of the compared outputs is larger than the bound, so that zeros would fail."""
    parts = attention(cache, starts, lens, pages, q, scale, window)
    want, top = parts[0], parts[3]
    lim = bound(*parts, got.dtype, cache.dh, many)
    g = got.double().cpu()
    use = torch.zeros(g.shape[:2], dtype=torch.bool)
    use[:int(starts[-1])] = True
    if rows is not None:
        use &= rows
    assert torch.equal(torch.isnan(g)[use], torch.isnan(want)[use])
    use &= ~torch.isnan(want).any(-1)
    err = (g - want).abs()
    worst = (err / lim)[use].max().item() if use.any() else 0.0
    print("error over bound %.3f" % worst)
    assert (err <= lim)[use].all(), worst
    some = use & (top > 0)
    assert not some.any() or (want.abs() > lim)[some].double().mean() >= telling
    return worst
