"""tboa_kv_cache_attention in 64 bits (torch on the host) and the bound of its error, row by row: nothing in a row's bound comes from tokens that the row does not see, or from other rows."""
import numpy as np
import torch

F64 = torch.float64


def attention(cache, starts, lens, pages, q, scale, window, dtype=torch.float32, many=False, rows_of_call=None):
    """Output (NaN for rows of no sequence and those that see a scale that is no number) and the bound of an output's error, per element.  With A the probabilities, x the scores and, of a token,
    X = scale sum |q| |k|; many: the kernel for many rows:
      scores          dh + 4 fp32 operations on terms that add up to X (and fp32 queries in two half terms, 2^-22 of them): (dh + 4 + [8 for fp32]) 2^-24 X, and 2 * 2^-24 |x - max x| for the
                      difference to the maximum, whose own error numerator and sum share; the exponential 2^-22.  Of every token, in the numerator and in the sum
      probabilities   times scale, in two halves 2^-22; in one 2^-11 (bf16 sequences of more than 32 rows; rows_of_call: of one sequence alone, the call's)
      sums            (n + 8) 2^-24, twice, n tokens
      next to nothing a half below 2^-14 is off by 2^-25 whatever it is.  The largest probability times scale of the row is at least 2^14 as half (2^-1 for many rows): 2^-39 (2^-24) of it for every
                      token, times at most 255 levels
      output          half a step of the type"""
    q = q.double().cpu()
    rows, hq, dh = q.shape
    rep, pt, st = hq // cache.heads, cache.pt, cache.st
    out, lim = torch.full((rows, hq, dh), float("nan"), dtype=F64), torch.zeros(rows, hq, dh, dtype=F64)
    for b in range(len(lens)):
        n, end = int(starts[b + 1] - starts[b]), min(int(lens[b]), pages.shape[1] * pt)
        if n == 0:
            continue
        halves = 2.0 ** (-11 if dtype == torch.bfloat16 and (rows_of_call or n * rep) > 32 else -22)
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
        count = seen.sum(1, keepdim=True).double()
        r = slice(int(starts[b]), int(starts[b]) + n)
        for h in range(hq):
            g = h // rep
            if end == 0:
                out[r, h] = 0
                continue
            x = scale * (q[r, h] @ key[:, g].T)
            none = ~seen.any(1, keepdim=True)
            a = torch.softmax(x.masked_fill(~seen, -torch.inf), 1).masked_fill(none, 0.0)
            a = torch.where(seen, a, 0.0)
            v, s = val[:, g].nan_to_num(), vg[:, g, 0].nan_to_num()
            lost = (seen & ~torch.isfinite(vg[:, g, 0])[None]).any(1, keepdim=True)
            o = a @ v
            out[r, h] = torch.where(lost, torch.nan, o)
            big = scale * (q[r, h].abs() @ key[:, g].nan_to_num().abs().T)
            apart = torch.where(a > 0, (x - x.masked_fill(~seen, -torch.inf).amax(1, keepdim=True)).abs(), 0.0)
            e = a * ((dh + 4 + 8 * (dtype == torch.float32)) * 2.0 ** -24 * big + 2 * 2.0 ** -24 * apart + 2.0 ** -22)
            e = torch.where(seen, e, 0.0)
            low = count * 255 * 2.0 ** (-24 if many else -39) * (a * s[None]).amax(1, keepdim=True)
            lim[r, h] = torch.finfo(dtype).eps / 2 * o.abs() + 1.01 * (e @ v.abs() + e.sum(1, keepdim=True) * o.abs() + (halves + 2 * (count + 8) * 2.0 ** -24) * (a @ v.abs()) + low) + 2.0 ** -133
    return out, lim


def check(got, cache, starts, lens, pages, q, scale, window, many=False, rows=None, telling=0.9, rows_of_call=None):
    """rows: a mask [rows, heads] of what is compared (all that belong to sequences).  `telling`: at least this share of the compared outputs is larger than the bound, so that zeros would fail."""
    want, lim = attention(cache, starts, lens, pages, q, scale, window, got.dtype, many, rows_of_call)
    g = got.double().cpu()
    use = torch.zeros(g.shape[:2], dtype=torch.bool)
    use[:int(starts[-1])] = True
    if rows is not None:
        use &= rows
    assert torch.equal(torch.isnan(g)[use], torch.isnan(want)[use])
    use &= ~torch.isnan(want).any(-1)
    err = (g - want).abs()
    worst = (err / lim.clamp(min=1e-300))[use].max().item() if use.any() else 0.0
    print("error over bound %.3f" % worst)
    assert (err <= lim)[use].all(), worst
    some = use & (want != 0).any(-1)
    assert not some.any() or (want.abs() > lim)[some].double().mean() >= telling
    return worst
