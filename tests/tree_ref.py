"""Attention of drafted trees over a quantized cache in 64 bits (torch on the host), with the bound of its error row by row: nothing in a row's bound comes from tokens that it does not see."""
import numpy as np
import torch

F64 = torch.float64


def masks(parents, counts, words):
    """Rows of bits [tokens, 32 words] of trees: ancestors and the token itself."""
    rows, at = [], 0
    for n in counts:
        first = len(rows)
        for i in range(n):
            row = np.zeros(32 * words, bool)
            if parents[at + i] >= 0:
                row |= rows[first + parents[at + i]]
            row[i:i + 1] = True      # (a token behind the last word has no bit)
            rows.append(row)
        at += n
    return np.array(rows, bool).reshape(-1, 32 * words)


def as_words(bits):
    b = bits.reshape(len(bits), -1, 32).astype(np.uint64)
    return torch.from_numpy((b << np.arange(32, dtype=np.uint64)).sum(-1).astype(np.uint32).view(np.int32))


def attention(cache, starts, lens, pages, q, bits, scale, window, dtype):
    """Output (NaN for rows of no sequence and those that see a value's scale that is no number) and its bound.  With A the probabilities, x the scores and, of a token, X = scale sum |q| |k|:
      scores          dh + 4 fp32 operations on terms that add up to X (and fp32 queries in two half terms, 2^-22 of them): (dh + 4 + [8 for fp32]) 2^-24 X, and 2 * 2^-24 |x - max x| for the
                      difference to the maximum; the exponential 2^-22.  Of every token, in the numerator and in the sum
      probabilities   times scale, in two halves 2^-22; in one 2^-11 (bf16)
      sums            (n + 8) 2^-24, twice, n tokens
      next to nothing a half below 2^-14 is off by 2^-25 whatever it is; the largest probability times scale of the row is at least 2^14 as half (2^-1 for bf16
                      sequences, or a call for one sequence, of more than 64 rows, the kernel for many rows): 2^-39 (2^-24) of it for every token, times at most 255 levels
      output          half a step of the type"""
    q = q.double().cpu()
    rows, hq, dh = q.shape
    rep, pt, st = hq // cache.heads, cache.pt, cache.st
    out, lim = torch.full((rows, hq, dh), float("nan"), dtype=F64), torch.zeros(rows, hq, dh, dtype=F64)
    for b in range(len(lens)):
        n, length = int(starts[b + 1] - starts[b]), int(lens[b])
        end = min(length, pages.shape[1] * pt)
        if n == 0:
            continue
        halves = 2.0 ** (-11 if dtype == torch.bfloat16 else -22)
        r = slice(int(starts[b]), int(starts[b]) + n)
        if end <= 0:
            out[r] = 0
            continue
        p = np.arange(end)
        page = np.asarray(pages[b])[p // pt]
        there = (page >= 0) & (page < len(cache.data))
        page = np.where(there, page, 0)
        kg, vg = (torch.tensor(np.where(there[:, None, None], g[page, :, p % pt // st], 0.0), dtype=F64) for g in (cache.kg, cache.vg))
        key = (torch.tensor(cache.k[page, :, p % pt, :dh], dtype=F64) - kg[..., 1:]) * kg[..., :1]
        val = (torch.tensor(cache.v[page, :, p % pt // 16, :dh, p % 16], dtype=F64) - vg[..., 1:]) * vg[..., :1]
        seen, before = np.zeros((n, end), bool), length - n
        for i in range(n):
            if before + i < 0:
                continue
            mine = [j for j in range(min(n, bits.shape[1])) if bits[starts[b] + i, j]]
            low = max(before + len(mine) - window, 0) if window else 0
            seen[i, low:max(before, 0)] = True
            seen[i, [before + j for j in mine if 0 <= before + j < end]] = True
        seen = torch.tensor(seen & there)
        count = seen.sum(1, keepdim=True).double()
        none = ~seen.any(1, keepdim=True)
        for h in range(hq):
            g = h // rep
            x = scale * (q[r, h] @ key[:, g].T)
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
            low = count * 255 * 2.0 ** (-24 if dtype == torch.bfloat16 and (n * rep > 64 or (len(lens) == 1 and rows * rep > 64)) else -39) * (a * s[None]).amax(1, keepdim=True)
            lim[r, h] = torch.finfo(dtype).eps / 2 * o.abs() + 1.01 * (e @ v.abs() + e.sum(1, keepdim=True) * o.abs() + (halves + 2 * (count + 8) * 2.0 ** -24) * (a @ v.abs()) + low) + 2.0 ** -133
    return out, lim


def check(got, cache, starts, lens, pages, q, bits, scale, window=0, rows=None, telling=0.9):
    """rows: a mask [rows, heads] of what is compared.  `telling`: at least this share of the compared outputs is larger than the bound, so that zeros would fail."""
    want, lim = attention(cache, starts, lens, pages, q, bits, scale, window, got.dtype)
    g = got.double().cpu()
    use = torch.zeros(g.shape[:2], dtype=torch.bool)
    use[:int(starts[-1])] = True
    if rows is not None:
        use &= rows
    assert torch.equal(torch.isnan(g)[use], torch.isnan(want)[use])
    use &= ~torch.isnan(want).any(-1)
    err = (g - want).abs()
    worst = (err / lim.clamp(min=1e-300))[use].max().item() if use.any() else 0.0
    print("error over bound %.3f" % worst, flush=True)
    assert (err <= lim)[use].all(), worst
    some = use & (want != 0).any(-1)
    assert not some.any() or (want.abs() > lim)[some].double().mean() >= telling
    return want
