"""Serving with a quantized key/value cache: the operators as cases whose time and results can be measured.

Kinds:

  rotate   norms of the query and key vectors of every head, with the rotation by position in the same pass
  append   new keys and values into a paged cache of 8-bit levels, the keys rotated on the way
  attend   attention of a ragged batch of query tokens over that cache

Cache.  One buffer [n_pages, page_bytes] of bytes; a page holds `pt` tokens of all heads: the levels of K [head][token][channel], those
of V [head][token / 16][channel][token % 16] (channels padded to dp), then the grids of K and of V, fp32 (scale, zero) per head and
block of `st` tokens.  A level c stands for scale * (c - zero).  Levels, scales and zeros are outputs of their own: the levels are
whole numbers, decided in 64 bits.

`own` false: the operators in elementary torch operations.  `own` true: the framework's calls.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
F64 = torch.float64
FLOOR = 2.0 ** -126          # the least scale
SLACK = 9.0 / 16.0           # a block's grid stays as it is for values at most this share of a step beyond its ends
_CONTEXT = []          # the framework's context, kept as a program keeps it


# ---------------------------------------------------------------------------------------------------- the cases
def _rotate(name, tokens, hq, hkv, dh, rot, adjacent=0, norm=1, bf16=1):
    return dict(name=name, kind="rotate", tokens=tokens, hq=hq, hkv=hkv, dh=dh, rot=rot, adjacent=adjacent, norm=norm, bf16=bf16)


def _append(name, seqs, new, grown, hkv, dh, rot, adjacent=0, pt=64, st=1, bf16=1):
    """`new`: most new tokens of a sequence (1: one each); `grown`: most tokens that a sequence has in the cache before."""
    return dict(name=name, kind="append", seqs=seqs, new=new, grown=grown, hkv=hkv, dh=dh, rot=rot, adjacent=adjacent, pt=pt, st=st, bf16=bf16)


def _attend(name, seqs, new, grown, hq, hkv, dh, window=0, pt=64, st=1, bf16=1):
    return dict(name=name, kind="attend", seqs=seqs, new=new, grown=grown, hq=hq, hkv=hkv, dh=dh, window=window, pt=pt, st=st, bf16=bf16)


def listed():
    return [
        # one decoding step of a small batch, 70B-shaped heads: a launch is all that a user waits for
        _rotate("rotate_step", 16, 64, 8, 128, 128),
        # a long prompt, or a batch of calibration sequences, with the same heads
        _rotate("rotate_prompt", 16384, 64, 8, 128, 128),
        # heads of an odd size, pairs side by side, half of the channels rotated, fp32
        _rotate("rotate_odd", 1003, 10, 5, 100, 52, adjacent=1, bf16=0),
        # one decoding step of 64 sequences: a token each, a grid per token
        _append("append_step", 64, 1, 4000, 8, 128, 128),
        # prompts of four sequences, 7B-shaped heads, a grid per 16 tokens
        _append("append_prompt", 4, 2048, 300, 32, 128, 128, st=16),
        # odd everything: pieces of sequences that begin and end inside blocks whose grids have to grow, fp32
        _append("append_odd", 7, 333, 500, 5, 100, 52, adjacent=1, st=64, bf16=0),
        # a single request early in its answer: latency counts
        _attend("attend_step", 1, 1, 500, 64, 8, 128),
        # one decoding step of 32 ragged requests, grouped heads: the cache is what is read
        _attend("attend_batch", 32, 1, 8000, 64, 8, 128),
        # one decoding step with a key head for every query head, a grid per 16 tokens
        _attend("attend_heads", 16, 1, 4000, 32, 32, 128, st=16),
        # one request with a long context
        _attend("attend_long", 1, 1, 131000, 64, 8, 128),
        # pieces of two prompts behind what the cache holds of them
        _attend("attend_prompt", 2, 2048, 4096, 64, 8, 128),
        # short ragged pieces over a window, heads of an odd size, fp32
        _attend("attend_odd", 5, 200, 700, 10, 5, 100, window=257, pt=16, st=16, bf16=0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    hq, hkv, dh = rng.choice([(4, 4, 64), (32, 32, 128), (40, 40, 128), (64, 8, 128), (10, 5, 100), (4, 2, 32), (12, 1, 64), (16, 2, 256)])
    rot, adjacent, bf16 = rng.choice([dh, dh, dh // 4 * 2]), rng.choice([0, 0, 1]), int(rng.random() < 0.75)
    pt = rng.choice([16, 64, 64, 128])
    st = rng.choice([s for s in (1, 1, 16, 64) if s <= pt])
    kind = rng.choice(["rotate", "append", "attend", "attend", "attend"])
    if kind == "rotate":
        return dict(_rotate("", _log(rng, 1, min(16384, 150_000_000 // ((hq + hkv) * dh * (2 - bf16)))), hq, hkv, dh, rot, adjacent, int(rng.random() < 0.7), bf16))
    if kind == "append":
        seqs = _log(rng, 1, 64)
        new = rng.choice([1, _log(rng, 1, max(1, min(4096, 30_000_000 // (seqs * hkv * dh * (2 - bf16)))))])
        return dict(_append("", seqs, new, _log(rng, 1, 4000), hkv, dh, rot, adjacent, pt, st, bf16))
    seqs = _log(rng, 1, 48)
    window = rng.choice([0, 0, 0, _log(rng, 1, 4096)])
    if rng.random() < 0.6:      # decoding, one token or a few
        grown = _log(rng, 16, max(17, min(131000, 250_000_000 // (seqs * hkv * dh))))
        return dict(_attend("", seqs, rng.choice([1, 1, 1, 2, 5]), grown, hq, hkv, dh, window, pt, st, bf16))
    seqs = min(seqs, 6)
    grown = _log(rng, 1, 4096)
    new = _log(rng, 2, max(3, min(2048, int(2048 * 2048 * 2 * 64 * 128 / (seqs * (grown + 2048) * hq * dh * (3 - 2 * bf16))))))
    return dict(_attend("", seqs, new, grown, hq, hkv, dh, window, pt, st, bf16))


def _ragged(n, least, most, phase):
    """n whole numbers from `least` to `most`, spread evenly and in no order; the largest is there."""
    x = [least + int((most - least + 1) * ((phase + 0.6180339887498949 * i) % 1.0)) for i in range(n)]
    x[n // 2] = most
    return x


def _lengths(c):
    """New tokens of every sequence, and its tokens in the cache with them."""
    new = _ragged(c["seqs"], min(1, c["new"]), c["new"], 0.13)
    old = _ragged(c["seqs"], c["grown"] // 8, c["grown"], 0.57)
    return new, [n + g for n, g in zip(new, old)]


def _pairs(c):
    """Tokens that the query tokens see, summed, and tokens that are read."""
    new, lens = _lengths(c)
    w, pairs, read = c["window"] or 1 << 60, 0, 0
    for n, length in zip(new, lens):
        p = np.arange(length - n, length)
        pairs += int(np.minimum(p + 1, w).sum())
        read += min(length, w + n - 1)
    return pairs, read


def work(c):
    size = 2 if c["bf16"] else 4
    if c["kind"] == "rotate":
        n = c["tokens"] * (c["hq"] + c["hkv"]) * c["dh"]
        return dict(bytes=2 * n * size + c["tokens"] * (4 * c["rot"] + 4), flops=n * (4 * c["norm"] + 3 * c["rot"] / c["dh"]))
    new, lens = _lengths(c)
    if c["kind"] == "append":
        n = sum(new) * c["hkv"] * c["dh"]
        blocks = sum(-(-length // c["st"]) - (length - k) // c["st"] for k, length in zip(new, lens))
        return dict(bytes=2 * n * size + 2 * n + 16 * blocks * c["hkv"] + 4 * sum(new) * c["rot"], flops=2 * n * 5 + n * 3)
    pairs, read = _pairs(c)
    q = sum(new) * c["hq"] * c["dh"]
    return dict(bytes=2 * q * size + 2 * c["hkv"] * (read * c["dh"] + 8 * read / c["st"]), flops=4 * pairs * c["hq"] * c["dh"])


# ---------------------------------------------------------------------------------------------------- inputs
def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(7919 * seed + 11)
    return g


def _table(length, rot):
    """cos, then sin, of position * 10000^(-2i/rot) in fp32."""
    inv = 10000.0 ** (-torch.arange(rot // 2, dtype=F64, device=DEV) * 2 / rot)
    a = torch.arange(length, dtype=F64, device=DEV)[:, None] * inv
    return torch.cat([a.cos(), a.sin()], 1).float()


def _activations(g, *shape, bf16):
    """Gaussian, with a few channels ten times as large, as keys have them."""
    x = torch.randn(*shape, generator=g, device=DEV)
    x[..., :: max(1, shape[-1] // 3)] *= 10
    return x.to(torch.bfloat16 if bf16 else torch.float32)


def _padded(dh):
    return next(p for p in (32, 64, 96, 128, 192, 256) if p >= dh)


def _views(data, c):
    """Levels of K and V and their grids in a cache's buffer."""
    h, pt, st, dp = c["hkv"], c["pt"], c["st"], _padded(c["dh"])
    levels, grids = h * pt * dp, h * (pt // st) * 8
    n = data.shape[0]
    return dict(k=data[:, :levels].view(n, h, pt, dp), v=data[:, levels:2 * levels].view(n, h, pt // 16, dp, 16),
                kg=data[:, 2 * levels:2 * levels + grids].view(torch.float32).view(n, h, pt // st, 2),
                vg=data[:, 2 * levels + grids:2 * levels + 2 * grids].view(torch.float32).view(n, h, pt // st, 2))


def _cache(c, g, n_pages):
    """A cache whose every page holds quantized Gaussian keys and values."""
    h, pt, st, dh, dp = c["hkv"], c["pt"], c["st"], c["dh"], _padded(c["dh"])
    page = 2 * h * pt * dp + 2 * h * (pt // st) * 8
    data = torch.zeros(n_pages, (page + 255) // 256 * 256, dtype=torch.uint8, device=DEV)
    views = _views(data, c)
    some = max(1, 32_000_000 // (h * pt * dh))
    for a in range(0, n_pages, some):
        b = min(n_pages, a + some)
        for kv in "kv":
            x = _activations(g, b - a, h, pt // st, st, dh, bf16=0)
            lo, hi = x.amin((-2, -1)).clamp(max=0), x.amax((-2, -1)).clamp(min=0)
            s = (hi - lo) / 255
            z = torch.round(-lo / s)
            q = (torch.round(x / s[..., None, None]) + z[..., None, None]).clamp(0, 255).to(torch.uint8).view(b - a, h, pt, dh)
            if kv == "k":
                views["k"][a:b, :, :, :dh] = q
            else:
                views["v"][a:b, :, :, :dh] = q.view(b - a, h, pt // 16, 16, dh).transpose(3, 4)
            views[kv + "g"][a:b] = torch.stack([s, z], -1)
    return data


def prepare(case, seed):
    c = case
    g = _generator(seed)
    if c["kind"] == "rotate":
        q = _activations(g, c["tokens"], c["hq"], c["dh"], bf16=c["bf16"])
        k = _activations(g, c["tokens"], c["hkv"], c["dh"], bf16=c["bf16"])
        w = [1 + 0.1 * torch.randn(c["dh"], generator=g, device=DEV) if c["norm"] else None for _ in "qk"]
        positions = torch.randint(0, 32768, (c["tokens"],), generator=g, device=DEV, dtype=torch.int32)
        return dict(c=c, q=q, k=k, wq=w[0], wk=w[1], table=_table(32768, c["rot"]), positions=positions)
    new, lens = _lengths(c)
    per = -(-max(lens) // c["pt"])
    n_pages = sum(-(-n // c["pt"]) for n in lens) + 3
    order = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32).cpu()
    pages = torch.zeros(c["seqs"], per, dtype=torch.int32)
    at = 0
    for b, n in enumerate(lens):
        k = -(-n // c["pt"])
        pages[b, :k] = order[at:at + k]
        at += k
    starts = torch.tensor([0] + list(np.cumsum(new)), dtype=torch.int32)
    s = dict(c=c, cache=_cache(c, g, n_pages), pages=pages.to(DEV), starts=starts.to(DEV), lens=torch.tensor(lens, dtype=torch.int32, device=DEV), most=max(new))
    if c["kind"] == "append":
        s.update(k=_activations(g, sum(new), c["hkv"], c["dh"], bf16=c["bf16"]), v=_activations(g, sum(new), c["hkv"], c["dh"], bf16=c["bf16"]),
                 table=_table(max(lens), c["rot"]))
    else:
        q = torch.randn(sum(new), c["hq"], c["dh"], generator=g, device=DEV)
        s["q"] = (q / 4).to(torch.bfloat16 if c["bf16"] else torch.float32)
    return s


# ---------------------------------------------------------------------------------------------------- the plain forms
def _rotated(x, row, rot, adjacent):
    """x [.., heads, dh] rotated by the table's rows [.., rot]."""
    cos, sin = row[..., None, : rot // 2], row[..., None, rot // 2:]
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if adjacent else (x[..., : rot // 2], x[..., rot // 2:rot])
    y = torch.stack([a * cos - b * sin, b * cos + a * sin], -1 if adjacent else -2).flatten(-2)
    return torch.cat([y, x[..., rot:]], -1)


def _normed(x, w):
    return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * w


def _plain_rotate(s):
    c, row = s["c"], s["table"][s["positions"].long()]
    out = []
    for x, w in ((s["q"], s["wq"]), (s["k"], s["wk"])):
        y = x.float() if w is None else _normed(x.float(), w)
        out.append(_rotated(y, row, c["rot"], c["adjacent"]).to(x.dtype))
    return out


def _tokens(s, n):
    """Sequence and position of every new token."""
    t = torch.arange(n, device=DEV)
    b = torch.searchsorted(s["starts"][1:].long(), t, right=True)
    return b, s["lens"].long()[b] - (s["starts"].long()[b + 1] - t)


def _plain_append(s):
    c, views = s["c"], _views(s["cache"], s["c"])
    h, pt, st, dh = c["hkv"], c["pt"], c["st"], c["dh"]
    b, pos = _tokens(s, s["k"].shape[0])
    page, off = s["pages"].long()[b, pos // pt], pos % pt
    key, at = torch.unique(page * (pt // st) + off // st, return_inverse=True)      # the blocks that get tokens
    kp, kb = key // (pt // st), key % (pt // st)
    first = torch.full((len(key),), st, device=DEV).scatter_reduce(0, at, off % st, "amin")      # tokens that a block had before
    slot = torch.arange(st, device=DEV)
    where = kb[:, None] * st + slot          # [blocks, st]: place in the page
    k64 = _rotated(s["k"].double(), s["table"][pos].double(), c["rot"], c["adjacent"])
    for x, kv in ((k64, "k"), (s["v"].double(), "v")):
        ends = [torch.zeros(len(key), h, dtype=F64, device=DEV).scatter_reduce(0, at[:, None].expand(-1, h), f, r) for f, r in ((x.amin(-1), "amin"), (x.amax(-1), "amax"))]
        lo, hi = ends
        grid = views[kv + "g"][kp, :, kb].double()          # [blocks, h, 2]
        had = (first > 0)[:, None]
        s0, z0 = grid[..., 0], grid[..., 1]
        lo0, hi0 = -z0 * s0, (255 - z0) * s0
        keep = had & (lo >= lo0 - SLACK * s0) & (hi <= hi0 + SLACK * s0)
        lo, hi = torch.where(had, torch.minimum(lo, lo0), lo), torch.where(had, torch.maximum(hi, hi0), hi)
        flat = lo == hi
        lo, hi = torch.where(flat, -1.0, lo), torch.where(flat, 1.0, hi)
        s1 = ((hi - lo) / 255).float().double().clamp(min=FLOOR)
        s1 = torch.where(keep, s0, s1)
        z1 = torch.where(keep, z0, torch.round(-lo / s1))
        if kv == "k":
            old = views["k"][kp[:, None], :, where]          # [blocks, st, h, dp]
        else:
            old = views["v"][kp[:, None], :, where // 16, :, where % 16]
        taken = (torch.round((old[..., :dh].double() - z0[:, None, :, None]) * s0[:, None, :, None] / s1[:, None, :, None]) + z1[:, None, :, None]).clamp(0, 255)
        over = (had & ~keep)[:, None, :, None] & (slot < first[:, None])[:, :, None, None]
        old[..., :dh] = torch.where(over, taken.to(torch.uint8), old[..., :dh])
        level = (torch.round(x / s1[at][..., None]) + z1[at][..., None]).clamp(0, 255).to(torch.uint8)
        old[at, off % st, :, :dh] = level
        if kv == "k":
            views["k"][kp[:, None], :, where] = old
        else:
            views["v"][kp[:, None], :, where // 16, :, where % 16] = old
        views[kv + "g"][kp, :, kb] = torch.stack([s1, z1], -1).float()
    return views


def _dense(s, kv):
    """Keys or values of every sequence in fp32, [seqs, heads, longest, dh]."""
    c, views = s["c"], _views(s["cache"], s["c"])
    x = views[kv][s["pages"].long()]          # [seqs, pages, h, ..]
    n, p, h = x.shape[:3]
    if kv == "v":
        x = x.transpose(-1, -2)
    x = x.reshape(n, p, h, c["pt"], -1)[..., : c["dh"]]
    grid = views[kv + "g"][s["pages"].long()].repeat_interleave(c["st"], 3)
    x = (x.float() - grid[..., 1:]) * grid[..., :1]
    return x.transpose(1, 2).reshape(n, h, p * c["pt"], c["dh"])


def _plain_attend(s):
    c, q = s["c"], s["q"]
    b, pos = _tokens(s, q.shape[0])
    h, rep, dh = c["hkv"], c["hq"] // c["hkv"], c["dh"]
    at = torch.arange(q.shape[0], device=DEV) - s["starts"].long()[b]
    rows = torch.zeros(c["seqs"], s["most"], c["hq"], dh, device=DEV)
    rows[b, at] = q.float()
    rows = rows.view(c["seqs"], s["most"], h, rep, dh).permute(0, 2, 1, 3, 4).reshape(c["seqs"], h, s["most"] * rep, dh)
    x = torch.matmul(rows, _dense(s, "k").transpose(-1, -2)) / math.sqrt(dh)
    t = torch.arange(x.shape[-1], device=DEV)
    place = torch.full((c["seqs"], s["most"]), -1, device=DEV)
    place[b, at] = pos
    place = place.repeat_interleave(rep, 1)[:, :, None]
    seen = t <= place
    if c["window"]:
        seen &= t > place - c["window"]
    x.masked_fill_(~seen[:, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    x = torch.exp_(x - torch.where(torch.isinf(top), 0.0, top))
    total = x.sum(-1, keepdim=True)
    o = torch.matmul(x, _dense(s, "v")) / torch.where(total == 0, 1.0, total)
    o = o.view(c["seqs"], h, s["most"], rep, dh).permute(0, 2, 1, 3, 4).reshape(c["seqs"], s["most"], c["hq"], dh)
    return o[b, at].to(q.dtype)


# ---------------------------------------------------------------------------------------------------- the framework's calls
def _own(s):
    c = s["c"]
    if not _CONTEXT:
        import paper_2602_04929_amd as tb
        _CONTEXT.extend([tb, tb.Context()])
    tb, ctx = _CONTEXT
    if c["kind"] == "rotate":
        rotation = tb.Rotation(s["table"], adjacent=bool(c["adjacent"]))
        return list(ctx.head_norm_rotate(s["q"], s["k"], s["wq"], s["wk"], eps=1e-6, rotation=rotation, positions=s["positions"]))
    cache = tb.KVCache(s["cache"], c["hkv"], c["dh"], page_tokens=c["pt"], scale_tokens=c["st"])
    batch = tb.KVBatch(s["starts"], s["lens"], s["pages"], max_new=s["most"])
    if c["kind"] == "append":
        ctx.kv_cache_append(cache, batch, s["k"], s["v"], rotation=tb.Rotation(s["table"], adjacent=bool(c["adjacent"])))
        return _views(s["cache"], c)
    return ctx.kv_cache_attention(cache, batch, s["q"], window=c["window"])


def run(state):
    if own:
        return _own(state)
    return {"rotate": _plain_rotate, "append": _plain_append, "attend": _plain_attend}[state["c"]["kind"]](state)


# ---------------------------------------------------------------------------------------------------- the definitions in 64 bits
def _exact_rotate(s):
    c = s["c"]
    row = s["table"].double()[s["positions"].long()]
    half = c["rot"] // 2
    out = []
    for x, w in ((s["q"].double(), s["wq"]), (s["k"].double(), s["wk"])):
        if w is not None:
            x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / c["dh"] + 1e-6) * w.double()
        y = x.clone()
        for i in range(half):
            a, b = (2 * i, 2 * i + 1) if c["adjacent"] else (i, i + half)
            cos, sin = row[:, i, None], row[:, half + i, None]
            y[..., a] = x[..., a] * cos - x[..., b] * sin
            y[..., b] = x[..., a] * sin + x[..., b] * cos
        out.append(y)
    return out


def _exact_append(s):
    """One sequence, one block of tokens at a time."""
    c = s["c"]
    h, pt, st, dh = c["hkv"], c["pt"], c["st"], c["dh"]
    views = {n: v.cpu().numpy().copy() for n, v in _views(s["cache"], c).items()}
    starts, lens, pages = (s[n].cpu().numpy() for n in ("starts", "lens", "pages"))
    cos, sin = (t.cpu().numpy().astype(np.float64) for t in s["table"].split(c["rot"] // 2, 1))
    k, v = (s[n].double().cpu().numpy() for n in "kv")
    for i in range(c["seqs"]):
        n = starts[i + 1] - starts[i]
        p0 = lens[i] - n
        for q0 in range(p0 // st * st, lens[i], st):
            a, e = max(q0, p0), min(q0 + st, lens[i])          # positions that this block gets
            rows = slice(starts[i] + a - p0, starts[i] + e - p0)
            page, o = pages[i, q0 // pt], q0 % pt
            key = k[rows].copy()
            even, odd = (slice(0, c["rot"], 2), slice(1, c["rot"], 2)) if c["adjacent"] else (slice(0, c["rot"] // 2), slice(c["rot"] // 2, c["rot"]))
            cs, sn = cos[a:e, None], sin[a:e, None]
            key[..., even], key[..., odd] = k[rows][..., even] * cs - k[rows][..., odd] * sn, k[rows][..., odd] * cs + k[rows][..., even] * sn
            for x, kv in ((key, "k"), (v[rows], "v")):
                lo, hi = np.minimum(x.min((0, 2)), 0), np.maximum(x.max((0, 2)), 0)
                grid = views[kv + "g"][page, :, o // st].astype(np.float64)
                scale, zero, kept = grid[:, 0], grid[:, 1], np.zeros(h, bool)
                if a > q0:
                    bottom, top = -zero * scale, (255 - zero) * scale
                    kept = (lo >= bottom - SLACK * scale) & (hi <= top + SLACK * scale)
                    lo, hi = np.minimum(lo, bottom), np.maximum(hi, top)
                lo, hi = np.where(lo == hi, -1.0, lo), np.where(lo == hi, 1.0, hi)
                fresh = np.maximum(((hi - lo) / 255).astype(np.float32).astype(np.float64), FLOOR)
                s1 = np.where(kept, scale, fresh)
                z1 = np.where(kept, zero, np.rint(-lo / s1))
                held = views[kv][page] if kv == "k" else views[kv][page].transpose(0, 1, 3, 2).reshape(h, pt, -1)
                held = held[:, o:o + st, :dh].astype(np.float64)
                moved = np.clip(np.rint((held - zero[:, None, None]) * scale[:, None, None] / s1[:, None, None]) + z1[:, None, None], 0, 255)
                held[:, :a - q0] = np.where(kept[:, None, None], held, moved)[:, :a - q0]
                held[:, a - q0:e - q0] = np.clip(np.rint(x.transpose(1, 0, 2) / s1[:, None, None]) + z1[:, None, None], 0, 255)
                for j in range(e - q0):
                    if kv == "k":
                        views["k"][page, :, o + j, :dh] = held[:, j]
                    else:
                        views["v"][page, :, (o + j) // 16, :dh, (o + j) % 16] = held[:, j]
                views[kv + "g"][page, :, o // st, 0], views[kv + "g"][page, :, o // st, 1] = s1, z1
    return views


def _exact_attend(s):
    """One sequence and head at a time."""
    c, views = s["c"], _views(s["cache"], s["c"])
    dh, rep = c["dh"], c["hq"] // c["hkv"]
    starts, lens = s["starts"].tolist(), s["lens"].tolist()
    out = torch.zeros(s["q"].shape, dtype=F64, device=DEV)
    for i, length in enumerate(lens):
        n, pages = starts[i + 1] - starts[i], s["pages"][i, : -(-length // c["pt"])].long()
        place = torch.arange(length - n, length, device=DEV)[:, None]
        t = torch.arange(length, device=DEV)[None]
        hidden = (t > place) | (t <= place - c["window"]) if c["window"] else t > place
        for g in range(c["hkv"]):
            grids = [views[kv + "g"][pages, g].double().reshape(-1, 2).repeat_interleave(c["st"], 0)[:length] for kv in "kv"]
            key = (views["k"][pages, g].reshape(-1, _padded(dh))[:length, :dh].double() - grids[0][:, 1:]) * grids[0][:, :1]
            val = (views["v"][pages, g].permute(0, 1, 3, 2).reshape(-1, _padded(dh))[:length, :dh].double() - grids[1][:, 1:]) * grids[1][:, :1]
            for r in range(g * rep, (g + 1) * rep):
                x = s["q"][starts[i]:starts[i + 1], r].double() @ key.T / math.sqrt(dh)
                out[starts[i]:starts[i + 1], r] = torch.softmax(x.masked_fill(hidden, -math.inf), 1) @ val
    return out


def exact(case, seed):
    if case["kind"] == "append":
        blocks = sum(-(-n // case["st"]) + 1 for n in _lengths(case)[0])
        if blocks * (1 + case["hkv"] * case["dh"] * case["st"] / 2e5) > 20000:
            return None
    s = prepare(case, seed)
    return {"rotate": _exact_rotate, "append": _exact_append, "attend": _exact_attend}[case["kind"]](s)
