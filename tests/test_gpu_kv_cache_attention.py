"""tboa_kv_cache_attention against the 64-bit form on the cache's own values (GPU).

Bound of an output's error, with A the probabilities, a = sum A |v| and X the largest scale * sum |q| |k| of a row, per element:
  scores          dh + 4 fp32 operations on terms that add up to X at most (and fp32 queries in two half terms, 2^-22 of them): e = (dh + 4 + [8 for fp32]) 2^-24 X
  probabilities   2 e + 2^-22 (the exponential and the difference to the maximum, X again: 2 * 2^-24 X) in both numerator and sum, and their rounding: 2^-11 (bf16), 2^-22 (fp32)
  sums            (tokens + 8) 2^-24, twice
  output          half a step of the type
  next to nothing probability times scale is held as a half, TOP for a probability of 1 with a scale of ref, ref at most twice the largest scale s (TOP is 2^14, and 2^8 for bf16 rows
                  that are many): below 2^-14 a half is off by up to 2^-25 whatever it is, that is 2^-25 / TOP of 2 s, times at most 255 levels, for every token, over a sum
                  of the probabilities (the one that gives the maximum is 1) of at least 1: tokens * 255 * 2^-24 / TOP * s
"""
import numpy as np
import pytest
import torch

from tests import serving_ref as ref
from tests.test_gpu_kv_cache_append import i32, layout

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx(lib):
    c = lib.Context()
    yield c
    c.close()


def filled(lib, total, heads, dh, pt, st, seed):
    """A cache of any levels, scales around 1/50 and zeros around the middle."""
    rng = np.random.default_rng(seed)
    c = ref.Cache(rng.integers(0, 256, (total, lib.KVCache.page_bytes(heads, dh, pt, st)), dtype=np.uint8), heads, dh, pt, st)
    for g in (c.kg, c.vg):
        g[..., 0] = np.exp(rng.normal(-5, 0.7, g.shape[:-1]))
        g[..., 1] = rng.integers(100, 150, g.shape[:-1])
    return c


def poison(cache, lens, pages):
    """Everything beyond the sequences' ends, and the pages of none, with NaN grids and any levels."""
    used = np.zeros((len(cache.data), cache.pt), bool)
    for b, n in enumerate(lens):
        for p in range(min(n, pages.shape[1] * cache.pt)):
            if 0 <= pages[b, p // cache.pt] < len(used):
                used[pages[b, p // cache.pt], p % cache.pt] = True
    free = ~used.reshape(len(used), -1, cache.st).any(-1)
    for g in (cache.kg, cache.vg):
        g[np.broadcast_to(free[:, None], g.shape[:-1])] = np.nan


def check(got, cache, starts, lens, pages, q, scale, window, dtype):
    want, size, most = ref.attention(cache, starts, lens, pages, q.double().cpu().numpy(), scale, window)
    n, dh = max(max(lens), 1), cache.dh
    fp32 = dtype == torch.float32
    e = (dh + 4 + 8 * fp32) * 2.0 ** -24 * most[..., None]
    rel = 2 * (2 * e + 2.0 ** -22 + 2 * 2.0 ** -24 * most[..., None]) + (2.0 ** -22 if fp32 else 2.0 ** -11) + 2 * (n + 8) * 2.0 ** -24
    low = n * 255 * 2.0 ** (-38 if fp32 else -32) * np.nanmax(cache.vg[..., 0])
    bound = torch.finfo(dtype).eps / 2 * np.abs(want) + 1.01 * rel * size + low + 2.0 ** -133
    g = got.double().cpu().numpy()
    rows = starts[-1]
    assert np.array_equal(np.isnan(g[:rows]), np.isnan(want[:rows]))
    err = np.abs(g - want)[:rows]
    with np.errstate(invalid="ignore"):
        assert not np.any(err > bound[:rows]), np.nanmax(err / bound[:rows])
    return np.nanmax(err / bound[:rows]) if err.size else 0.0


def case(lib, heads, rep, dh, new, lens, pt, st, dtype, seed, spare_rows=0):
    starts = np.concatenate([[0], np.cumsum(new)]).astype(int)
    total, pages = layout(lens, pt, seed)
    cache = filled(lib, total, heads, dh, pt, st, seed)
    poison(cache, lens, pages)
    g = torch.Generator().manual_seed(seed)
    q = (torch.randn(starts[-1] + spare_rows, heads * rep, dh, generator=g) * torch.exp(torch.randn(starts[-1] + spare_rows, heads * rep, 1, generator=g))).to(dtype).cuda()
    return starts, pages, cache, lib.KVCache(torch.tensor(cache.data).cuda(), heads, dh, pt, st), q


SHAPES = [
    # heads, rep, dh, new tokens, lengths, window, page, scale tokens
    (1, 1, 128, [1], [1], 0, 64, 1),
    (2, 8, 128, [1], [500], 0, 64, 1),
    (2, 1, 64, [1, 1, 1], [1, 64, 65], 0, 64, 1),
    (1, 3, 100, [1, 0, 2, 5], [130, 40, 2, 200], 0, 16, 16),
    (2, 2, 32, [7, 1, 0, 30], [7, 300, 0, 95], 0, 32, 4),
    (1, 8, 96, [3], [333], 0, 128, 2),
    (1, 17, 64, [2, 1], [70, 1030], 0, 1024, 32),
    (1, 2, 256, [2, 33], [200, 70], 0, 64, 64),
    (1, 1, 192, [65], [257], 0, 16, 1),
    (2, 4, 128, [40, 1], [200, 777], 50, 64, 1),
    (1, 2, 33, [20, 3], [20, 200], 1, 16, 2),
    (1, 4, 80, [64, 64], [64, 500], 65, 64, 16),
    (1, 1, 1, [3], [40], 0, 16, 1),
    (1, 5, 128, [4, 3, 1], [2, 0, 1], 0, 16, 1),      # more new tokens than places: rows that see nothing
    (1, 2, 64, [300], [300], 0, 64, 1),
    (1, 1, 128, [129, 200], [700, 201], 0, 64, 16),
]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(str(x).replace(" ", "") for x in s))
def test_ragged_batches(ctx, lib, dtype, shape):
    heads, rep, dh, new, lens, window, pt, st = shape
    starts, pages, cache, dev, q = case(lib, heads, rep, dh, new, lens, pt, st, dtype, 11 * dh + len(new), spare_rows=3)
    out = torch.full_like(q, 7)
    for most in (0, max(new)):      # what the caller knows of the batch changes nothing but the kernel
        got = ctx.kv_cache_attention(dev, lib.KVBatch(i32(starts), i32(lens), i32(pages), max_new=most), q, window=window, out=out)
        torch.cuda.synchronize()
        r = check(got, cache, starts, lens, pages, q, 1 / np.sqrt(dh), window, dtype)
        print("error over bound %.3f" % r)
        assert (got[starts[-1]:] == 7).all()          # rows of no sequence


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_a_long_context_in_pieces(ctx, lib, dtype):
    """Tokens split over many workgroups, one and several rows, a scale of the caller's, and queries that make one token count nearly alone."""
    for new, length, gain in ((1, 20000, 1.0), (3, 9001, 30.0), (20, 5000, 3.0)):
        starts, pages, cache, dev, q = case(lib, 1, 2, 64, [new], [length], 64, 1, dtype, new)
        q = (q.float() * gain).to(dtype)
        got = ctx.kv_cache_attention(dev, lib.KVBatch(i32(starts), i32([length]), i32(pages)), q, scale=0.2)
        torch.cuda.synchronize()
        check(got, cache, starts, [length], pages, q, 0.2, 0, dtype)


@pytest.mark.parametrize("max_new", [0, 1])
def test_many_sequences(ctx, lib, max_new):
    rng = np.random.default_rng(4)
    new, old = rng.integers(0, 2, 150), rng.integers(0, 90, 150)
    new[64:128] = 0
    lens = (new + old).tolist()
    starts, pages, cache, dev, q = case(lib, 1, 2, 32, new, lens, 16, 1, torch.bfloat16, 9)
    got = ctx.kv_cache_attention(dev, lib.KVBatch(i32(starts), i32(lens), i32(pages), max_new=max_new), q)
    torch.cuda.synchronize()
    check(got, cache, starts, lens, pages, q, 1 / np.sqrt(32), 0, torch.bfloat16)


@pytest.mark.parametrize("new", [[1, 1, 1], [40, 33, 70]])
def test_pages_that_are_not_there(ctx, lib, new):
    """Pages outside the cache are invisible, the rest is not; places beyond the row of pages too; a shared page serves two sequences."""
    lens = [100, 90, 80]
    starts, pages, cache, dev, q = case(lib, 1, 2, 64, new, lens, 16, 1, torch.float32, 21)
    pages = pages[:, :5].copy()      # 80 places
    pages[0, 1], pages[1, 0], pages[2, :] = -1, len(cache.data), [-5, 1 << 30, -1, -1, -1]
    pages[1, 3] = pages[0, 3]
    cache.kg[pages[1, 3]], cache.vg[pages[1, 3]] = [0.01, 120], [0.02, 130]
    dev = lib.KVCache(torch.tensor(cache.data).cuda(), 1, 64, 16, 1)
    got = ctx.kv_cache_attention(dev, lib.KVBatch(i32(starts), i32(lens), i32(pages)), q)
    torch.cuda.synchronize()
    check(got, cache, starts, lens, pages, q, 1 / 8, 0, torch.float32)
    assert (got[starts[2]:] == 0).all()


@pytest.mark.parametrize("new", [1, 50])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_values_that_are_special(ctx, lib, dtype, new):
    """A NaN scale of K or V reaches the rows that see its token and no other; a NaN or infinite query its own row; scales far apart and queries of any size stay exact."""
    starts, pages, cache, dev, q = case(lib, 1, 2, 64, [new, new], [150, 150], 16, 1, dtype, 5)
    cache.kg[pages[0, 140 // 16], 0, 140 % 16, 0] = np.nan      # seen by rows at place 140 and later of the first sequence
    cache.vg[pages[1, 145 // 16], 0, 145 % 16, 0] = np.nan
    cache.vg[pages[1, 2], 0, :, 0] *= 1e-6
    cache.vg[pages[1, 1], 0, :, 0] *= 1e6
    q[-1, 1, 3] = float("inf")
    q[0] *= 1e-20
    if new > 1:
        q[3, 0, 0] = float("nan")
        q[5] *= 1e-3
    dev = lib.KVCache(torch.tensor(cache.data).cuda(), 1, 64, 16, 1)
    got = ctx.kv_cache_attention(dev, lib.KVBatch(i32(starts), i32([150, 150]), i32(pages)), q)
    torch.cuda.synchronize()
    q = q.clone()
    g, ok = got.float(), torch.ones(len(q), 2, dtype=torch.bool)
    ok[-1, 1] = False
    assert torch.isnan(g[-1, 1]).all()
    if new > 1:
        ok[3, 0] = False
        assert torch.isnan(g[3, 0]).all()
    q[~ok.cuda()] = 0
    got[~ok.cuda()] = 0
    want, _, _ = ref.attention(cache, starts, [150, 150], pages, q.double().cpu().numpy(), 1 / 8, 0)
    bad = np.isnan(want).any(-1)
    assert np.array_equal(np.isnan(got.float().cpu().numpy()).any(-1)[ok.numpy()], bad[ok.numpy()])
    q[torch.tensor(bad).cuda()] = 0
    # the rows that see no NaN, against the form with the NaN tokens' scales taken as 1 (they do not count for these rows)
    cache.kg[...] = np.nan_to_num(cache.kg, nan=1.0)
    cache.vg[...] = np.nan_to_num(cache.vg, nan=1.0)
    want, size, most = ref.attention(cache, starts, [150, 150], pages, q.double().cpu().numpy(), 1 / 8, 0)
    use = ok.numpy() & ~bad
    fp32 = dtype == torch.float32
    e = (64 + 12) * 2.0 ** -24 * most[..., None]
    rel = 2 * (2 * e + 2.0 ** -22 + 2 * 2.0 ** -24 * most[..., None]) + (2.0 ** -22 if fp32 else 2.0 ** -11) + 2 * 158 * 2.0 ** -24
    low = 150 * 255 * 2.0 ** (-38 if fp32 else -32) * np.nanmax(cache.vg[..., 0])
    err = np.abs(got.double().cpu().numpy() - want)
    assert np.all((err <= torch.finfo(dtype).eps / 2 * np.abs(want) + 1.01 * rel * size + low)[use])


def test_strides_streams_and_offsets(ctx, lib):
    """Queries inside a fused projection, outputs inside a wider tensor, a context on a stream of its own, and pages beyond 2^32 bytes."""
    heads, rep, dh, pt, st = 8, 2, 128, 64, 1
    new, lens = [1, 2, 20], [70, 300, 150]
    starts, pages, cache, dev, q = case(lib, heads, rep, dh, new, lens, pt, st, torch.bfloat16, 31)
    base = ctx.kv_cache_attention(dev, lib.KVBatch(i32(starts), i32(lens), i32(pages)), q)
    wide = torch.randn(23, heads * (rep + 2) + 1, dh, device="cuda").bfloat16()
    wide[:, 1:1 + heads * rep] = q
    out = torch.zeros(23, heads * rep + 5, dh, device="cuda", dtype=torch.bfloat16)
    ctx.kv_cache_attention(dev, lib.KVBatch(i32(starts), i32(lens), i32(pages)), wide[:, 1:1 + heads * rep], out=out[:, 2:2 + heads * rep])
    torch.cuda.synchronize()
    assert torch.equal(out[:, 2:2 + heads * rep], base) and (out[:, :2] == 0).all() and (out[:, 2 + heads * rep:] == 0).all()
    # the same pages at the far end of a large cache
    per = dev.data.shape[1]
    far = (1 << 32) // per + 50
    big = torch.zeros(far + len(cache.data), per, dtype=torch.uint8, device="cuda")
    big[far:] = dev.data
    side = torch.cuda.Stream()
    other = lib.Context(stream=side)
    try:
        moved = lib.KVBatch(i32(starts), i32(lens), i32(pages + far))
        side.wait_stream(torch.cuda.current_stream())
        got = other.kv_cache_attention(lib.KVCache(big, heads, dh, pt, st), moved, q)
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        assert torch.equal(got, base)
        k, v = torch.randn(23, heads, dh, device="cuda").bfloat16(), torch.randn(23, heads, dh, device="cuda").bfloat16()
        ctx.kv_cache_append(dev, lib.KVBatch(i32(starts), i32(lens), i32(pages)), k, v)
        ctx.kv_cache_append(lib.KVCache(big, heads, dh, pt, st), moved, k, v)
        torch.cuda.synchronize()
        assert torch.equal(big[far:], dev.data) and not big[:far].any()
    finally:
        other.close()


def test_refusals(ctx, lib):
    starts, pages, cache, dev, q = case(lib, 2, 2, 64, [1], [10], 16, 1, torch.bfloat16, 3)
    batch = lib.KVBatch(i32(starts), i32([10]), i32(pages))
    for bad in (dict(window=-1), dict(scale=-1.0), dict(scale=float("nan"))):
        with pytest.raises(lib.TurboBoAError) as e:
            ctx.kv_cache_attention(dev, batch, q, **bad)
        assert e.value.code == -1
    with pytest.raises(lib.TurboBoAError):
        ctx.kv_cache_attention(dev, batch, q[:, :3])          # 3 query heads for 2 KV heads
    with pytest.raises(lib.TurboBoAError):
        ctx.kv_cache_attention(dev, lib.KVBatch(i32(starts), i32([10]), i32(pages[:, :0])), q)
    with pytest.raises(AssertionError):
        ctx.kv_cache_attention(dev, batch, q[..., :32])
    with pytest.raises(KeyError):
        ctx.kv_cache_attention(dev, batch, q.half())
    with pytest.raises(lib.TurboBoAError):
        ctx.kv_cache_attention(dev, batch, q.double())
    assert ctx.kv_cache_attention(dev, batch, q[:0]).shape == (0, 4, 64)
