"""tboa_kv_cache_append against the 64-bit form (GPU): the same bytes, in every page and also where nothing was to be written."""
import numpy as np
import pytest
import torch

from oracle import turboboa_ref as O
from tests import serving_ref as ref
from tests.test_gpu_head_norm_rotate import table

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx(lib):
    c = lib.Context()
    yield c
    c.close()


def layout(lens, pt, seed, spare=2, wide=None):
    """Page numbers in no order, and rows wide enough for the longest sequence."""
    need = [-(-n // pt) for n in lens]
    total = sum(need) + spare
    order = np.random.default_rng(seed).permutation(total)
    pages = np.full((len(lens), max(max(need), 1) if wide is None else wide), 0, np.int32)
    at = 0
    for b, n in enumerate(need):
        pages[b, :n] = order[at:at + n]
        at += n
    return total, pages


def values(rows, heads, dh, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, heads, dh, generator=g) * torch.exp(torch.randn(rows, heads, 1, generator=g))
    return x.to(dtype)


def run(ctx, lib, cache, batch, k, v, tab, adjacent, positions=None):
    ctx.kv_cache_append(cache, batch, k, v, rotation=lib.Rotation(tab.cuda(), adjacent=adjacent) if tab is not None else None, positions=positions)
    torch.cuda.synchronize()


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("heads,dh,rot,adjacent,pt,st", [
    (2, 128, 128, False, 64, 1), (3, 128, 64, True, 16, 16), (2, 100, 52, True, 64, 64), (1, 64, 0, False, 128, 2), (2, 96, 96, False, 32, 8), (1, 256, 256, False, 64, 32),
    (2, 33, 10, False, 16, 4), (1, 1, 0, False, 16, 1), (2, 192, 64, True, 128, 128), (5, 32, 32, False, 1024, 1024), (1, 80, 80, True, 16, 1)])
def test_steps_of_a_ragged_batch(ctx, lib, dtype, heads, dh, rot, adjacent, pt, st):
    """Prompts, then tokens one at a time and in small pieces, sequences that pause, come late and stay empty."""
    plan = [[37, 0, 1, 0, 130], [1, 1, 1, 0, 1], [0, 3, 1, 0, 70], [1, 16, 0, 0, 1], [2, 1, 40, 0, 1]]
    final = np.sum(plan, 0)
    total, pages = layout(final, pt, 5)
    data = torch.randint(0, 256, (total, lib.KVCache.page_bytes(heads, dh, pt, st)), generator=torch.Generator().manual_seed(1), dtype=torch.uint8)
    cache = lib.KVCache(data.cuda(), heads, dh, pt, st)
    want = ref.Cache(data.numpy(), heads, dh, pt, st)
    tab = table(400, rot) if rot else None
    lens = np.zeros(5, int)
    for step, new in enumerate(plan):
        lens = lens + new
        starts = np.concatenate([[0], np.cumsum(new)])
        rows = starts[-1] + 2          # two rows behind the last sequence
        wide = values(rows, 2 * heads + 1, dh, dtype, 100 * step + dh).cuda()      # keys and values of one fused projection
        k, v = wide[:, :heads], wide[:, heads + 1:]
        batch = lib.KVBatch(i32(starts), i32(lens), i32(pages))
        run(ctx, lib, cache, batch, k, v, tab, adjacent)
        k64, v64 = k.double().cpu().numpy(), v.double().cpu().numpy()
        place = np.concatenate([np.arange(l - n, l) for l, n in zip(lens, new)] + [[0, 0]]).astype(int)
        ref.append(want, starts, lens, pages, ref.norm_rotate(k64, None, 0, None if tab is None else tab.numpy(), place, adjacent), v64, rows)
        got = cache.data.cpu().numpy()
        assert np.array_equal(got, want.data), (step, np.argwhere(got != want.data)[:5])
        run(ctx, lib, cache, batch, k, v, tab, adjacent)      # the same tokens once more: nothing changes
        assert np.array_equal(cache.data.cpu().numpy(), want.data), step


def test_is_the_quantizer_of_the_hessians(ctx, lib):
    """A grid per token: the values are those of the per-token Min-Max quantizer at 8 bits, up to the rounding of the scale to fp32 (2^-24 of a value of at most 255 steps) and a
    level where a value lies within that of a border."""
    heads, dh, n = 2, 128, 64
    x = values(n, heads, dh, torch.float32, 7)
    cache = lib.KVCache.empty(1, heads, dh)
    run(ctx, lib, cache, lib.KVBatch(i32([0, n]), i32([n]), i32([[0]])), x.cuda(), x.flip(0).contiguous().cuda(), None, False)
    got = ref.Cache(cache.data.cpu().numpy(), heads, dh, 64, 1)
    for kv, y in (("k", x), ("v", x.flip(0))):
        want = O.act_fakequant_per_token(y.numpy().reshape(-1, dh), 8).reshape(n, heads, dh)
        have = np.stack([got.values(kv, 0, t) for t in range(n)])
        step = got.grid(kv)[0, :, :, 0].astype(np.float64).T[..., None]
        off = np.abs(have - want) / step
        assert np.all(off <= 1.001) and np.mean(off > 1e-4) < 1e-4


def test_values_that_are_special(ctx, lib):
    """Zeros, one sign only, values next to nothing, the largest ones, NaN and infinities (their block alone, and it stays so)."""
    for st in (1, 4, 16, 32):
        heads, dh, pt, n = 2, 40, 32, 32
        x = torch.randn(n, heads, dh, generator=torch.Generator().manual_seed(1))
        x[0] = 0
        x[1] = x[1].abs() + 5
        x[2] = -x[2].abs() - 5
        x[3] *= 1e-42
        x[4] *= 3e37
        x[9, 0, 3] = float("nan")
        x[14, 1, 0] = float("inf")
        x[20, 1, 39] = -float("inf")
        data = np.full((1, lib.KVCache.page_bytes(heads, dh, pt, st)), 255, np.uint8)
        cache, want = lib.KVCache(torch.tensor(data).cuda(), heads, dh, pt, st), ref.Cache(data, heads, dh, pt, st)
        for a, e in ((0, 21), (21, 22), (22, 32)):
            k, v = x[a:e].cuda(), x.flip(2)[a:e].contiguous().cuda()
            run(ctx, lib, cache, lib.KVBatch(i32([0, e - a]), i32([e]), i32([[0]])), k, v, None, False)
            ref.append(want, [0, e - a], [e], np.zeros((1, 1), int), k.double().cpu().numpy(), v.double().cpu().numpy(), e - a)
        got = cache.data.cpu().numpy()
        w = ref.Cache(got, heads, dh, pt, st)
        for kv in "kv":
            g, r = w.grid(kv), want.grid(kv)
            assert np.array_equal(np.isnan(g[..., 0]), np.isnan(r[..., 0])) and np.array_equal(np.nan_to_num(g, nan=-1), np.nan_to_num(r, nan=-1))
        assert np.array_equal(w.k[..., :dh], want.k[..., :dh]) and np.array_equal(w.v[..., :dh, :], want.v[..., :dh, :])


def test_what_has_no_place(ctx, lib):
    """Pages outside the cache, places beyond the row of pages, more new tokens than the length says, rows that starts leaves out: nothing is written for them."""
    heads, dh, pt, st = 2, 64, 16, 4
    starts, lens = [0, 20, 41, 50, 50], [40, 60, 5, 10]
    pages = np.array([[3, -1, 5], [7, 2, 9], [8, 1, 0], [4, 4, 4]], np.int32)      # 9 is no page; the second sequence's places beyond 48 have none
    data = torch.randint(0, 256, (9, lib.KVCache.page_bytes(heads, dh, pt, st)), generator=torch.Generator().manual_seed(2), dtype=torch.uint8)
    k, v = values(47, heads, dh, torch.float32, 1), values(47, heads, dh, torch.float32, 2)      # starts goes beyond the rows
    cache, want = lib.KVCache(data.cuda(), heads, dh, pt, st), ref.Cache(data.numpy(), heads, dh, pt, st)
    run(ctx, lib, cache, lib.KVBatch(i32(starts), i32(lens), i32(pages)), k.cuda(), v.cuda(), None, False)
    clipped = np.minimum(starts, 47)
    ref.append(want, clipped, lens, pages, k.double().numpy(), v.double().numpy(), 47)
    assert np.array_equal(cache.data.cpu().numpy(), want.data)


def test_positions_of_their_own(ctx, lib):
    heads, dh = 1, 64
    k = values(5, heads, dh, torch.bfloat16, 3)
    tab = table(50, 64)
    pos = [40, 3, 49, 50, 7]
    cache = lib.KVCache(torch.zeros(1, lib.KVCache.page_bytes(heads, dh), dtype=torch.uint8, device="cuda"), heads, dh)
    run(ctx, lib, cache, lib.KVBatch(i32([0, 5]), i32([5]), i32([[0]])), k.cuda(), k.cuda(), tab, False, positions=i32(pos))
    want = ref.Cache(np.zeros_like(cache.data.cpu().numpy()), heads, dh, 64, 1)
    ref.append(want, [0, 5], [5], np.zeros((1, 1), int), ref.norm_rotate(k.double().numpy(), None, 0, tab.numpy(), pos, False), k.double().numpy(), 5)
    assert np.array_equal(np.nan_to_num(ref.Cache(cache.data.cpu().numpy(), heads, dh, 64, 1).kg, nan=-7), np.nan_to_num(want.kg, nan=-7))
    assert np.isnan(want.kg[0, 0, 3, 0])      # the table has 50 positions


def test_many_sequences(ctx, lib):
    """More sequences than a wavefront has lanes, most of them without a new token."""
    heads, dh, pt, st, B = 1, 32, 16, 1, 203
    rng = np.random.default_rng(0)
    new, old = rng.integers(0, 3, B), rng.integers(0, 20, B)
    new[70:140] = 0
    starts, lens = np.concatenate([[0], np.cumsum(new)]), new + old
    total, pages = layout(lens, pt, 1)
    k, v = values(starts[-1], heads, dh, torch.bfloat16, 1), values(starts[-1], heads, dh, torch.bfloat16, 2)
    data = torch.zeros(total, lib.KVCache.page_bytes(heads, dh, pt, st), dtype=torch.uint8)
    cache, want = lib.KVCache(data.cuda(), heads, dh, pt, st), ref.Cache(data.numpy(), heads, dh, pt, st)
    run(ctx, lib, cache, lib.KVBatch(i32(starts), i32(lens), i32(pages)), k.cuda(), v.cuda(), None, False)
    ref.append(want, starts, lens, pages, k.double().numpy(), v.double().numpy(), starts[-1])
    assert np.array_equal(cache.data.cpu().numpy(), want.data)
