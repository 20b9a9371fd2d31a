"""tboa_kv_cache_attention where numbers of different size meet (GPU): every row to the bound of its own values (tests/attention_bounds.py), whatever the tokens that it does not see and the rows beside it hold."""
import numpy as np
import pytest
import torch

from tests.attention_bounds import attention, check
from tests.test_gpu_kv_cache_append import i32
from tests.test_gpu_kv_cache_attention import SHAPES, case

pytestmark = pytest.mark.gpu


def kinds(*cases):
    """The cases, whose last entry says whether they are the kernel's for many rows, in both types; fp32 has no such kernel."""
    return [(dtype, *c) for dtype in (torch.bfloat16, torch.float32) for c in cases if not (c[-1] and dtype == torch.float32)]


@pytest.fixture(scope="module")
def ctx(lib):
    c = lib.Context()
    yield c
    c.close()


def wide(pages, pt):
    """Rows of pages for 2^22 tokens, of which the sequences have few: by what the host knows these are long calls, and more than 32 rows of 16-bit inputs take the kernel for many."""
    return np.pad(pages, ((0, 0), (0, (1 << 22) // pt - pages.shape[1])), constant_values=-1)


def attend(ctx, lib, cache, starts, lens, pages, q, **kw):
    dev = lib.KVCache(torch.tensor(cache.data).cuda(), cache.heads, cache.dh, cache.pt, cache.st)
    out = ctx.kv_cache_attention(dev, lib.KVBatch(i32(starts), i32(lens), i32(pages)), q, **kw)
    torch.cuda.synchronize()
    return out


@pytest.mark.parametrize("shape", [s for s in SHAPES if max(s[3]) * s[1] <= 32] + [(2, 4, 128, [1, 1], [3000, 6001], 0, 64, 1), (1, 8, 64, [2], [5000], 700, 16, 16)],
                         ids=lambda s: "-".join(str(x).replace(" ", "") for x in s))
def test_probabilities_of_few_rows(ctx, lib, shape):
    """bf16 queries of sequences of up to 32 rows: probabilities have the 22 bits that those of fp32 queries have."""
    heads, rep, dh, new, lens, window, pt, st = shape
    starts, pages, cache, _, q = case(lib, heads, rep, dh, new, lens, pt, st, torch.bfloat16, 3 * dh + len(new))
    got = attend(ctx, lib, cache, starts, lens, pages, q, window=window)
    # what the rounding of the output hides: the share of outputs that are not the correctly rounded ones.  A probability off by 2^-22 moves an output by 2^-14 of a step of bf16, so a
    # ten-thousandth of them; the scores' own errors (fp32 sums of dh terms, 2^-20 of the sizes here) ten times that.  One half's 2^-11 would be one in ten
    check(got, cache, starts, lens, pages, q, 1 / np.sqrt(dh), window, telling=0.8)
    want = attention(cache, starts, lens, pages, q, 1 / np.sqrt(dh), window)[0]
    other = (got.double().cpu() != want.to(torch.bfloat16).double()).double().mean().item()
    print("outputs that are not the nearest: %.5f" % other)
    assert other < 0.01 + 3 / got.numel()


@pytest.mark.parametrize("factor", [1e7, 1e12, 1e30])
@pytest.mark.parametrize("dtype,new,window,many", kinds((1, 40, False), (7, 0, False), (7, 30, False), (50, 0, False), (50, 0, True), (70, 33, True), (200, 150, True)))
def test_scales_of_tokens_that_are_not_seen(ctx, lib, dtype, factor, new, window, many):
    """A scale of V far above the others, behind a row's own place or before its window, changes nothing in the row."""
    length, dh, rep = 300, 64, 2
    starts, pages, cache, _, q = case(lib, 2, rep, dh, [new], [length], 16, 1, dtype, 40 + new)
    last = length - 1 - (new - 1) // 2      # seen by the last half of the rows; the row before it does not
    spots = [last] if new > 1 else []
    if window:
        spots += [length - new - window, length - new - window + new // 2]      # out of the first row's window; leaves it half way
    for t in spots:
        cache.vg[pages[0, t // 16], :, t % 16, 0] *= factor
    if many:
        pages = wide(pages, 16)
    got = attend(ctx, lib, cache, starts, [length], pages, q, window=window)
    check(got, cache, starts, [length], pages, q, 1 / 8, window, many=many)


@pytest.mark.parametrize("dtype,new,many", kinds((1, False), (5, False), (40, False), (40, True), (300, True)))
def test_scales_of_tokens_that_hardly_count(ctx, lib, dtype, new, many):
    """Scales of V that grow as the scores fall: large ones with probabilities next to nothing, met first, in between and last."""
    length, dh = 700, 64
    starts, pages, cache, _, q = case(lib, 1, 1, dh, [new], [length], 64, 1, dtype, 60 + new)
    q[:] = (torch.randn(dh, generator=torch.Generator().manual_seed(1)).to(dtype) / 8).cuda()      # every row asks the same
    sign = np.sign(q[0, 0].float().cpu().numpy()).astype(int)
    for t, (low, factor) in {3: (40, 1e10), 100: (80, 1e25), 250: (25, 1e5), 390: (60, 1e16), 398: (127, 1e30)}.items():      # all rows see them
        at = pages[0, t // 64]
        cache.k[at, 0, t % 64, :dh], cache.kg[at, 0, t % 64] = 128 - sign * low, (1.0, 128)      # a score of -low / 8 sum |q|
        cache.vg[at, 0, t % 64, 0] *= factor
    if many:
        pages = wide(pages, 64)
    got = attend(ctx, lib, cache, starts, [length], pages, q)
    check(got, cache, starts, [length], pages, q, 1 / 8, 0, many=many)


@pytest.mark.parametrize("dtype,new,many", kinds((4, False), (60, False), (60, True)))
def test_scales_as_far_apart_as_an_append_makes_them(ctx, lib, dtype, new, many):
    """Beside scales of 1e-14, the largest there is: behind the rows' place, and in a token that they see with a probability of 2^-126 or less."""
    length, dh = 200, 64
    starts, pages, cache, _, q = case(lib, 1, 1, dh, [new], [length], 64, 1, dtype, 70 + new)
    q[:] = (torch.randn(dh, generator=torch.Generator().manual_seed(1)).to(dtype)).cuda()
    cache.vg[..., 0] *= 1e-12
    sign = np.sign(q[0, 0].float().cpu().numpy()).astype(int)
    for t in (5, 120):
        at = pages[0, t // 64]
        cache.k[at, 0, t % 64, :dh], cache.kg[at, 0, t % 64] = 128 - sign * 127, (4.0, 128)      # a score of -63 sum |q|, some -3000
        cache.vg[at, 0, t % 64, 0] = 2.0 ** 121
    cache.vg[pages[0, (length - 1) // 64], 0, (length - 1) % 64, 0] = 2.0 ** 121      # the last row alone sees it
    if many:
        pages = wide(pages, 64)
    got = attend(ctx, lib, cache, starts, [length], pages, q)
    check(got, cache, starts, [length], pages, q, 1 / 8, 0, many=many)


@pytest.mark.parametrize("factor", [1e9, 1e15, 1e30, 3e36])
@pytest.mark.parametrize("dtype,new,many", kinds((3, False), (40, False), (40, True), (200, True)))
def test_queries_of_other_rows(ctx, lib, dtype, factor, new, many):
    """One finite row far above the others, and one far below: the others are what they are without them, to the bound of their own values."""
    length, dh, rep = 260, 64, 2
    starts, pages, cache, _, q = case(lib, 1, rep, dh, [new], [length], 16, 1, dtype, 80 + new)
    q[1, 0] *= factor
    q[2, 1] /= factor
    q[0, 1] = 0
    rows = torch.ones(new, rep, dtype=torch.bool)
    rows[1, 0] = False      # a softmax of scores of 1e9 and more: one token alone, which fp32 scores may not tell from its next
    if many:
        pages = wide(pages, 16)
    got = attend(ctx, lib, cache, starts, [length], pages, q)
    assert torch.isfinite(got).all()
    check(got, cache, starts, [length], pages, q, 1 / 8, 0, many=many, rows=rows)
    # what the large row itself says: the token of the largest score, where no other comes near it
    key = torch.tensor(cache.k[pages[0, np.arange(length) // 16], 0, np.arange(length) % 16, :dh], dtype=torch.float64)
    grid = torch.tensor(cache.kg[pages[0, np.arange(length) // 16], 0, np.arange(length) % 16], dtype=torch.float64)
    seen = length - new + 2      # row 1's
    x = (((key - grid[:, 1:]) * grid[:, :1]) @ q[1, 0].double().cpu())[:seen]
    best, next_ = x.topk(2).values
    if (best - next_) / best.abs() > 1e-4 and best < 1e37:
        t = int(x.argmax())
        page, off = pages[0, t // 16], t % 16
        v = (torch.tensor(cache.v[page, 0, off // 16, :dh, off % 16], dtype=torch.float64) - float(cache.vg[page, 0, off, 1])) * float(cache.vg[page, 0, off, 0])
        assert ((got[1, 0].double().cpu() - v).abs() <= (torch.finfo(dtype).eps / 2 + 2.0 ** (-11 if many else -21)) * v.abs() + 2.0 ** -24 * 255 * float(cache.vg[page, 0, off, 0])).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_special_values_to_the_bound_of_each_sequence(ctx, lib, dtype):
    """Two sequences, one with scales of V from 1e-8 to 1e4 and a NaN: the other one's rows, with a NaN query, queries of 1e-20 and of 1e-3 among them, to their own bound; both kernels."""
    for new, many in ((1, False), (50, False), (50, True)):
        if many and dtype == torch.float32:
            continue
        starts, pages, cache, _, q = case(lib, 1, 2, 64, [new, new], [150, 150], 16, 1, dtype, 5)
        cache.vg[pages[1, 145 // 16], 0, 145 % 16, 0] = np.nan
        cache.vg[pages[1, 2], 0, :, 0] *= 1e-6
        cache.vg[pages[1, 1], 0, :, 0] *= 1e6
        q[0] *= 1e-20
        rows = torch.ones(len(q), 2, dtype=torch.bool)
        if new > 1:
            q[3, 0, 0] = float("nan")
            q[5] *= 1e-3
            rows[3, 0] = False
        table = wide(pages, 16) if many else pages
        got = attend(ctx, lib, cache, starts, [150, 150], table, q)
        assert new == 1 or torch.isnan(got[3, 0]).all()
        check(got, cache, starts, [150, 150], table, q, 1 / 8, 0, many=many, rows=rows)


@pytest.mark.parametrize("new,spare", [(4, 60), (16, 1), (3, 13)])
def test_probabilities_of_one_padded_sequence(ctx, lib, new, spare):
    """Up to 32 rows alone in a call of more: by its n_tokens a long one, in either kernel."""
    starts, pages, cache, _, q = case(lib, 4, 2, 64, [new], [300], 16, 1, torch.bfloat16, 90 + new, spare_rows=spare)
    want = attention(cache, starts, [300], pages, q, 1 / 8, 0)[0][:new].to(torch.bfloat16)
    for p, many in ((pages, False), (wide(pages, 16), True)):
        got = attend(ctx, lib, cache, starts, [300], p, q)
        check(got, cache, starts, [300], p, q, 1 / 8, 0, many=many, rows_of_call=len(q) * 2)
        other = (got[:new].cpu() != want).double().mean().item()
        print("outputs that are not the nearest: %.5f" % other)
        assert (other > 0.02) == (len(q) * 2 > 32)


@pytest.mark.parametrize("dtype,heads,new,many", kinds((800, 1, False), (1, 5, False), (150, 40, False), (1, 40, True), (150, 40, True)))
def test_scales_that_vanish_in_between(ctx, lib, dtype, heads, new, many):
    """Large scales first, then scores so much higher that those count for nothing, of tokens whose scale is 0, then small scales at the same height.  (Many units: a wavefront goes through all three.)"""
    length, dh = 1700, 32
    starts, pages, cache, _, q = case(lib, heads, 1, dh, [new], [length], 64, 1, dtype, 110 + new)
    q[:] = (torch.randn(dh, generator=torch.Generator().manual_seed(1)).to(dtype)).cuda()
    sign = np.sign(q[0, 0].float().cpu().numpy()).astype(int)
    for t in range(length):
        at, off = pages[0, t // 64], t % 64
        if t < 256:
            cache.k[at, :, off, :dh], cache.kg[at, :, off] = 128 - sign * 127, (4.0, 128)      # a score of -90 sum |q|, some -2000
        cache.vg[at, :, off, 0] = 2.0 ** 115 if t < 256 else 0.0 if t < 512 else 2.0 ** -100
    if many:
        pages = wide(pages, 64)
    got = attend(ctx, lib, cache, starts, [length], pages, q)
    assert torch.isfinite(got).all()
    check(got, cache, starts, [length], pages, q, 1 / np.sqrt(dh), 0, many=many)
