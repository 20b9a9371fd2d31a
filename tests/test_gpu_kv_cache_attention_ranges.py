"""tboa_kv_cache_attention where numbers of different size meet (GPU): every row to the bound of its own values (tests/attention_bounds.py), whatever the tokens that it does not see and the rows beside it hold."""
import numpy as np
import pytest
import torch

from tests.attention_bounds import attention, check
from tests.test_gpu_kv_cache_append import i32
from tests.test_gpu_kv_cache_attention import SHAPES, case

pytestmark = pytest.mark.gpu


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


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("factor", [1e9, 1e15, 1e30, 3e36])
@pytest.mark.parametrize("new,many", [(3, False), (40, False), (40, True), (200, True)])
def test_queries_of_other_rows(ctx, lib, dtype, factor, new, many):
    """One finite row far above the others, and one far below: the others are what they are without them, to the bound of their own values."""
    if many and dtype == torch.float32:
        pytest.skip("fp32 has one kernel")
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
