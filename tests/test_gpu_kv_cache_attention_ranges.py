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
