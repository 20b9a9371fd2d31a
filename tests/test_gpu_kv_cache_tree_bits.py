"""tboa_kv_cache_tree_attention: the bits that probabilities keep (GPU).  Bounds are those of tests/tree_ref.py."""
import numpy as np
import pytest
import torch

from tests import tree_ref as ref
from tests.test_gpu_kv_cache_append import i32
from tests.test_gpu_kv_cache_tree_attention import drafted

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx(lib):
    c = lib.Context()
    yield c
    c.close()


def rounded(got, want, lim, rows):
    """Every output of `rows` is the bf16 of some value within the bound of a result before its last rounding: rounding is monotonic, so it lies between the bf16 of the bound's ends."""
    g, low, high = got.cpu()[rows].float(), (want - lim)[rows].float().bfloat16().float(), (want + lim)[rows].float().bfloat16().float()
    print("rounded elsewhere: %d of %d" % (((g < low) | (g > high)).sum(), g.numel()), flush=True)
    assert ((g >= low) & (g <= high)).all()


@pytest.mark.parametrize("heads,rep,dh,new,lens,window", [
    (2, 4, 128, [8], [900], 0), (1, 1, 64, [32, 5, 40, 0, 1], [500, 5, 300, 7, 2000], 0), (2, 2, 100, [16, 3], [700, 40], 50), (1, 2, 256, [16, 20], [400, 90], 0), (8, 8, 128, [4, 1, 3, 2], [600, 2000, 3, 65], 0),
    (1, 1, 32, [17], [1300], 0), (2, 8, 128, [16], [500], 0), (1, 4, 64, [64, 7, 30], [800, 50, 400], 70), (1, 2, 96, [120, 2], [300, 30], 0), (1, 4, 256, [33], [200], 0), (1, 8, 128, [70, 20], [700, 90], 0), (1, 20, 64, [30], [400], 100)])
def test_probabilities_keep_22_bits(ctx, lib, heads, rep, dh, new, lens, window):
    """Probabilities times scale are pairs of 11 bits for bf16 queries too: before its last rounding a result is within the bound that fp32 queries have.  In the kernel for many rows (more than 512 of a
    sequence, or of a call for one) the row's largest is 2^-1 or more as half, so that each is off by 2^-25 at most: 2^-24 of at most the largest scale, times 255 levels."""
    starts, pages, cache, dev, q, bits = drafted(lib, heads, rep, dh, new, lens, 64, 1, torch.bfloat16, dh + len(new))
    want, lim = ref.attention(cache, starts, lens, pages, q, bits, 1 / np.sqrt(dh), window, torch.float32)
    used = torch.zeros(len(q), dtype=torch.bool)
    used[:starts[-1]] = True
    for b, n in enumerate(new):
        if n * rep > 512 or (len(new) == 1 and len(q) * rep > 512):
            lim[starts[b]:starts[b + 1]] += lens[b] * 255 * 2.0 ** -24 * float(np.nanmax(cache.vg[..., 0][np.isfinite(cache.vg[..., 0])]))
    for most in (0, max(new)):
        got = ctx.kv_cache_tree_attention(dev, lib.KVBatch(i32(starts), i32(lens), i32(pages), max_new=most), q, ref.as_words(bits).cuda(), window=window)
        torch.cuda.synchronize()
        rounded(got, want, lim, used)
