"""tboa_kv_cache_tree_attention of trees without branches, in a window, beside attention of a chain (GPU).  Bounds are those of tests/tree_ref.py."""
import numpy as np
import pytest
import torch

from tests import tree_ref as ref
from tests.test_gpu_kv_cache_append import i32
from tests.test_gpu_kv_cache_attention import case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx(lib):
    c = lib.Context()
    yield c
    c.close()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("heads,rep,dh,new,lens,window", [(2, 4, 128, [7, 1, 40], [500, 33, 90], 0), (2, 4, 128, [7, 1, 40], [500, 33, 90], 25), (1, 2, 64, [20, 3], [20, 200], 30), (1, 1, 64, [9, 12], [300, 40], 5),
                                                          (1, 2, 64, [70], [90], 16)])
def test_a_chain_in_a_window(ctx, lib, dtype, heads, rep, dh, new, lens, window):
    """A chain whose masks are cut to the window's length is what attention of a chain computes with that window: where a token has `window` ancestors or more the mask's last `window` bits are all that it
    sees, else the row stands as far behind the others as its mask has bits.  Either is within the bound, and the two differ by no more than both bounds together."""
    starts, pages, cache, dev, q = case(lib, heads, rep, dh, new, lens, 16, 1, dtype, 5)
    bits = ref.masks([i - 1 for n in new for i in range(n)], new, -(-max(new) // 32))
    if window:
        for b, n in enumerate(new):
            for i in range(n):
                bits[starts[b] + i, :max(i - window + 1, 0)] = False
    batch = lib.KVBatch(i32(starts), i32(lens), i32(pages))
    got = ctx.kv_cache_tree_attention(dev, batch, q, ref.as_words(bits).cuda(), window=window)
    chain = ctx.kv_cache_attention(dev, batch, q, window=window)
    torch.cuda.synchronize()
    ref.check(got, cache, starts, lens, pages, q, bits, 1 / np.sqrt(dh), window)
    ref.check(chain, cache, starts, lens, pages, q, bits, 1 / np.sqrt(dh), window)
    _, lim = ref.attention(cache, starts, lens, pages, q, bits, 1 / np.sqrt(dh), window, dtype)
    assert ((got.double() - chain.double()).abs().cpu() <= 2 * lim).all()
