"""tboa_kv_cache_tree_attention of bf16 sequences of more than 512 rows, which a kernel of its own takes (GPU), beside shorter ones of the same call; the bound of an output's error is derived in
tests/tree_ref.py."""
import numpy as np
import pytest
import torch

from tests import test_gpu_kv_cache_tree_attention as few
from tests import tree_ref as ref
from tests.test_gpu_kv_cache_append import i32
from tests.test_gpu_kv_cache_attention import case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx(lib):
    c = lib.Context()
    yield c
    c.close()


SHAPES = [
    # heads, rep, dh, drafted tokens, lengths with them, window, page, scale tokens, words of masks
    (1, 8, 128, [70, 5, 0, 130], [2000, 60, 10, 140], 0, 64, 1, 5),
    (1, 16, 64, [40], [3000], 700, 16, 16, 2),
    (2, 10, 100, [60, 64], [64, 500], 90, 32, 4, 2),
    (1, 32, 32, [20, 17, 3], [20, 9000, 70], 0, 128, 2, 1),
    (1, 24, 256, [25, 30], [400, 30], 33, 64, 64, 1),
    (1, 20, 192, [33], [2], 0, 16, 1, 2),      # more new tokens than places
    (1, 13, 96, [64, 45], [900, 60], 0, 16, 1, 1),
    (1, 1, 128, [600, 7], [700, 200], 0, 64, 1, 19),
    (3, 40, 33, [14], [300], 1, 16, 2, 1),
]


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(str(x).replace(" ", "") for x in s))
def test_ragged_trees(ctx, lib, shape):
    few.test_ragged_trees(ctx, lib, torch.bfloat16, shape)


@pytest.mark.parametrize("before", [0, 70])
def test_masks_of_any_kind(ctx, lib, before):
    new, lens = [40, 3, 45], [40 + before, 3 + before, 45 + before]
    starts, pages, cache, dev, q = case(lib, 1, 14, 64, new, lens, 16, 1, torch.bfloat16, 8)
    rng = np.random.default_rng(1)
    bits = rng.random((88, 64)) < 0.3
    bits[5], bits[6], bits[41], bits[42] = False, True, False, True
    bits[7] = False
    bits[7, 39] = True
    for window in (0, 33):
        got = ctx.kv_cache_tree_attention(dev, lib.KVBatch(i32(starts), i32(lens), i32(pages)), q, ref.as_words(bits).cuda(), window=window)
        torch.cuda.synchronize()
        ref.check(got, cache, starts, lens, pages, q, bits, 1 / 8, window)
        if not before:
            assert (got[[5, 41]] == 0).all()


@pytest.mark.parametrize("new", [40, 64])
def test_values_that_are_special(ctx, lib, new):
    few.test_values_that_are_special(ctx, lib, torch.bfloat16, new, 16)


@pytest.mark.parametrize("heads,rep,new,lens", [(1, 20, [40, 33, 70], [100, 90, 80]), (2, 18, [30], [79]), (3, 24, [25, 2, 0], [90, 60, 30])])
def test_pages_that_are_not_there(ctx, lib, heads, rep, new, lens):
    few.test_many_rows_whose_pages_are_not_there(ctx, lib, heads, rep, new, lens)


@pytest.mark.parametrize("new,lens", [([140, 7], [400, 90]), ([150], [1500])])
def test_captured_and_replayed(lib, new, lens):
    few.test_captured_and_replayed(lib, new, lens)


def test_strides_and_streams(ctx, lib):
    """Queries inside a fused projection, outputs inside a wider tensor, aligned and not, a context on a stream of its own; rows of no sequence left as they were."""
    heads, rep, dh, new, lens = 2, 12, 128, [50, 2, 60], [470, 300, 3000]
    starts, pages, cache, dev, q, bits = few.drafted(lib, heads, rep, dh, new, lens, 64, 1, torch.bfloat16, 33, spare_rows=4)
    tree, rows = ref.as_words(bits).cuda(), starts[-1]
    batch = lib.KVBatch(i32(starts), i32(lens), i32(pages))
    base = ctx.kv_cache_tree_attention(dev, batch, q, tree, out=torch.full_like(q, 7))
    torch.cuda.synchronize()
    ref.check(base, cache, starts, lens, pages, q, bits, 1 / np.sqrt(dh))
    assert (base[rows:] == 7).all()
    n = len(q)
    for shift in (0, 1, 4):
        wide = torch.randn(n * (heads * (rep + 2) + 1) * dh + shift, device="cuda").bfloat16()[shift:].view(n, heads * (rep + 2) + 1, dh)
        wide[:, 1:1 + heads * rep] = q
        out = torch.full((n * (heads * rep + 5) * dh + shift,), 7.0, device="cuda", dtype=torch.bfloat16)[shift:].view(n, heads * rep + 5, dh)
        ctx.kv_cache_tree_attention(dev, batch, wide[:, 1:1 + heads * rep], tree, out=out[:, 2:2 + heads * rep])
        torch.cuda.synchronize()
        assert torch.equal(out[:, 2:2 + heads * rep], base) and (out[:, :2] == 7).all() and (out[:, 2 + heads * rep:] == 7).all()
    side = torch.cuda.Stream()
    other = lib.Context(stream=side)
    try:
        side.wait_stream(torch.cuda.current_stream())
        got = other.kv_cache_tree_attention(dev, batch, q, tree)
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        assert torch.equal(got[:rows], base[:rows])
    finally:
        other.close()


@pytest.mark.parametrize("max_new", [0, 3, 70])
def test_what_the_caller_tells_of_the_batch(ctx, lib, max_new):
    """max_new, also too small a one, chooses between kernels only."""
    new, lens = [70, 3, 31], [900, 2000, 31]
    starts, pages, cache, dev, q, bits = few.drafted(lib, 1, 8, 64, new, lens, 64, 1, torch.bfloat16, 17)
    got = ctx.kv_cache_tree_attention(dev, lib.KVBatch(i32(starts), i32(lens), i32(pages), max_new=max_new), q, ref.as_words(bits).cuda())
    torch.cuda.synchronize()
    ref.check(got, cache, starts, lens, pages, q, bits, 1 / 8)
