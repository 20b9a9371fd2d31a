"""tboa_kv_cache_attention's kernel for many rows where a unit of rows is cut into pieces of its tokens and joined, in graphs, beside itself and far from the cache's first byte (GPU).  Rows of pages for
2^22 tokens send short calls to that kernel."""
import numpy as np
import pytest
import torch

from tests.attention_bounds import check
from tests.test_gpu_kv_cache_append import i32, layout
from tests.test_gpu_kv_cache_attention import case
from tests.test_gpu_kv_cache_attention_ranges import wide
from tests.test_gpu_serving import Step, captured

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx(lib):
    c = lib.Context()
    yield c
    c.close()


@pytest.mark.parametrize("window", [0, 700])
@pytest.mark.parametrize("pt", [16, 64])
@pytest.mark.parametrize("dh", [32, 64, 90, 128, 192, 256])
@pytest.mark.parametrize("holes", [False, True])
def test_units_cut_into_pieces(ctx, lib, dh, pt, window, holes):
    """80 rows behind 5000 tokens in up to 19 pieces, and 66 behind 270 in one, or none where pages are missing: a piece of which no row, or not every row, sees anything."""
    new, lens = [40, 33], [5000, 270]
    starts, pages, cache, dev, q = case(lib, 1, 2, dh, new, lens, pt, 1, torch.bfloat16, dh + pt, spare_rows=2)
    pages = wide(pages, pt)
    if holes:
        pages[0, 1024 // pt:1600 // pt] = -1
        pages[0, 4480 // pt:4800 // pt] = len(cache.data)
        pages[0, 4985 // pt] = 1 << 30
        pages[1] = -5
    out = torch.full_like(q, 7)
    got = ctx.kv_cache_attention(dev, lib.KVBatch(i32(starts), i32(lens), i32(pages)), q, window=window, out=out)
    torch.cuda.synchronize()
    check(got, cache, starts, lens, pages, q, 1 / np.sqrt(dh), window, many=True)
    assert (got[starts[-1]:] == 7).all() and (not holes or (got[starts[1]:starts[2]] == 0).all())


@pytest.mark.parametrize("heads,rep,dh,new,lens", [(3, 4, 128, [300, 20], [300, 900]), (2, 8, 64, [513], [700]), (1, 5, 256, [129, 1, 60], [400, 3000, 2000]), (5, 1, 100, [257], [1500])])
def test_units_of_several_row_tiles_in_pieces(ctx, lib, heads, rep, dh, new, lens):
    """Row tiles that see less than others of their call, and so have fewer pieces than the call is cut into."""
    starts, pages, cache, dev, q = case(lib, heads, rep, dh, new, lens, 64, 16, torch.bfloat16, 17)
    pages = wide(pages, 64)
    got = ctx.kv_cache_attention(dev, lib.KVBatch(i32(starts), i32(lens), i32(pages)), q)
    torch.cuda.synchronize()
    # the sequences of up to 32 rows are the other kernel's, whose bound is tighter
    check(got, cache, starts, lens, pages, q, 1 / np.sqrt(dh), 0, many=True)


def long_step(lib, lens, pages, total, dh, seed):
    return Step(lib, [40, 3, 17, 60], lens, wide(pages, 64), total, 2, 4, dh, 64, 16, torch.bfloat16, seed)


@pytest.mark.parametrize("dh", [128, 256])
def test_prompts_replayed_from_a_graph(ctx, lib, dh):
    lens = np.array([5, 1200, 64, 0])
    total, pages = layout(lens + 400, 64, 4)
    stream = torch.cuda.Stream()
    own = lib.Context(stream=stream)
    try:
        step = long_step(lib, lens, pages, total, dh, 1)
        own.reserve_workspace(step.need(own))
        held = own.workspace_bytes()
        shadow = step.data.clone()
        torch.cuda.synchronize()
        graph = captured(lib, step, own, stream)
        assert own.workspace_bytes() == held
        for turn in range(4):
            lens = lens + step.new
            step.fill(lens, 10 * turn)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            got = step.out.clone()
            want = step.run(ctx, data=shadow, out=torch.empty_like(step.out), turned=torch.empty_like(step.turned))
            torch.cuda.synchronize()
            assert torch.equal(step.data, shadow) and torch.equal(got, want) and torch.isfinite(got).all(), turn
            if turn == 1:
                own.reserve_workspace(held + (64 << 20))
                filler = torch.full((held,), 255, dtype=torch.uint8, device="cuda")
                assert filler[0] == 255
    finally:
        own.close()


def test_prompts_of_two_contexts(ctx, lib):
    """Each with a workspace of its own: the bits of one after the other."""
    lens = np.array([70, 1290, 17, 100])
    total, pages = layout(lens, 64, 3)
    ctxs = [lib.Context(stream=torch.cuda.Stream()) for _ in range(2)]
    try:
        steps = [long_step(lib, lens, pages, total, 128, s) for s in range(2)]
        for i, s in enumerate(steps):
            s.fill(lens, 50 + i)
        torch.cuda.synchronize()
        got = [[], []]
        for _ in range(3):
            for i, (s, c) in enumerate(zip(steps, ctxs)):
                got[i].append(s.run(c, out=torch.empty_like(s.out)))
        torch.cuda.synchronize()
        for s, outs in zip(steps, got):
            data = torch.zeros_like(s.data)
            want = s.run(ctx, data=data, out=torch.empty_like(s.out))
            torch.cuda.synchronize()
            assert all(torch.equal(o, want) for o in outs) and torch.equal(data, s.data)
    finally:
        for c in ctxs:
            c.close()


@pytest.mark.parametrize("pt", [16, 64])
def test_prompts_over_pages_beyond_32_bits(ctx, lib, pt):
    heads, rep, dh = 8, 2, 128
    new, lens = [40, 100], [900, 150]
    starts, pages, cache, dev, q = case(lib, heads, rep, dh, new, lens, pt, 1, torch.bfloat16, 31)
    pages = wide(pages, pt)
    batch = lib.KVBatch(i32(starts), i32(lens), i32(pages))
    base = ctx.kv_cache_attention(dev, batch, q)
    torch.cuda.synchronize()
    check(base, cache, starts, lens, pages, q, 1 / np.sqrt(dh), 0, many=True)
    per = dev.data.shape[1]
    far = (1 << 32) // per + 50
    big = torch.zeros(far + len(cache.data), per, dtype=torch.uint8, device="cuda")
    big[far:] = dev.data
    moved = np.where(pages >= 0, pages + far, -1)
    got = ctx.kv_cache_attention(lib.KVCache(big, heads, dh, pt, 1), lib.KVBatch(i32(starts), i32(lens), i32(moved)), q)
    torch.cuda.synchronize()
    assert torch.equal(got, base)
