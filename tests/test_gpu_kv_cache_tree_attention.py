"""tboa_kv_cache_tree_attention against the 64-bit form on the cache's own values (GPU); the bound of an output's error is derived in tests/tree_ref.py."""
import numpy as np
import pytest
import torch

from tests import tree_ref as ref
from tests.test_gpu_kv_cache_append import i32, layout
from tests.test_gpu_kv_cache_attention import case, filled

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx(lib):
    c = lib.Context()
    yield c
    c.close()


def grown(new, seed, wide=6):
    """Parents of random trees: a token's parent is one of the `wide` before it, or none."""
    rng = np.random.default_rng(seed)
    return [max(i - 1 - int(rng.integers(0, wide)), -1) for n in new for i in range(n)]


def drafted(lib, heads, rep, dh, new, lens, pt, st, dtype, seed, words=0, spare_rows=0):
    starts, pages, cache, dev, q = case(lib, heads, rep, dh, new, lens, pt, st, dtype, seed, spare_rows)
    words = words or max(-(-max(new) // 32), 1)
    bits = np.concatenate([ref.masks(grown(new, seed), new, words), np.zeros((spare_rows, 32 * words), bool)])
    return starts, pages, cache, dev, q, bits


SHAPES = [
    # heads, rep, dh, drafted tokens, lengths with them, window, page, scale tokens, words of masks
    (1, 1, 128, [1], [1], 0, 64, 1, 1),
    (2, 8, 128, [16], [500], 0, 64, 1, 1),
    (2, 1, 64, [5, 1, 33], [5, 64, 97], 0, 64, 1, 2),
    (1, 3, 100, [11, 0, 2, 5], [130, 40, 2, 200], 0, 16, 16, 1),
    (2, 2, 32, [7, 1, 0, 30], [7, 300, 0, 95], 0, 32, 4, 3),
    (1, 8, 96, [13], [333], 0, 128, 2, 1),
    (1, 17, 64, [2, 9], [70, 1030], 0, 1024, 32, 1),
    (1, 2, 256, [20, 33], [200, 70], 0, 64, 64, 2),
    (1, 1, 192, [65], [257], 0, 16, 1, 3),
    (2, 4, 128, [40, 1], [200, 777], 50, 64, 1, 2),
    (1, 2, 33, [20, 3], [20, 200], 1, 16, 2, 1),
    (1, 4, 80, [64, 64], [64, 500], 65, 64, 16, 2),
    (1, 1, 1, [3], [40], 0, 16, 1, 1),
    (1, 5, 128, [4, 3, 1], [2, 0, 1], 0, 16, 1, 1),      # more new tokens than places
    (1, 2, 64, [300], [300], 0, 64, 1, 10),
    (1, 1, 128, [129, 200], [700, 201], 0, 64, 16, 7),
    (1, 3, 128, [40, 7], [140, 90], 0, 64, 1, 1),         # new tokens that no mask has bits for
    (2, 8, 64, [70], [2000], 1000, 64, 1, 3),
]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(str(x).replace(" ", "") for x in s))
def test_ragged_trees(ctx, lib, dtype, shape):
    heads, rep, dh, new, lens, window, pt, st, words = shape
    starts, pages, cache, dev, q, bits = drafted(lib, heads, rep, dh, new, lens, pt, st, dtype, 11 * dh + len(new), words, spare_rows=3)
    out = torch.full_like(q, 7)
    for most in (0, max(new)) if max(new) <= 32 * words else (0,):      # what the caller knows of the batch changes nothing but the kernel
        got = ctx.kv_cache_tree_attention(dev, lib.KVBatch(i32(starts), i32(lens), i32(pages), max_new=most), q, ref.as_words(bits).cuda(), window=window, out=out)
        torch.cuda.synchronize()
        ref.check(got, cache, starts, lens, pages, q, bits, 1 / np.sqrt(dh), window, telling=0.8)
        assert (got[starts[-1]:] == 7).all()          # rows of no sequence


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("heads,rep,dh,new,lens,window", [(2, 4, 128, [7, 1, 40], [500, 33, 90], 0), (1, 2, 64, [20, 3], [20, 200], 30)])
def test_a_chain_is_causal_attention(ctx, lib, dtype, heads, rep, dh, new, lens, window):
    """Trees without branches: both calls compute the same, each within the bound."""
    starts, pages, cache, dev, q = case(lib, heads, rep, dh, new, lens, 16, 1, dtype, 5)
    tree, depth = lib.tree_masks([i - 1 for n in new for i in range(n)], new)
    assert depth.tolist() == [i for n in new for i in range(n)]
    bits = ref.masks([i - 1 for n in new for i in range(n)], new, tree.shape[1])
    assert torch.equal(ref.as_words(bits), tree)
    if window:
        for b, n in enumerate(new):      # the mask alone decides on new tokens
            for i in range(n):
                bits[starts[b] + i, :max(i - window + 1, 0)] = False
    batch = lib.KVBatch(i32(starts), i32(lens), i32(pages))
    got = ctx.kv_cache_tree_attention(dev, batch, q, ref.as_words(bits).cuda())
    torch.cuda.synchronize()
    if not window:
        want = ref.check(got, cache, starts, lens, pages, q, bits, 1 / np.sqrt(dh))
        chain = ctx.kv_cache_attention(dev, batch, q)
        torch.cuda.synchronize()
        ref.check(chain, cache, starts, lens, pages, q, bits, 1 / np.sqrt(dh))
        assert want.shape == chain.shape


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_a_long_context_in_pieces(ctx, lib, dtype):
    """Tokens split over many workgroups, a scale of the caller's, and queries that make one token count nearly alone."""
    for new, length, gain, rep in ((1, 20000, 1.0, 2), (3, 9001, 30.0, 2), (20, 5000, 3.0, 2), (64, 7000, 1.0, 4)):
        starts, pages, cache, dev, q, bits = drafted(lib, 1, rep, 64, [new], [length], 64, 1, dtype, new)
        q = (q.float() * gain).to(dtype)
        got = ctx.kv_cache_tree_attention(dev, lib.KVBatch(i32(starts), i32([length]), i32(pages)), q, ref.as_words(bits).cuda(), scale=0.2)
        torch.cuda.synchronize()
        ref.check(got, cache, starts, [length], pages, q, bits, 0.2)


@pytest.mark.parametrize("max_new", [0, 20])
def test_many_sequences(ctx, lib, max_new):
    rng = np.random.default_rng(4)
    new, old = rng.integers(0, 21, 150), rng.integers(0, 300, 150)
    new[64:100] = 0
    lens = (new + old).tolist()
    starts, pages, cache, dev, q, bits = drafted(lib, 2, 3, 32, new.tolist(), lens, 16, 1, torch.bfloat16, 9)
    got = ctx.kv_cache_tree_attention(dev, lib.KVBatch(i32(starts), i32(lens), i32(pages), max_new=max_new), q, ref.as_words(bits).cuda())
    torch.cuda.synchronize()
    ref.check(got, cache, starts, lens, pages, q, bits, 1 / np.sqrt(32))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("before", [0, 70])
def test_masks_of_any_kind(ctx, lib, dtype, before):
    """Masks that are no trees: empty ones, all bits (those beyond the new tokens included), only others than the token itself; with nothing before the new tokens, a row with an empty mask gets 0."""
    new, lens = [40, 3], [40 + before, 3 + before]
    starts, pages, cache, dev, q = case(lib, 2, 2, 64, new, lens, 16, 1, dtype, 8)
    rng = np.random.default_rng(1)
    bits = rng.random((43, 64)) < 0.3
    bits[5], bits[6], bits[41], bits[42] = False, True, False, True
    bits[7] = False
    bits[7, 39] = True
    for window in (0, 33):
        got = ctx.kv_cache_tree_attention(dev, lib.KVBatch(i32(starts), i32(lens), i32(pages)), q, ref.as_words(bits).cuda(), window=window)
        torch.cuda.synchronize()
        ref.check(got, cache, starts, lens, pages, q, bits, 1 / 8, window)
        if not before:
            assert (got[[5, 41]] == 0).all()


@pytest.mark.parametrize("new", [[3, 3, 3], [40, 33, 70]])
def test_pages_that_are_not_there(ctx, lib, new):
    """Pages outside the cache are invisible, the rest is not; places beyond the row of pages too; a shared page serves two sequences."""
    lens = [100, 90, 80]
    starts, pages, cache, dev, q, bits = drafted(lib, 1, 2, 64, new, lens, 16, 1, torch.float32, 21)
    pages = pages[:, :5].copy()      # 80 places
    pages[0, 1], pages[1, 0], pages[2, :] = -1, len(cache.data), [-5, 1 << 30, -1, -1, -1]
    pages[1, 3] = pages[0, 3]
    cache.kg[pages[1, 3]], cache.vg[pages[1, 3]] = [0.01, 120], [0.02, 130]
    dev = lib.KVCache(torch.tensor(cache.data).cuda(), 1, 64, 16, 1)
    got = ctx.kv_cache_tree_attention(dev, lib.KVBatch(i32(starts), i32(lens), i32(pages)), q, ref.as_words(bits).cuda())
    torch.cuda.synchronize()
    ref.check(got, cache, starts, lens, pages, q, bits, 1 / 8)
    assert (got[starts[2]:] == 0).all()


@pytest.mark.parametrize("new,rep", [(4, 2), (50, 2), (30, 8)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_values_that_are_special(ctx, lib, dtype, new, rep):
    """A NaN, infinite or huge scale of a drafted token's value reaches the rows that see it and no other; a NaN or infinite query its own row; scales far apart and queries of any size stay exact."""
    lens = [150, 150]
    starts, pages, cache, dev, q, bits = drafted(lib, 1, rep, 64, [new, new], lens, 16, 1, dtype, 5)
    at = lambda b, p: (pages[b, p // 16], 0, p % 16, 0)  # noqa: E731
    first, second = 150 - new + 1, 150 - new + 2
    bits[:2 * new, :3] = False      # new tokens 1 and 2: seen by one other row each
    bits[3, 1] = bits[new + 3, 2] = True
    cache.vg[at(0, first)] = np.nan
    cache.vg[at(1, first)] = np.inf
    cache.vg[at(0, second)] = 1e30
    cache.vg[at(1, second)] = 1e20
    cache.vg[pages[1, 2], 0, :, 0] *= 1e-6
    q[0] *= 1e-20
    q[-1, 1, 3] = float("inf")
    q[2, 0, 0] = float("nan")
    dev = lib.KVCache(torch.tensor(cache.data).cuda(), 1, 64, 16, 1)
    got = ctx.kv_cache_tree_attention(dev, lib.KVBatch(i32(starts), i32(lens), i32(pages)), q, ref.as_words(bits).cuda())
    torch.cuda.synchronize()
    ok = torch.ones(len(q), rep, dtype=torch.bool)
    ok[-1, 1] = ok[2, 0] = False
    assert torch.isnan(got[-1, 1]).all() and torch.isnan(got[2, 0]).all()
    q[-1, 1], q[2, 0] = 0, 0
    ref.check(got, cache, starts, lens, pages, q, bits, 1 / 8, rows=ok)


def test_strides_streams_and_offsets(ctx, lib):
    """Queries inside a fused projection, outputs inside a wider tensor, a context on a stream of its own, and pages beyond 2^32 bytes."""
    heads, rep, dh, pt, st = 8, 2, 128, 64, 1
    new, lens = [9, 2, 20], [70, 300, 150]
    starts, pages, cache, dev, q, bits = drafted(lib, heads, rep, dh, new, lens, pt, st, torch.bfloat16, 31)
    tree = ref.as_words(bits).cuda()
    base = ctx.kv_cache_tree_attention(dev, lib.KVBatch(i32(starts), i32(lens), i32(pages)), q, tree)
    torch.cuda.synchronize()
    ref.check(base, cache, starts, lens, pages, q, bits, 1 / np.sqrt(dh))
    for shift in (0, 1):      # aligned, and not
        wide = torch.randn(31 * (heads * (rep + 2) + 1) * dh + 4 * shift, device="cuda").bfloat16()[4 * shift:].view(31, heads * (rep + 2) + 1, dh)
        wide[:, 1:1 + heads * rep] = q
        out = torch.zeros(31, heads * rep + 5, dh, device="cuda", dtype=torch.bfloat16)
        ctx.kv_cache_tree_attention(dev, lib.KVBatch(i32(starts), i32(lens), i32(pages)), wide[:, 1:1 + heads * rep], tree, out=out[:, 2:2 + heads * rep])
        torch.cuda.synchronize()
        assert torch.equal(out[:, 2:2 + heads * rep], base) and (out[:, :2] == 0).all() and (out[:, 2 + heads * rep:] == 0).all()
    per = dev.data.shape[1]
    far = (1 << 32) // per + 50
    big = torch.zeros(far + len(cache.data), per, dtype=torch.uint8, device="cuda")
    big[far:] = dev.data
    side = torch.cuda.Stream()
    other = lib.Context(stream=side)
    try:
        side.wait_stream(torch.cuda.current_stream())
        got = other.kv_cache_tree_attention(lib.KVCache(big, heads, dh, pt, st), lib.KVBatch(i32(starts), i32(lens), i32(pages + far)), q, tree)
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        assert torch.equal(got, base)
    finally:
        other.close()


@pytest.mark.parametrize("new,lens", [([20, 7], [400, 90]), ([64], [1500])])
def test_captured_and_replayed(lib, new, lens):
    """A graph over fixed buffers, replayed with eager calls of the same context between the replays; a capture without room is refused, and the context goes on."""
    stream = torch.cuda.Stream()
    ctx = lib.Context(stream=stream)
    try:
        with torch.cuda.stream(stream):
            starts, pages, cache, dev, q, bits = drafted(lib, 2, 4, 128, new, lens, 16, 1, torch.bfloat16, 3)
            tree, batch, out = ref.as_words(bits).cuda(), lib.KVBatch(i32(starts), i32(lens), i32(pages)), torch.empty_like(q)
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=stream):
                with pytest.raises(lib.TurboBoAError) as e:
                    ctx.kv_cache_tree_attention(dev, batch, q, tree, out=out)
                assert e.value.code == -3
                out.zero_()
            ctx.reserve_workspace(ctx.kv_cache_tree_attention_workspace_bytes(dev, 8, len(new), len(q)))
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=stream):
                ctx.kv_cache_tree_attention(dev, batch, q, tree, out=out)
            for k in range(4):
                q.copy_(torch.randn(q.shape, generator=torch.Generator().manual_seed(k)).to(q.dtype))
                want = ctx.kv_cache_tree_attention(dev, batch, q, tree).clone()
                out.fill_(7)
                g.replay()
                stream.synchronize()
                assert torch.equal(out, want), k
                if k == 0:
                    ref.check(out, cache, starts, lens, pages, q, bits, 1 / np.sqrt(128))
                ctx.reserve_workspace(ctx.workspace_bytes() + (1 << 20))      # a growth leaves what the graph holds
    finally:
        ctx.close()


def test_refusals(ctx, lib):
    starts, pages, cache, dev, q = case(lib, 2, 2, 64, [2], [10], 16, 1, torch.bfloat16, 3)
    batch, tree = lib.KVBatch(i32(starts), i32([10]), i32(pages)), i32([[1], [3]])
    for bad in (dict(window=-1), dict(scale=-1.0), dict(scale=float("nan"))):
        with pytest.raises(lib.TurboBoAError) as e:
            ctx.kv_cache_tree_attention(dev, batch, q, tree, **bad)
        assert e.value.code == -1
    for args in ((dev, batch, q[:, :3], tree), (dev, lib.KVBatch(i32(starts), i32([10]), i32(pages[:, :0])), q, tree), (dev, lib.KVBatch(i32(starts), i32([10]), i32(pages), max_new=33), q, tree),
                 (dev, batch, q, torch.zeros(2, 1025, dtype=torch.int32, device="cuda")), (dev, batch, q, tree[:, :0].contiguous()), (dev, batch, q.double(), tree)):
        with pytest.raises(lib.TurboBoAError) as e:
            ctx.kv_cache_tree_attention(*args)
        assert e.value.code == -1
    for bad in (tree[:1], tree.long(), tree[:, 0], tree.cpu()):
        with pytest.raises(AssertionError):
            ctx.kv_cache_tree_attention(dev, batch, q, bad)
    assert ctx.kv_cache_tree_attention(dev, batch, q[:0], tree[:0]).shape == (0, 4, 64)


@pytest.mark.parametrize("heads,rep,new,lens", [(1, 2, [40, 33, 70], [100, 90, 80]), (2, 8, [30], [79]), (3, 4, [25, 2, 0], [90, 60, 30])])
def test_many_rows_whose_pages_are_not_there(ctx, lib, heads, rep, new, lens):
    """bf16 trees of more rows than one workgroup of the kernel for few rows takes: pages outside the cache, and places beyond the row of pages, are invisible; a sequence without pages gets 0."""
    starts, pages, cache, dev, q, bits = drafted(lib, heads, rep, 64, new, lens, 16, 1, torch.bfloat16, 22)
    pages = pages[:, :5].copy()      # 80 places
    pages[0, 1] = -1
    if len(new) > 1:
        pages[1, 0], pages[2, :] = len(cache.data), [-5, 1 << 30, -1, -1, -1]
    got = ctx.kv_cache_tree_attention(dev, lib.KVBatch(i32(starts), i32(lens), i32(pages)), q, ref.as_words(bits).cuda())
    torch.cuda.synchronize()
    ref.check(got, cache, starts, lens, pages, q, bits, 1 / 8)
    assert len(new) == 1 or (got[starts[2]:] == 0).all()


def test_many_rows_strides_streams_and_offsets(ctx, lib):
    """The same calls with queries inside a fused projection, outputs inside a wider tensor, a context on a stream of its own, pages beyond 2^32 bytes, and rows of no sequence left as they were."""
    heads, rep, dh, pt = 4, 4, 128, 64
    new, lens = [30, 2, 70], [470, 300, 3000]
    starts, pages, cache, dev, q, bits = drafted(lib, heads, rep, dh, new, lens, pt, 1, torch.bfloat16, 33, spare_rows=4)
    tree = ref.as_words(bits).cuda()
    base = ctx.kv_cache_tree_attention(dev, lib.KVBatch(i32(starts), i32(lens), i32(pages)), q, tree, out=torch.full_like(q, 7))
    torch.cuda.synchronize()
    ref.check(base, cache, starts, lens, pages, q, bits, 1 / np.sqrt(dh))
    assert (base[102:] == 7).all()
    for shift in (0, 1, 4):
        wide = torch.randn(106 * (heads * (rep + 2) + 1) * dh + shift, device="cuda").bfloat16()[shift:].view(106, heads * (rep + 2) + 1, dh)
        wide[:, 1:1 + heads * rep] = q
        out = torch.full((106 * (heads * rep + 5) * dh + shift,), 7.0, device="cuda", dtype=torch.bfloat16)[shift:].view(106, heads * rep + 5, dh)
        ctx.kv_cache_tree_attention(dev, lib.KVBatch(i32(starts), i32(lens), i32(pages)), wide[:, 1:1 + heads * rep], tree, out=out[:, 2:2 + heads * rep])
        torch.cuda.synchronize()
        assert torch.equal(out[:, 2:2 + heads * rep], base) and (out[:, :2] == 7).all() and (out[:, 2 + heads * rep:] == 7).all()
    per = dev.data.shape[1]
    far = (1 << 32) // per + 50
    big = torch.zeros(far + len(cache.data), per, dtype=torch.uint8, device="cuda")
    big[far:] = dev.data
    side = torch.cuda.Stream()
    other = lib.Context(stream=side)
    try:
        side.wait_stream(torch.cuda.current_stream())
        got = other.kv_cache_tree_attention(lib.KVCache(big, heads, dh, pt, 1), lib.KVBatch(i32(starts), i32(lens), i32(pages + far)), q, tree)
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        assert torch.equal(got[:102], base[:102])
    finally:
        other.close()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("max_new", [1, 3, 9, 17])
def test_sequences_of_more_new_tokens_than_told(ctx, lib, dtype, max_new):
    """max_new chooses between kernels only: sequences of more new tokens get the same, within the workspace that was made for fewer."""
    new, lens = [100, 3, 31, 0, 9], [900, 2000, 31, 50, 700]
    starts, pages, cache, dev, q, bits = drafted(lib, 2, 4, 64, new, lens, 64, 1, dtype, 17)
    got = ctx.kv_cache_tree_attention(dev, lib.KVBatch(i32(starts), i32(lens), i32(pages), max_new=max_new), q, ref.as_words(bits).cuda())
    torch.cuda.synchronize()
    ref.check(got, cache, starts, lens, pages, q, bits, 1 / 8)
