"""Packed weights and drafted trees as they are used together (GPU): a quantized block and its MLP through a prompt, drafted trees, the tokens of them that are accepted and single tokens; every stage
against its 64-bit form on what the stage before it gave; and a step of drafted trees captured and replayed."""
import numpy as np
import pytest
import torch

from paper_2602_04929_amd import pipeline, synth
from tests import packed_ref, serving_ref, tree_ref
from tests.test_gpu_head_norm_rotate import table
from tests.test_gpu_kv_cache_append import i32, layout
from tests.test_gpu_kv_cache_attention import check as check_chain
from tests.test_gpu_kv_cache_tree_attention import grown
from tests.test_gpu_packed_linear import silu, swiglu_bound

pytestmark = pytest.mark.gpu
HQ, HKV, DH, D, FF, PT = 4, 2, 64, 256, 384, 16


@pytest.fixture(scope="module")
def ctx(lib):
    c = lib.Context()
    yield c
    c.close()


def exact(layers, group):
    """The dequantized matrix of packed layers, one below the other, in 64 bits."""
    def of(l):
        c = l["codes"].double()
        n = c.shape[1] // (group or c.shape[1])
        return ((c.view(len(c), n, -1) - l["zeros"].double().view(len(c), n, 1)) * l["scales"].double().view(len(c), n, 1)).view(c.shape)
    return torch.cat([of(l) for l in layers])


def linear(got, x, w, packed, residual=None):
    want, lim = x.double() @ w.T, packed_ref.bound(x, w, packed)
    if residual is not None:
        lim = lim + 2.0 ** -24 * (want.abs() + residual.double().abs())
        want = want + residual.double()
    packed_ref.check(got, want, lim, telling=0.7)


def quantized(ctx, name, bits, group):
    cfg = synth.scaled(synth.CONFIGS[name], d_model=D, n_q_heads=HQ, n_kv_heads=HKV, head_dim=DH, n_seqs=2, seq_len=64, n_outlier=3, bits=bits, group=group, d_ff=FF)
    blk, mlp = synth.make_block(cfg, seed=7, device="cuda"), synth.make_mlp(cfg, seed=8, device="cuda")
    return pipeline.quantize_attention_block(ctx, blk, cfg, kv_bits=8), pipeline.quantize_mlp(ctx, mlp, cfg), blk["X_fp"].dtype


@pytest.mark.parametrize("name,bits,group,norm,window", [("tiny", 4, 64, False, 0), ("llama2-7b", 4, 128, True, 0), ("llama2-7b", 2, 0, False, 30), ("llama2-7b", 3, 64, True, 0)])
def test_prompt_drafts_and_accepted_tokens(ctx, lib, name, bits, group, norm, window):
    att, mlp, dtype = quantized(ctx, name, bits, group)
    W, M = pipeline.pack_attention_block(ctx, att, bits, group), pipeline.pack_mlp(ctx, mlp, bits, group)
    wqkv, wo = exact([att[n] for n in "qkv"], group), exact([att["o"]], group)
    wg, wu, wd = (exact([mlp[n]], group) for n in ("gate", "up", "down"))
    rotation = lib.Rotation(table(300, DH).cuda())
    g = torch.Generator().manual_seed(3)
    nq, nk = ((1 + 0.3 * torch.randn(DH, generator=g)).cuda() for _ in "qk") if norm else (None, None)
    total, pages = layout(np.array([160, 120]), PT, 9)
    fresh = lambda: lib.KVCache(torch.zeros(total, lib.KVCache.page_bytes(HKV, DH, PT, 1), dtype=torch.uint8, device="cuda"), HKV, DH, PT, 1)
    cache, chain = fresh(), fresh()      # chain: what accepted tokens alone leave
    lens = np.zeros(2, int)

    def step(new, tree=None, depth=None):
        starts = np.concatenate([[0], np.cumsum(new)])
        place = np.concatenate([np.arange(l, l + n) for l, n in zip(lens, new)]) if depth is None else np.repeat(lens, new) + depth
        batch = lib.KVBatch(i32(starts), i32(lens + new), i32(pages))
        X = torch.randn(starts[-1], D, generator=g).to(dtype).cuda()
        r = pipeline.serve_attention_block(ctx, W, X, cache, batch, HQ, rotation=rotation, positions=i32(place), norm_q=nq, norm_k=nk, window=window, residual=X, tree=tree)
        m = pipeline.serve_mlp(ctx, M, r["Y"], residual=r["Y"])
        torch.cuda.synchronize()
        # q and k are turned in place: the projections once more
        qkv = ctx.packed_linear(W["Wqkv"], X)
        linear(qkv, X, wqkv, W["Wqkv"])
        turned = qkv.view(-1, HQ + 2 * HKV, DH).clone()
        assert torch.equal(r["v"], turned[:, HQ + HKV:])
        ctx.head_norm_rotate(turned[:, :HQ], turned[:, HQ:HQ + HKV] if norm else None, nq, nk, 1e-6, rotation, i32(place), out_q=turned[:, :HQ], out_k=turned[:, HQ:HQ + HKV] if norm else None)
        assert torch.equal(r["q"], turned[:, :HQ]) and torch.equal(r["k"], turned[:, HQ:HQ + HKV])
        held = serving_ref.Cache(cache.data.cpu().numpy(), HKV, DH, PT, 1)
        if tree is None:
            check_chain(r["o"], held, starts, lens + new, pages, r["q"], 1 / np.sqrt(DH), window, dtype)
        else:
            seen = np.array([[bool(int(w) >> i & 1) for w in row for i in range(32)] for row in tree.cpu().numpy().view(np.uint32)])
            tree_ref.check(r["o"], held, starts, lens + new, pages, r["q"], seen, 1 / np.sqrt(DH), window)
        o = r["o"].view(-1, HQ * DH)
        linear(r["Y"], o, wo, W["Wo"], X)
        y, act = r["Y"], m["act"]
        gate, up = y.double() @ wg.T, y.double() @ wu.T
        packed_ref.check(act, silu(gate) * up, swiglu_bound(gate, up, packed_ref.bound(y, wg, M["Wg"]), packed_ref.bound(y, wu, M["Wu"])), telling=0.2)
        linear(m["Y"], act, wd, M["Wd"], y)
        return r, place

    def append(into, k, v, new, place):
        batch = lib.KVBatch(i32(np.concatenate([[0], np.cumsum(new)])), i32(lens + new), i32(pages))
        ctx.kv_cache_append(into, batch, k, v, *(() if norm else (rotation, i32(place))))

    for new, drafts in (([70, 9], [12, 40]), ([1, 1], [9, 1]), ([1, 3], [0, 33])):
        r, place = step(np.array(new))
        append(chain, r["k"], r["v"], np.array(new), place)
        lens = lens + new
        parents = grown(drafts, sum(drafts))
        tree, depth = lib.tree_masks(parents, drafts)
        r, place = step(np.array(drafts), tree.cuda(), depth.numpy())
        # the ancestors of the last drafted token are accepted
        keep, at = [], 0
        for n in drafts:
            path, t = [], n - 1
            while t >= 0:
                path.append(at + t)
                t = parents[at + t]
            keep.append(path[::-1])
            at += n
        rows = torch.tensor(sum(keep, []), device="cuda")
        count = np.array([len(p) for p in keep])
        k, v, where = r["k"][rows].contiguous(), r["v"][rows].contiguous(), place[rows.cpu().numpy()]
        assert np.array_equal(where, np.concatenate([np.arange(l, l + n) for l, n in zip(lens, count)]))
        append(cache, k, v, count, where)
        append(chain, k, v, count, where)
        lens = lens + count
    torch.cuda.synchronize()
    # what the sequences hold is what their accepted tokens alone would have left
    a, b = (serving_ref.Cache(c.data.cpu().numpy(), HKV, DH, PT, 1) for c in (cache, chain))
    for s, n in enumerate(lens):
        p = np.arange(n)
        page, off = pages[s][p // PT], p % PT
        for x in ("k", "kg", "vg"):
            assert np.array_equal(getattr(a, x)[page, :, off], getattr(b, x)[page, :, off])
        assert np.array_equal(a.v[page, :, off // 16, :, off % 16], b.v[page, :, off // 16, :, off % 16])


def test_steps_of_drafted_trees_replayed(ctx, lib):
    """A block and its MLP over drafted trees in a graph, replayed on new tokens, masks and lengths with eager work and synchronizations between: the bits of the eager calls."""
    bits, group = 4, 128
    att, mlp, dtype = quantized(ctx, "llama2-7b", bits, group)
    W, M = pipeline.pack_attention_block(ctx, att, bits, group), pipeline.pack_mlp(ctx, mlp, bits, group)
    rotation = lib.Rotation(table(700, DH).cuda())
    new = np.array([40, 7, 0, 25])
    rows, starts = int(new.sum()), np.concatenate([[0], np.cumsum(new)])
    total, pages = layout(np.full(4, 600), PT, 5)
    g = torch.Generator().manual_seed(5)
    # levels of any value with grids of a usual size
    cache = lib.KVCache(torch.zeros(total, lib.KVCache.page_bytes(HKV, DH, PT, 1), dtype=torch.uint8, device="cuda"), HKV, DH, PT, 1)
    full = lib.KVBatch(i32([0, 600, 1200, 1800, 2400]), i32([600] * 4), i32(pages))
    ctx.kv_cache_append(cache, full, *(torch.randn(2400, HKV, DH, generator=g).to(dtype).cuda() for _ in "kv"))
    shadow = lib.KVCache(cache.data.clone(), HKV, DH, PT, 1)
    X = torch.zeros(rows, D, dtype=dtype, device="cuda")
    tree, positions, lens = (torch.zeros(*s, dtype=torch.int32, device="cuda") for s in ((rows, 2), (rows,), (4,)))
    batch = lib.KVBatch(i32(starts), lens, i32(pages), max_new=int(new.max()))

    def run(c, cache):
        r = pipeline.serve_attention_block(c, W, X, cache, batch, HQ, rotation=rotation, positions=positions, residual=X, tree=tree)
        return pipeline.serve_mlp(c, M, r["Y"], residual=r["Y"])["Y"]

    stream = torch.cuda.Stream()
    own = lib.Context(stream=stream)
    try:
        own.reserve_workspace(max([own.kv_cache_tree_attention_workspace_bytes(cache, HQ, 4, rows)] + [own.packed_workspace_bytes(w, rows, dtype) for w in (*W.values(), *M.values())]))
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            out = run(own, cache)
        for turn in range(5):
            have = np.array([200 + 60 * turn, 3 * turn, 11, 500 - turn])
            words, depth = lib.tree_masks(grown(new, turn), new, words=2)
            X.copy_(torch.randn(rows, D, generator=g).to(dtype))
            tree.copy_(words)
            positions.copy_(i32(np.repeat(have, new) + depth.numpy()))
            lens.copy_(i32(have + new))
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            got = out.clone()
            want = run(ctx, shadow)
            torch.cuda.synchronize()
            assert torch.equal(cache.data, shadow.data), turn
            assert torch.equal(got, want) and torch.isfinite(got).all(), turn
    finally:
        own.close()
