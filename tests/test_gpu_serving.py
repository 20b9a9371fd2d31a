"""The serving operators together, as they are used (GPU): an attention block with quantized weights and a quantized cache through prompts and single tokens, every stage against its 64-bit form on what
the stage before it gave; a captured step that is replayed; contexts, streams and graphs side by side."""
import numpy as np
import pytest
import torch

from paper_2602_04929_amd import pipeline, synth
from tests import serving_ref as ref
from tests import test_gpu_kv_cache_attention as attention
from tests.test_gpu_head_norm_rotate import close, table
from tests.test_gpu_kv_cache_append import i32, layout
from tests.test_gpu_kv_cache_attention import case, check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx(lib):
    c = lib.Context()
    yield c
    c.close()


def f64(t):
    return t.detach().double().cpu().numpy()


@pytest.mark.parametrize("name,norm,adjacent,st,window", [("tiny", False, False, 1, 0), ("tiny", True, True, 16, 20), ("llama2-7b", False, False, 16, 0), ("llama2-7b", True, False, 1, 0)])
def test_a_block_with_quantized_weights(ctx, lib, name, norm, adjacent, st, window):
    Hq, Hkv, dh, d = 4, 2, 64, 256
    cfg = synth.scaled(synth.CONFIGS[name], d_model=d, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=dh, n_seqs=2, seq_len=64, n_outlier=3)
    blk = synth.make_block(cfg, seed=7, device="cuda")
    out = pipeline.quantize_attention_block(ctx, blk, cfg, kv_bits=8)
    W = dict(Wqkv=torch.cat([out[n]["W_deq"] for n in "qkv"]), Wo=out["o"]["W_deq"])
    dtype = blk["X_fp"].dtype
    tab = table(300, dh)
    rotation = lib.Rotation(tab.cuda(), adjacent=adjacent)
    g = torch.Generator().manual_seed(3)
    nq, nk = ((1 + 0.3 * torch.randn(dh, generator=g)).cuda() for _ in "qk") if norm else (None, None)
    plan = [[40, 7], [1, 1], [1, 0], [1, 30], [1, 1]]
    total, pages = layout(np.sum(plan, 0), 16, 9)
    cache = lib.KVCache(torch.zeros(total, lib.KVCache.page_bytes(Hkv, dh, 16, st), dtype=torch.uint8, device="cuda"), Hkv, dh, 16, st)
    want = ref.Cache(cache.data.cpu().numpy(), Hkv, dh, 16, st)
    lens = np.zeros(2, int)
    half = torch.finfo(dtype).eps / 2
    for new in plan:
        lens = lens + new
        starts = np.concatenate([[0], np.cumsum(new)])
        place = np.concatenate([np.arange(l - n, l) for l, n in zip(lens, new)]).astype(int)
        X = torch.randn(starts[-1], d, generator=g).to(dtype).cuda()
        r = pipeline.serve_attention_block(ctx, W, X, cache, lib.KVBatch(i32(starts), i32(lens), i32(pages)), Hq, rotation=rotation, positions=i32(place), norm_q=nq, norm_k=nk,
                                           window=window, residual=X)
        torch.cuda.synchronize()
        # the projections, by themselves: half a step of the type, and 1e-5 (bf16 operands in several terms) or 1e-6 of the largest (see the tests of that entry point)
        qkv = ctx.linear_forward(X, W["Wqkv"]).view(-1, Hq + 2 * Hkv, dh)
        w64 = f64(X) @ f64(W["Wqkv"]).T
        assert (np.abs(f64(qkv).reshape(w64.shape) - w64) <= half * np.abs(w64) + (1e-6 if dtype == torch.float32 else 1e-5) * np.abs(w64).max()).all()
        q64, k64, v64 = f64(qkv[:, :Hq]), f64(qkv[:, Hq:Hq + Hkv]), f64(qkv[:, Hq + Hkv:])
        n64 = [None if n is None else f64(n) for n in (nq, nk)]
        close(r["q"], ref.norm_rotate(q64, n64[0], 1e-6, tab.numpy(), place, adjacent), q64, n64[0], tab.numpy(), place, adjacent, 1e-6)
        if norm:      # normalised and rotated before the append
            close(r["k"], ref.norm_rotate(k64, n64[1], 1e-6, tab.numpy(), place, adjacent), k64, n64[1], tab.numpy(), place, adjacent, 1e-6)
            keys = f64(r["k"])
        else:
            assert torch.equal(r["k"], qkv[:, Hq:Hq + Hkv])
            keys = ref.norm_rotate(k64, None, 0, tab.numpy(), place, adjacent)
        assert torch.equal(r["v"], qkv[:, Hq + Hkv:])
        ref.append(want, starts, lens, pages, keys, v64, starts[-1])
        assert np.array_equal(cache.data.cpu().numpy(), want.data)
        check(r["o"], want, starts, lens, pages, r["q"], 1 / np.sqrt(dh), window, dtype)
        y64 = f64(r["o"]).reshape(-1, Hq * dh) @ f64(W["Wo"]).T + f64(X)
        assert (np.abs(f64(r["Y"]) - y64) <= half * np.abs(y64) + (1e-6 if dtype == torch.float32 else 1e-5) * np.abs(y64).max()).all()


class Step:
    """One step of `new` tokens per sequence over fixed buffers, as a graph needs it: rotation, append, attention."""

    def __init__(self, lib, new, lens, pages, total, heads, rep, dh, pt, st, dtype, seed):
        self.lib, self.new, self.seed = lib, np.asarray(new), seed
        self.rows, self.geometry, self.dtype = int(self.new.sum()), (heads, dh, pt, st), dtype
        starts = np.concatenate([[0], np.cumsum(new)])
        self.qkv = torch.empty(self.rows, heads * (rep + 2), dh, dtype=dtype, device="cuda")
        self.q, self.k, self.v = self.qkv[:, :heads * rep], self.qkv[:, heads * rep:heads * (rep + 1)], self.qkv[:, heads * (rep + 1):]
        self.out, self.turned = (torch.empty(self.rows, heads * rep, dh, dtype=dtype, device="cuda") for _ in "oq")
        self.positions, self.lens, self.max_new = i32(np.zeros(self.rows)), i32(lens), int(max(new))
        self.starts, self.pages = i32(starts), i32(pages)
        self.data = torch.zeros(total, lib.KVCache.page_bytes(*self.geometry), dtype=torch.uint8, device="cuda")
        self.rotation = lib.Rotation(table(2000, dh).cuda())

    def fill(self, lens, seed):
        g = torch.Generator().manual_seed(seed)
        self.qkv.copy_(torch.randn(self.qkv.shape, generator=g).to(self.dtype))
        self.lens.copy_(i32(lens))
        self.positions.copy_(i32(np.concatenate([np.arange(n - m, n) for n, m in zip(lens, self.new)])))

    def run(self, ctx, data=None, out=None, turned=None):
        lib = self.lib
        cache = lib.KVCache(self.data if data is None else data, *self.geometry)
        batch = lib.KVBatch(self.starts, self.lens, self.pages, max_new=self.max_new)
        turned = self.turned if turned is None else turned
        ctx.head_norm_rotate(self.q, rotation=self.rotation, positions=self.positions, out_q=turned)
        ctx.kv_cache_append(cache, batch, self.k, self.v, rotation=self.rotation)
        return ctx.kv_cache_attention(cache, batch, turned, out=self.out if out is None else out)

    def need(self, ctx):
        heads = self.geometry[0]
        return ctx.kv_cache_attention_workspace_bytes(self.lib.KVCache(self.data, *self.geometry), self.q.shape[1], len(self.new), self.rows)


def captured(lib, step, ctx, stream):
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        step.run(ctx)
    return graph


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("st", [1, 16])
def test_steps_replayed_from_graphs(ctx, lib, dtype, st):
    """Two graphs of one context, of single tokens and of prompts, replayed in turn as the sequences grow, with eager work of another context and synchronizations between, and after the context's
    workspace has grown: every replay gives the bits of the eager calls."""
    heads, rep, dh, pt = 2, 4, 128, 64
    lens = np.array([5, 300, 64, 0])
    total, pages = layout(lens + 400, pt, 4)
    stream = torch.cuda.Stream()
    own = lib.Context(stream=stream)
    try:
        one = Step(lib, [1, 1, 1, 1], lens, pages, total, heads, rep, dh, pt, st, dtype, 1)
        many = Step(lib, [40, 3, 17, 60], lens, pages, total, heads, rep, dh, pt, st, dtype, 2)
        many.data = one.data
        with pytest.raises(lib.TurboBoAError) as e:      # nothing reserved yet
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=stream):
                many.out.zero_()
                many.run(own)
        assert e.value.code == -3 and "captured" in str(e.value)
        own.reserve_workspace(max(one.need(own), many.need(own)))
        shadow = one.data.clone()
        graphs = [(one, captured(lib, one, own, stream)), (many, captured(lib, many, own, stream))]
        held = own.workspace_bytes()
        for turn, which in enumerate([0, 0, 1, 0, 1, 1, 0, 0]):
            step, graph = graphs[which]
            lens = lens + step.new
            step.fill(lens, 10 * turn)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            got, cache = step.out.clone(), one.data.clone()
            want = step.run(ctx, data=shadow, out=torch.empty_like(step.out), turned=torch.empty_like(step.turned))
            torch.cuda.synchronize()
            assert torch.equal(cache, shadow), turn
            assert torch.equal(got, want) and torch.isfinite(got).all(), turn
            if turn == 3:      # the graphs keep the workspace that they were captured with
                own.reserve_workspace(held + (64 << 20))
                filler = torch.full((held,), 255, dtype=torch.uint8, device="cuda")
                assert own.workspace_bytes() > held and filler[0] == 255
            if turn == 5:      # eager calls of the graphs' own context, on its stream, between replays
                with torch.cuda.stream(stream):
                    other = step.run(own, data=shadow, out=torch.empty_like(step.out), turned=torch.empty_like(step.turned))
                torch.cuda.synchronize()
                assert torch.equal(other, want)
    finally:
        own.close()


def test_contexts_side_by_side(ctx, lib):
    """Two contexts on two streams at once, each with a cache of its own, and tensors that were allocated on a third: the bits of one after the other."""
    lens = np.array([70, 129])
    total, pages = layout(lens, 64, 3)
    ctxs = [lib.Context(stream=torch.cuda.Stream()) for _ in range(2)]
    try:
        steps = [Step(lib, [70, 129], lens, pages, total, 2, 2, 96, 64, 4, torch.bfloat16, s) for s in range(2)]
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


@pytest.mark.parametrize("new", [[4, 3, 1], [50, 3, 1]])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_windows_longer_than_any_sequence(ctx, lib, dtype, new):
    """Also for tokens that have no place, before the sequence's first one."""
    lens = [2, 3, 1]
    starts, pages, cache, dev, q = case(lib, 2, 2, 64, new, lens, 16, 1, dtype, 77)
    batch = lib.KVBatch(i32(starts), i32(lens), i32(pages))
    base = ctx.kv_cache_attention(dev, batch, q)
    for window in (1 << 30, (1 << 31) - 1, (1 << 30) - 1, 3):
        assert torch.equal(ctx.kv_cache_attention(dev, batch, q, window=window), base), window
    check(base, cache, starts, lens, pages, q, 1 / 8, 0, dtype)


@pytest.fixture
def wide_tables(monkeypatch):
    """Rows of pages for 2^22 tokens, of which the sequences have few: by what the host knows these are long calls, and prompts of 16-bit inputs take the kernel for many rows."""
    def wide(lens, pt, seed, *args):
        total, pages = layout(lens, pt, seed, *args)
        return total, np.pad(pages, ((0, 0), (0, (1 << 22) // pt - pages.shape[1])), constant_values=-1)
    monkeypatch.setattr(attention, "layout", wide)


@pytest.mark.parametrize("shape", [s for s in attention.SHAPES if max(s[3]) * s[1] > 32 and not s[5]], ids=lambda s: "-".join(str(x).replace(" ", "") for x in s))
def test_few_rows_in_wide_tables(ctx, lib, wide_tables, shape):
    attention.test_ragged_batches(ctx, lib, torch.bfloat16, shape)


def test_special_cases_in_wide_tables(ctx, lib, wide_tables):
    attention.test_values_that_are_special(ctx, lib, torch.bfloat16, 50)
    for kind in ("nothing", "least", "small", "mixed", "late"):
        test_scales_of_any_size(ctx, lib, torch.bfloat16, 50, kind)
    test_windows_longer_than_any_sequence(ctx, lib, torch.bfloat16, [50, 3, 1])


@pytest.mark.parametrize("pt", [16, 64])
def test_holes_in_wide_tables(ctx, lib, wide_tables, pt):
    """Pages outside the cache, the first and the last one of a sequence among them, and one sequence that has none."""
    new, lens = [40, 33, 70, 20], [300, 290, 80, 64]
    starts, pages, cache, dev, q = case(lib, 2, 2, 64, new, lens, pt, 1, torch.bfloat16, 22)
    pages[0, 1], pages[1, 0], pages[1, 289 // pt], pages[2, :] = -1, len(cache.data), 1 << 30, -7
    got = ctx.kv_cache_attention(dev, lib.KVBatch(i32(starts), i32(lens), i32(pages)), q)
    torch.cuda.synchronize()
    check(got, cache, starts, lens, pages, q, 1 / 8, 0, torch.bfloat16)
    assert (got[starts[2]:starts[3]] == 0).all()


@pytest.mark.parametrize("heads,rep,dh,window,pt,st", [(12, 8, 128, 100, 64, 1), (6, 8, 256, 33, 16, 16), (20, 8, 64, 1, 128, 4), (13, 8, 90, 257, 32, 32), (25, 6, 32, 64, 64, 1)])
def test_windows_of_many_rows(ctx, lib, heads, rep, dh, window, pt, st):
    """Windows that cut tiles at their lower end, so many rows that the kernel for many takes them."""
    new, lens = [200, 90, 3], [400, 91, 500]
    starts, pages, cache, dev, q = case(lib, heads, rep, dh, new, lens, pt, st, torch.bfloat16, 13, spare_rows=2)
    batch = lib.KVBatch(i32(starts), i32(lens), i32(pages))
    out = torch.full_like(q, 7)
    ctx.kv_cache_attention(dev, batch, q, window=window, out=out)
    torch.cuda.synchronize()
    check(out, cache, starts, lens, pages, q, 1 / np.sqrt(dh), window, torch.bfloat16)
    assert (out[starts[-1]:] == 7).all()
    shifted(ctx, dev, batch, q, out, window=window)


def shifted(ctx, cache, batch, q, out, **kw):
    """Queries and outputs that are not aligned to 16 bytes, or to 8: the same values."""
    for shift in (4, 1):
        odd, moved = (torch.full((q.numel() + 8,), 7, dtype=q.dtype, device="cuda") for _ in "oq")
        view, query = (x[shift:shift + q.numel()].view(q.shape) for x in (odd, moved))
        query.copy_(q)
        for a in (q, query):
            view.fill_(7)
            ctx.kv_cache_attention(cache, batch, a, out=view, **kw)
            torch.cuda.synchronize()
            assert torch.equal(view, out) and (odd[:shift] == 7).all() and (odd[shift + q.numel():] == 7).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("dh", [128, 100, 33])
def test_unaligned_rows(ctx, lib, dtype, dh):
    new, lens = [3, 1, 0, 9], [200, 90, 4, 2000]
    starts, pages, cache, dev, q = case(lib, 2, 2, dh, new, lens, 16, 4, dtype, 14, spare_rows=1)
    batch = lib.KVBatch(i32(starts), i32(lens), i32(pages))
    out = torch.full_like(q, 7)
    ctx.kv_cache_attention(dev, batch, q, out=out)
    torch.cuda.synchronize()
    check(out, cache, starts, lens, pages, q, 1 / np.sqrt(dh), 0, dtype)
    shifted(ctx, dev, batch, q, out)


@pytest.mark.parametrize("new", [1, 50])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kind", ["nothing", "least", "small", "mixed", "late"])
def test_scales_of_any_size(ctx, lib, dtype, new, kind):
    """Scales of 0 (pages that were cleared and never written), the least that an append gives, and both beside ordinary ones."""
    lens, dh = [200, 70], 64
    starts, pages, cache, dev, q = case(lib, 2, 2, dh, [new, 1], lens, 64, 1, dtype, 21)
    rng = np.random.default_rng(5)
    g = cache.vg[..., 0]
    seen = np.isfinite(g)
    g[seen] = {"nothing": 0.0, "least": 2.0 ** -126, "small": 2.0 ** -118 * (1 + rng.random(g.shape)[seen]), "mixed": rng.choice([0.0, 2.0 ** -126, 2.0 ** -60, 0.01], g.shape)[seen], "late": 0.0}[kind]
    if kind == "late":      # all tiles but each sequence's last one
        for b, n in enumerate(lens):
            g[pages[b, (n - 1) // 64], :, (n - 1) % 64] = 0.01
    got = ctx.kv_cache_attention(lib.KVCache(torch.tensor(cache.data).cuda(), 2, dh, 64, 1), lib.KVBatch(i32(starts), i32(lens), i32(pages)), q)
    check(got, cache, starts, lens, pages, q, 1 / 8, 0, dtype)


@pytest.mark.parametrize("heads,dh,st,new", [(9, 64, 1, 4101), (33, 64, 16, 2050), (13, 128, 16, 2050), (33, 128, 64, 1030), (18, 256, 64, 1030), (34, 32, 8, 2050)])
def test_prompts_that_fill_the_chip(ctx, lib, heads, dh, st, new):
    """So many blocks that a wavefront goes through several heads, whose number is no multiple of anything; the prompt begins inside a block whose grid has to grow."""
    had = st // 2
    total, pages = layout([had + new], 64, 6)
    cache = lib.KVCache(torch.zeros(total, lib.KVCache.page_bytes(heads, dh, 64, st), dtype=torch.uint8, device="cuda"), heads, dh, 64, st)
    want = ref.Cache(cache.data.cpu().numpy(), heads, dh, 64, st)
    g = torch.Generator().manual_seed(heads)
    tab = table(had + new, dh)
    for size, a, e in ((0.1, 0, had), (1.0, had, had + new)):
        if a == e:
            continue
        k, v = ((size * torch.randn(e - a, heads, dh, generator=g)).bfloat16() for _ in "kv")
        ctx.kv_cache_append(cache, lib.KVBatch(i32([0, e - a]), i32([e]), i32(pages)), k.cuda(), v.cuda(), rotation=lib.Rotation(tab.cuda()))
        torch.cuda.synchronize()
        x = f64(k).reshape(e - a, heads, 2, dh // 2)
        c, s = (np.asarray(tab[a:e], np.float64).reshape(e - a, 1, 2, dh // 2)[:, :, i] for i in range(2))
        turned = np.stack([x[:, :, 0] * c - x[:, :, 1] * s, x[:, :, 1] * c + x[:, :, 0] * s], 2).reshape(e - a, heads, dh)
        ref.append(want, [0, e - a], [e], pages, turned, f64(v), e - a)
        got = cache.data.cpu().numpy()
        assert np.array_equal(got, want.data), np.argwhere(got != want.data)[:5]


def test_refusals_of_the_append(ctx, lib):
    cache = lib.KVCache.empty(3, 2, 64, 16, 1)
    x = torch.zeros(2, 2, 64, device="cuda")
    batch = lib.KVBatch(i32([0, 2]), i32([2]), i32([[0]]))
    before = cache.data.clone()
    for rotation in (lib.Rotation(table(4, 66).cuda()), lib.Rotation(torch.zeros(4, 5, device="cuda")), lib.Rotation(torch.zeros(0, 64, device="cuda"))):
        with pytest.raises(lib.TurboBoAError) as e:
            ctx.kv_cache_append(cache, batch, x, x, rotation=rotation)
        assert e.value.code == -1 and "kv_cache_append" in str(e.value)
    with pytest.raises(lib.TurboBoAError):
        ctx.kv_cache_append(cache, batch, x.double(), x.double())
    with pytest.raises(lib.TurboBoAError):
        ctx.kv_cache_append(cache, lib.KVBatch(i32([0, 2]), i32([2]), torch.zeros(1, (1 << 26) + 1, dtype=torch.int32, device="cuda")), x, x)      # more than 2^30 tokens
    ctx.kv_cache_append(cache, batch, x[:0], x[:0])
    ctx.kv_cache_append(cache, lib.KVBatch(i32([0]), i32([]), i32(np.zeros((0, 1)))), x, x)
    ctx.kv_cache_append(lib.KVCache.empty(0, 2, 64, 16, 1), batch, x, x)
    torch.cuda.synchronize()
    assert torch.equal(cache.data, before)
    with pytest.raises(lib.TurboBoAError):
        ctx.kv_cache_attention(lib.KVCache.empty(0, 2, 64, 16, 1), batch, x)
