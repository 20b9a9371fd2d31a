"""What the entry points for packed weights and drafted trees refuse before a device is touched, their descriptors and their host arithmetic (CPU)."""
import ctypes
import os
import re

import numpy as np
import pytest
import torch

import paper_2602_04929_amd as tb
from tests import tree_ref

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "turboboa.h")


def test_descriptor_matches_the_header():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    fields = []
    for decl in re.search(r"typedef struct \{([^}]*)\} tboa_packed_weight;", text).group(1).split(";"):
        if decl.strip():
            ctype, rest = re.match(r"\s*(?:const )?(\w+)\s*(.*)", decl.strip(), flags=re.S).groups()
            fields += [(n.strip(" *"), "pointer" if "*" in n else ctype) for n in rest.split(",")]
    cls = tb.binding.PackedWeightDesc
    assert [(n, {"c_int": "int", "c_void_p": "pointer"}[t.__name__]) for n, t in cls._fields_] == fields
    assert ctypes.sizeof(cls) == 40


def test_null_context_is_rejected():
    lib, w = tb.binding._lib, ctypes.byref(tb.binding.PackedWeightDesc(1, 32, 4, 0, None, None, None))
    d, b = ctypes.byref(tb.binding.KVCacheDesc(1, 64, 16, 1, 1)), ctypes.byref(tb.binding.KVBatchDesc(1, 1, 1, None, None, None, 0))
    assert lib.tboa_packed_linear(None, w, 1, 0, None, 32, None, 0, None, 1) == -1
    assert lib.tboa_packed_swiglu(None, w, w, 1, 0, None, 32, None, 1) == -1
    assert lib.tboa_kv_cache_tree_attention(None, d, b, 1, 0, None, 64, None, 1, None, 0.0, 0, None, 64) == -1


def test_workspaces_are_host_arithmetic():
    q = tb.binding._lib.tboa_kv_cache_tree_attention_workspace_bytes
    desc = tb.binding.KVCacheDesc(8, 128, 64, 1, 1000)
    one, many = (q(ctypes.byref(desc), 64, s, n) for s, n in ((1, 1), (16, 512)))
    assert 0 < one <= many < 1 << 30
    for heads, seqs, tokens in ((63, 1, 1), (0, 1, 1), (64, -1, 1), (64, 1, -1), (64, 1, 1 << 25), (64, (1 << 20) + 1, 1)):
        assert q(ctypes.byref(desc), heads, seqs, tokens) == 0
    assert q(None, 64, 1, 1) == 0 and q(ctypes.byref(desc), 64, 0, 5) == 0
    p = tb.binding._lib.tboa_packed_workspace_bytes
    for bad in ((0, 64, 4, 0), (64, 0, 4, 0), (64, 64, 5, 0), (64, 64, 4, 48), (64, 64, 4, -1), ((1 << 24) + 1, 64, 4, 0)):
        assert p(ctypes.byref(tb.binding.PackedWeightDesc(*bad, None, None, None)), 100, 1) == 0
    good = tb.binding.PackedWeightDesc(4096, 4096, 4, 128, None, None, None)
    assert p(None, 1, 1) == 0 and p(ctypes.byref(good), -1, 1) == 0 and p(ctypes.byref(good), 1, 7) == 0
    assert all(p(ctypes.byref(good), n, t) < 1 << 30 for n in (1, 17, 64, 65, 1000, 4096) for t in (0, 1))


class Reached(Exception):
    pass


@pytest.fixture
def ctx(monkeypatch):
    real = tb.binding._lib

    class Stub:
        tboa_kv_cache_page_bytes, tboa_packed_words_per_row = real.tboa_kv_cache_page_bytes, real.tboa_packed_words_per_row

        def __getattr__(self, name):
            def reached(*args):
                raise Reached
            return reached

    def dev(t, dtype=None):      # the binding's checks but for the device
        assert t.is_contiguous() and (dtype is None or t.dtype == dtype)
        return t

    class OnDevice(torch.Tensor):
        is_cuda = True
    monkeypatch.setattr(tb.binding, "_lib", Stub())
    monkeypatch.setattr(tb.binding, "_dev", dev)
    c = object.__new__(tb.Context)
    c._h = None
    c._used = lambda *tensors: None
    c.rows = lambda *shape, dtype=torch.float32: torch.zeros(*shape, dtype=dtype).as_subclass(OnDevice)
    return c


def weight(d_out=20, d_in=100, bits=3, group=0):
    z = torch.zeros
    return tb.PackedWeight(z(d_out, (d_in * bits + 31) // 32, dtype=torch.int32), z(d_out, d_in // group if group else 1), z(d_out, d_in // group if group else 1), d_in, bits, group)


def test_weights(ctx):
    weight(), weight(group=25), weight(bits=8)
    z = torch.zeros
    tb.PackedWeight(z(20, 10, dtype=torch.int32), z(20), z(20), 100, 3)
    for args in ((z(20, 9, dtype=torch.int32), z(20, 1), z(20, 1), 100, 3), (z(20, 10), z(20, 1), z(20, 1), 100, 3), (z(20, 10, dtype=torch.int32), z(20, 1), z(20, 2), 100, 3),
                 (z(20, 10, dtype=torch.int32), z(20, 4), z(20, 4), 100, 3, 30), (z(20, 10, dtype=torch.int32), z(20, 4), z(20, 4), 100, 3, 20), (z(20, 10, dtype=torch.int32), z(20, 1), z(20, 1), 100, 5),
                 (z(20, 10, dtype=torch.int32), z(20, 1).double(), z(20, 1), 100, 3), (z(10, 20, dtype=torch.int32).t(), z(20, 1), z(20, 1), 100, 3), (z(0, 10, dtype=torch.int32), z(0, 1), z(0, 1), 100, 3),
                 (z(20, 10, dtype=torch.int32), z(20, 1), z(20, 1), 100, 3, -1)):
        with pytest.raises(AssertionError):
            tb.PackedWeight(*args)


def test_arguments_of_the_products(ctx):
    w, x, y = weight(), ctx.rows(3, 100), ctx.rows(3, 20)
    for kw in (dict(out=y), dict(out=y, residual=y), dict(out=ctx.rows(3, 50)[:, 5:25]), dict(X=ctx.rows(3, 200)[:, 50:150], out=y), dict(X=ctx.rows(2, 3, 100), out=ctx.rows(2, 3, 20)),
               dict(X=ctx.rows(2, 3, 160)[..., :100], out=ctx.rows(2, 3, 20))):
        with pytest.raises(Reached):
            ctx.packed_linear(w, **dict(dict(X=x), **kw))
    for kw in (dict(X=ctx.rows(3, 99)), dict(out=ctx.rows(3, 21)), dict(out=ctx.rows(2, 20)), dict(residual=ctx.rows(3, 21)), dict(residual=ctx.rows(3, 20, dtype=torch.bfloat16)),
               dict(out=ctx.rows(3, 20, dtype=torch.bfloat16)), dict(X=ctx.rows(3, 200)[:, ::2]), dict(X=ctx.rows(4, 3, 100)[:, :2], out=ctx.rows(4, 2, 20)), dict(X=ctx.rows(100, 3).t())):
        with pytest.raises(AssertionError):
            ctx.packed_linear(w, **dict(dict(X=x, out=y), **kw))
    with pytest.raises(Reached):
        ctx.packed_swiglu(w, weight(), x, out=y)


def test_arguments_of_a_tree(ctx):
    cache = tb.KVCache(torch.zeros(5, tb.KVCache.page_bytes(2, 64, 16, 1), dtype=torch.uint8), 2, 64, 16, 1)
    z = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    batch, q = tb.KVBatch(z(3), z(2), z(2, 3)), ctx.rows(3, 4, 64)
    for tree in (z(3, 1), z(3, 4)):
        with pytest.raises(Reached):
            ctx.kv_cache_tree_attention(cache, batch, q, tree, out=ctx.rows(3, 4, 64))
    for args in ((q, z(2, 1)), (q, z(3)), (q, z(3, 1).long()), (q, z(2, 3).t()), (ctx.rows(3, 4, 32), z(3, 1))):
        with pytest.raises(AssertionError):
            ctx.kv_cache_tree_attention(cache, batch, *args, out=ctx.rows(3, 4, 64))


def test_masks_from_parents():
    rng = np.random.default_rng(0)
    counts = [70, 0, 1, 33]
    parents = [int(rng.integers(-1, i)) if i else -1 for n in counts for i in range(n)]
    tree, depth = tb.tree_masks(parents, counts)
    bits = tree_ref.masks(parents, counts, 3)
    assert torch.equal(tree, tree_ref.as_words(bits)) and np.array_equal(depth.numpy(), bits.sum(1) - 1)
    assert tb.tree_masks([-1], [1], words=4)[0].tolist() == [[1, 0, 0, 0]] and tb.tree_masks([], [0])[0].shape == (0, 1)
    for bad in (([0], [1]), ([-1, -2], [2]), ([-1, 1], [2]), ([-1], [2]), ([-1, -1], [1])):
        with pytest.raises((AssertionError, IndexError)):
            tb.tree_masks(*bad)
