"""What the serving entry points refuse before a device is touched, their descriptors and their host arithmetic (CPU)."""
import ctypes
import os
import re

import pytest
import torch

import paper_2602_04929_amd as tb
from tests import serving_ref as ref

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "turboboa.h")


def test_descriptors_match_the_header():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = {"c_int": "int", "c_long": "int64_t", "c_longlong": "int64_t", "c_void_p": "pointer"}
    for cname, cls in (("tboa_kv_cache_desc", tb.binding.KVCacheDesc), ("tboa_kv_batch", tb.binding.KVBatchDesc), ("tboa_rotation", tb.binding.RotationDesc)):
        fields = []
        for decl in re.search(r"typedef struct \{([^}]*)\} %s;" % cname, text).group(1).split(";"):
            if decl.strip():
                ctype, rest = re.match(r"\s*(?:const )?(\w+)\s*(.*)", decl.strip(), flags=re.S).groups()
                fields += [(n.strip(" *"), "pointer" if "*" in n else ctype) for n in rest.split(",")]
        assert [(n, names[t.__name__]) for n, t in cls._fields_] == fields
        assert ctypes.sizeof(cls) == {"tboa_kv_cache_desc": 24, "tboa_kv_batch": 48, "tboa_rotation": 24}[cname]


@pytest.mark.parametrize("heads,dh,pt,st", [(1, 1, 16, 1), (8, 128, 64, 1), (2, 100, 32, 32), (5, 256, 1024, 2), (3, 192, 16, 16), (65535, 33, 64, 4)])
def test_bytes_of_a_page(heads, dh, pt, st):
    want = 2 * heads * pt * ref.padded(dh) + 2 * heads * (pt // st) * 8
    assert tb.KVCache.page_bytes(heads, dh, pt, st) == -(-want // 256) * 256


@pytest.mark.parametrize("heads,dh,pt,st", [(0, 64, 64, 1), (65536, 64, 64, 1), (1, 0, 64, 1), (1, 257, 64, 1), (1, 64, 8, 1), (1, 64, 2048, 1), (1, 64, 48, 1), (1, 64, 64, 3), (1, 64, 64, 128),
                                            (1, 64, 64, 0), (-1, 64, 64, 1)])
def test_caches_that_do_not_exist(heads, dh, pt, st):
    with pytest.raises(AssertionError):
        tb.KVCache.page_bytes(heads, dh, pt, st)
    desc = tb.binding.KVCacheDesc(heads, dh, pt, st, 10)
    assert tb.binding._lib.tboa_kv_cache_page_bytes(ctypes.byref(desc)) == 0
    assert tb.binding._lib.tboa_kv_cache_attention_workspace_bytes(ctypes.byref(desc), max(heads, 1), 1, 1) == 0


def test_workspace_is_host_arithmetic():
    q = tb.binding._lib.tboa_kv_cache_attention_workspace_bytes
    desc = tb.binding.KVCacheDesc(8, 128, 64, 1, 1000)
    one, many, prompt = (q(ctypes.byref(desc), 64, s, n) for s, n in ((1, 1), (256, 256), (4, 16384)))
    assert 0 < one <= many and 0 < prompt < 1 << 30
    for heads, seqs, tokens in ((63, 1, 1), (0, 1, 1), (-8, 1, 1), (64, -1, 1), (64, 1, -1), (64, 1, 1 << 25), (64, (1 << 20) + 1, 1)):
        assert q(ctypes.byref(desc), heads, seqs, tokens) == 0, (heads, seqs, tokens)
    assert q(None, 64, 1, 1) == 0 and tb.binding._lib.tboa_kv_cache_page_bytes(None) == 0


def test_null_context_is_rejected():
    lib, d, b = tb.binding._lib, ctypes.byref(tb.binding.KVCacheDesc(1, 64, 16, 1, 1)), ctypes.byref(tb.binding.KVBatchDesc(1, 1, 1, None, None, None, 0))
    assert lib.tboa_head_norm_rotate(None, 1, 64, 0, 1, None, 64, None, 0, None, 0, None, 0.0, None, None, None, 64, None, 0) == -1
    assert lib.tboa_kv_cache_append(None, d, b, 0, None, 64, None, 64, None, None, None) == -1
    assert lib.tboa_kv_cache_attention(None, d, b, 1, 0, None, 64, None, 0.0, 0, None, 64) == -1


class Reached(Exception):
    pass


@pytest.fixture
def ctx(monkeypatch):
    real = tb.binding._lib

    class Stub:
        tboa_kv_cache_page_bytes = real.tboa_kv_cache_page_bytes

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


def batch(n_seqs=2, per=3):
    z = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    return tb.KVBatch(z(n_seqs + 1), z(n_seqs), z(n_seqs, per))


def test_arguments_of_the_rotation(ctx):
    x, y, k = ctx.rows(3, 4, 64), ctx.rows(3, 4, 64), ctx.rows(3, 2, 64)
    pos, w = torch.zeros(3, dtype=torch.int32), torch.zeros(64)
    rot = tb.Rotation(torch.zeros(10, 64))
    good = [dict(Q=x), dict(Q=x, K=k, out_k=k, wq=w, wk=w, rotation=rot, positions=pos), dict(Q=ctx.rows(3, 9, 64)[:, 2:6], K=k, out_k=k)]
    for kw in good:
        with pytest.raises(Reached):
            ctx.head_norm_rotate(out_q=y, **kw)
    bad = [dict(K=ctx.rows(2, 2, 64)), dict(K=ctx.rows(3, 2, 32)), dict(K=ctx.rows(3, 2, 64, dtype=torch.bfloat16)), dict(rotation=rot), dict(rotation=rot, positions=pos[:2]),
           dict(rotation=rot, positions=pos.long()), dict(wq=w[:32]), dict(wq=w.double()), dict(out_q=ctx.rows(2, 4, 64)), dict(out_q=ctx.rows(3, 5, 64)), dict(out_q=ctx.rows(3, 64, 4)[..., :4]),
           dict(K=k, out_k=ctx.rows(2, 2, 64)), dict(Q=ctx.rows(3, 4, 128)[..., ::2]), dict(Q=ctx.rows(3, 64, 4).transpose(1, 2)), dict(Q=ctx.rows(3, 4, 96)[..., :64])]
    for kw in bad:
        with pytest.raises(AssertionError):
            ctx.head_norm_rotate(**dict(dict(Q=x, out_q=y, out_k=k), **kw))
    for table in (torch.zeros(10, 64, dtype=torch.float64), torch.zeros(640), torch.zeros(64, 10).t()):
        with pytest.raises(AssertionError):
            tb.Rotation(table)


def test_arguments_of_the_cache(ctx):
    per = tb.KVCache.page_bytes(2, 64, 16, 1)
    cache = tb.KVCache(torch.zeros(5, per, dtype=torch.uint8), 2, 64, 16, 1)
    for data in (torch.zeros(5, per + 256, dtype=torch.uint8), torch.zeros(5 * per, dtype=torch.uint8), torch.zeros(5, per, dtype=torch.int8), torch.zeros(5, 2 * per, dtype=torch.uint8)[:, ::2]):
        with pytest.raises(AssertionError):
            tb.KVCache(data, 2, 64, 16, 1)
    k = ctx.rows(3, 2, 64)
    pos, rot = torch.zeros(3, dtype=torch.int32), tb.Rotation(torch.zeros(10, 64))
    for args in ((k, k), (k, k, rot), (k, k, rot, pos), (k[:0], k[:0])):
        with pytest.raises(Reached):
            ctx.kv_cache_append(cache, batch(), *args)
    for args in ((k, k[:2]), (k, ctx.rows(3, 2, 64, dtype=torch.bfloat16)), (ctx.rows(3, 1, 64), k), (k, ctx.rows(3, 2, 32)), (k, k, rot, pos[:2]), (k, k, rot, pos.long())):
        with pytest.raises(AssertionError):
            ctx.kv_cache_append(cache, batch(), *args)
    q = ctx.rows(3, 4, 64)
    for kw in (dict(out=ctx.rows(3, 4, 64)), dict(out=ctx.rows(3, 8, 64)[:, 2:6])):
        with pytest.raises(Reached):
            ctx.kv_cache_attention(cache, batch(), q, **kw)
    for kw in (dict(out=ctx.rows(2, 4, 64)), dict(out=ctx.rows(3, 3, 64)), dict(out=ctx.rows(3, 4, 64, dtype=torch.bfloat16)), dict(Q=ctx.rows(3, 4, 32))):
        with pytest.raises(AssertionError):
            ctx.kv_cache_attention(cache, batch(), **dict(dict(Q=q), **kw))


def test_arguments_of_a_batch(ctx):
    z = lambda *s, dtype=torch.int32: torch.zeros(*s, dtype=dtype)  # noqa: E731
    tb.KVBatch(z(3), z(2), z(2, 5))
    for starts, lens, pages in ((z(2), z(2), z(2, 5)), (z(3), z(3), z(2, 5)), (z(3), z(2), z(10)), (z(3, dtype=torch.int64), z(2), z(2, 5)), (z(3), z(2), z(5, 2).t()), (z(3), z(2, 1), z(2, 5))):
        with pytest.raises(AssertionError):
            tb.KVBatch(starts, lens, pages)
