"""A block served with rows that belong to no sequence (GPU)."""
import numpy as np
import pytest
import torch

from paper_2602_04929_amd import pipeline
from tests.test_gpu_head_norm_rotate import table
from tests.test_gpu_kv_cache_append import i32, layout

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("residual", [False, True])
def test_rows_behind_the_last_sequence(lib, dtype, residual):
    """They attend to nothing: o is 0 there and Y the residual, whatever was in the memory before; the others are those of the batch without them."""
    Hq, Hkv, dh, d = 4, 2, 64, 256
    g = torch.Generator(device="cuda").manual_seed(1)
    W = dict(Wqkv=0.05 * torch.randn((Hq + 2 * Hkv) * dh, d, generator=g, device="cuda"), Wo=0.05 * torch.randn(d, Hq * dh, generator=g, device="cuda"))
    new, lens, spare = [3, 1, 0], [40, 17, 5], 4
    total, pages = layout(lens, 16, 2)
    starts = np.concatenate([[0], np.cumsum(new)])
    rows = starts[-1] + spare
    X = torch.randn(rows, d, generator=g, device="cuda").to(dtype)
    place = i32(np.concatenate([np.arange(n - k, n) for n, k in zip(lens, new)] + [np.full(spare, 1 << 20)]))
    data = torch.randint(0, 256, (total, lib.KVCache.page_bytes(Hkv, dh, 16, 1)), generator=g, device="cuda", dtype=torch.uint8)
    c = lib.KVCache(data, Hkv, dh, 16, 1)
    for kv in range(2):      # grids of K and of V
        at = 2 * Hkv * 16 * 64 + kv * Hkv * 16 * 8
        data[:, at:at + Hkv * 16 * 8].view(torch.float32).view(total, Hkv, 16, 2).copy_(torch.tensor([0.01, 128.0], device="cuda"))
    ctx = lib.Context()
    try:
        def serve(n, cache):
            spoiled = [torch.full((rows, Hq, dh), float("nan"), dtype=dtype, device="cuda") for _ in range(8)]
            del spoiled      # what is allocated next holds NaN
            return pipeline.serve_attention_block(ctx, W, X[:n].contiguous(), lib.KVCache(cache, Hkv, dh, 16, 1), lib.KVBatch(i32(starts), i32(lens), i32(pages)), Hq,
                                                  rotation=lib.Rotation(table(64, dh).cuda()), positions=place[:n].contiguous(), residual=X[:n].contiguous() if residual else None)
        one, other = data.clone(), data.clone()
        got, want = serve(rows, one), serve(rows - spare, other)
        torch.cuda.synchronize()
        assert torch.equal(one, other)
        for n in ("Y", "o", "v"):
            assert torch.equal(got[n][:rows - spare], want[n]), n
        assert (got["o"][rows - spare:] == 0).all()
        assert torch.equal(got["Y"][rows - spare:], X[rows - spare:] if residual else torch.zeros_like(X[rows - spare:]))
    finally:
        ctx.close()
