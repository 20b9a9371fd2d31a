"""tboa_kv_cache_attention of values so large that their weighted sum, before it is divided by the sum of the weights, leaves fp32 (GPU): the outputs, averages of them, do not."""
import numpy as np
import pytest
import torch

from tests.attention_bounds import check
from tests.test_gpu_kv_cache_attention import case
from tests.test_gpu_kv_cache_attention_ranges import attend, kinds, wide

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx(lib):
    c = lib.Context()
    yield c
    c.close()


@pytest.mark.parametrize("dtype,heads,new,length,many", kinds((1, 1, 60, False), (1, 1, 250, False), (1, 3, 6000, False), (700, 1, 200, False), (1, 50, 400, False), (1, 50, 400, True), (1, 70, 5000, True),
                                                              (300, 20, 100, True)))
def test_averages_of_large_values(ctx, lib, dtype, heads, new, length, many):
    starts, pages, cache, _, q = case(lib, heads, 2, 32, [new], [length], 64, 1, dtype, new + length)
    rng = np.random.default_rng(1)
    cache.vg[..., 0] = 2.0 ** 119 * (0.5 + 0.5 * rng.random(cache.vg.shape[:-1]))
    cache.vg[..., 1] = rng.integers(0, 20, cache.vg.shape[:-1])      # values up to 2^127, most of them positive
    if many:
        pages = wide(pages, 64)
    got = attend(ctx, lib, cache, starts, [length], pages, q)
    assert torch.isfinite(got).all()
    check(got, cache, starts, [length], pages, q, 1 / np.sqrt(32), 0, many=many)
