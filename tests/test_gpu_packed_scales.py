"""tboa_packed_linear of scales that are zero, far below their row's largest, negative or no numbers (GPU); the bounds are derived in tests/packed_ref.py."""
import pytest
import torch

from tests import packed_ref as ref
from tests.test_gpu_packed_linear import rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx(lib):
    c = lib.Context()
    yield c
    c.close()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("tokens", [2, 40, 100, 300])
@pytest.mark.parametrize("bits,group,d_in", [(4, 128, 1024), (3, 256, 1280), (2, 64, 640), (8, 48, 960), (4, 0, 512)])
def test_scales_that_are_special(ctx, lib, bits, group, d_in, tokens, dtype):
    """Output by output: one group's scale 0, all 0, one 2^-70 of the others (it counts as 2^-60 of the largest for many tokens: far below what the smallest channels of X are off by), all 2^-100, a negative
    one, one infinite (no finite numbers there, the other outputs as they were)."""
    d_out = 40
    packed, w = ref.weight(lib, ctx, d_out, d_in, bits, group, 51)
    s, ng = packed.scales, packed.scales.shape[1]
    factor = torch.ones(d_out, ng, dtype=torch.float64)
    factor[3, ng // 2] = 0
    factor[4] = 0
    factor[5, -1] = 2.0 ** -70
    factor[6] = 2.0 ** -100
    factor[7, 0] = -1
    factor[8, 1:] = 0
    s.mul_(factor.to(s))
    w = (w.view(d_out, ng, -1) * factor.to(w)[..., None]).view(d_out, d_in)
    x = rows(tokens, d_in, dtype, 52, spread=0.3)
    got = ctx.packed_linear(packed, x)
    ref.check(got, x.double() @ w.T, ref.bound(x, w, packed), telling=0.8)
    assert (got[:, 4] == 0).all() and torch.isfinite(got).all()
    s[10, ng // 2] = float("inf")
    keep = torch.arange(d_out, device="cuda") != 10
    bad = ctx.packed_linear(packed, x)
    assert not torch.isfinite(bad[:, 10]).any() and torch.equal(bad[:, keep], got[:, keep])
