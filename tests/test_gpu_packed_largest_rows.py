"""tboa_packed_linear of the largest and smallest rows of X (GPU); the bounds are derived in tests/packed_ref.py."""
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
@pytest.mark.parametrize("tokens", [1, 3, 20, 50, 100, 400])
@pytest.mark.parametrize("bits,group", [(2, 0), (2, 64), (3, 128), (4, 0), (4, 32), (8, 0), (8, 128), (3, 16), (4, 8)])
def test_the_largest_rows(ctx, lib, bits, group, tokens, dtype):
    """Rows of X near the largest number that their type has (of one sign, so that an offset's share would leave fp32), whose results are ordinary numbers; and of the smallest."""
    d_out, d_in = 70, 768
    packed, w = ref.weight(lib, ctx, d_out, d_in, bits, group, 41)
    packed.scales.mul_(2.0 ** -14)
    w = w * 2.0 ** -14
    x = 1 + rows(tokens, d_in, torch.float32, 42, spread=0.0).abs().clamp(max=2)
    for power in (125, 126, -60):
        y = (x * 2.0 ** power).to(dtype)
        if power == 126:
            y[:, 5] = torch.finfo(dtype).max
        ref.check(ctx.packed_linear(packed, y), y.double() @ w.T, ref.bound(y, w, packed), telling=0.6)
