"""tboa_head_norm_rotate at both ends of the types' range (GPU): outputs are of the size of the weights there too."""
import numpy as np
import pytest
import torch

from tests import serving_ref as ref
from tests.test_gpu_head_norm_rotate import close, table

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx(lib):
    c = lib.Context()
    yield c
    c.close()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("dh,rot", [(128, 0), (96, 96), (33, 10)])
@pytest.mark.parametrize("eps", [0.0, 1e-60, 1e-30])
def test_from_the_least_to_the_largest(ctx, lib, dtype, dh, rot, eps):
    """Rows of sizes from subnormal ones to the largest, and an eps that fp32 does not hold."""
    sizes = [2.0 ** -140 if dtype == torch.float32 else 2.0 ** -128, 2.0 ** -126, 1e-30, 1e-15, 1.0, 1e15, 1e30, 2.0 ** 125]
    g = torch.Generator().manual_seed(dh)
    x = (torch.randn(len(sizes), 3, dh, generator=g).clamp(-4, 4) * torch.tensor(sizes, dtype=torch.float64)[:, None, None]).to(dtype)
    w = 1 + 0.3 * torch.randn(dh, generator=g)
    tab, pos = table(50, rot) if rot else None, torch.randint(0, 50, (len(sizes),), generator=g, dtype=torch.int32)
    y, _ = ctx.head_norm_rotate(x.cuda(), None, w.cuda(), eps=eps, rotation=lib.Rotation(tab.cuda()) if rot else None, positions=pos.cuda())
    torch.cuda.synchronize()
    x64, w64, t64 = x.double().numpy(), w.double().numpy(), None if tab is None else tab.numpy()
    want = ref.norm_rotate(x64, w64, eps, t64, pos.numpy(), False)
    assert np.isfinite(want).all() and torch.isfinite(y).all()
    close(y, want, x64, w64, t64, pos.numpy(), False, eps)
