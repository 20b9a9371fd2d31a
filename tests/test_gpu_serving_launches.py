"""Serving calls of more workgroups than one launch takes (GPU): of 2^32 work items and more the runtime starts what is left of their number modulo 2^32, and says nothing."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx(lib):
    c = lib.Context()
    yield c
    c.close()


def test_head_vectors_of_two_launches(ctx, lib):
    """72 million vectors of one channel, four to a workgroup of 256."""
    T, H = 1100, 65535
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(T, H, 1, generator=g, device="cuda")
    w = torch.tensor([1.25], device="cuda")
    y, _ = ctx.head_norm_rotate(x, None, w, eps=0.5)
    torch.cuda.synchronize()
    want = x.double() / torch.sqrt(x.double() ** 2 + 0.5) * 1.25
    assert ((y.double() - want).abs() <= 6 * 2.0 ** -24 * want.abs()).all()      # factor, two products, output: half a step each
