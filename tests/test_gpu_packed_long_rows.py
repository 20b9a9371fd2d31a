"""tboa_packed_linear of rows of millions of channels (GPU)."""
import pytest
import torch

from tests import packed_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx(lib):
    c = lib.Context()
    yield c
    c.close()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("bits,d_in,group,tokens", [(4, 16433536, 1173824, 1), (4, 3 * 87381 * 16, 87381 * 16, 65), (8, 8140704, 208736, 70), (2, 1 << 24, 1 << 23, 2), (2, 1 << 24, 1 << 19, 40)])
def test_groups_of_millions_of_channels(ctx, lib, bits, d_in, group, tokens, dtype):
    """Every channel has its own group's scale: X is 0 but for 64 channels on either side of the groups' borders, where scales and zeros jump."""
    d_out, ng = 3, d_in // group
    g = torch.Generator().manual_seed(5)
    codes = torch.randint(0, 2 ** bits, (d_out, d_in), generator=g, dtype=torch.uint8)
    scales, zeros = torch.exp2(10.0 * (torch.arange(ng) % 2))[None].expand(d_out, ng) * (1 + torch.rand(d_out, ng, generator=g)), torch.randint(0, 2 ** bits, (d_out, ng), generator=g).float()
    packed = lib.PackedWeight(ctx.pack_codes(codes.cuda(), bits), scales.cuda(), zeros.cuda(), d_in, bits, group)
    near = torch.cat([torch.arange(max(k * group - 64, 0), min(k * group + 64, d_in)) for k in range(ng + 1)])
    part = torch.randn(tokens, len(near), generator=g).to(dtype)
    x = torch.zeros(tokens, d_in, dtype=dtype, device="cuda")
    x[:, near.cuda()] = part.cuda()
    w = (codes[:, near].double() - zeros.double()[:, near // group]) * scales.double()[:, near // group]
    want, s = part.double() @ w.T, part.double().abs() @ (scales.double()[:, near // group] * 2 ** (bits + 2)).T
    # zeros add nothing to a sum; what is added is rounded once a matrix instruction that has anything to add (16 channels of 128 a border) and, in passing from group to group, 3 times a group
    lim = ((8 + 3) * (ng + 1) + 32) * 2.0 ** -24 * s + 2.0 ** -21 * s
    ref.check(ctx.packed_linear(packed, x), want.cuda(), lim.cuda(), telling=0.6)
