"""tboa_packed_linear and tboa_packed_swiglu of many tokens: the bits of codes and scales, and grids far apart in a row (GPU)."""
import pytest
import torch

from tests import packed_ref as ref
from tests.test_gpu_packed_linear import rows, silu, swiglu_bound

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx(lib):
    c = lib.Context()
    yield c
    c.close()


def weight(lib, ctx, d_out, d_in, bits, group, seed, scales):
    packed, w = ref.weight(lib, ctx, d_out, d_in, bits, group, seed)
    old = packed.scales.clone()
    packed.scales.copy_(scales.to(packed.scales).expand_as(old))
    ng = old.shape[1]
    return packed, (w.view(d_out, ng, -1) / old.double()[..., None] * packed.scales.double()[..., None]).view(d_out, d_in)


def bound(x, w, ng):
    """Of X W^T of more than 64 tokens before its last rounding.  With S = sum |x| |w|: codes less zeros and bf16 X are exact, a result is rounded at most d_in / 16 + 16 times by a matrix instruction's sum and
    3 ng times more where it passes from the unit of one group's scale to the next one's (the quotient of the scales, rounded, and the product), by 2^-24 of at most S each; fp32 X in two half
    terms 2^-22 of S; the smallest channels of X are off by 2^-39 of their row's largest at most."""
    size, d_in = x.double().abs(), x.shape[1]
    s = size @ w.abs().T
    return (d_in / 16 + 16 + 3 * ng) * 2.0 ** -24 * s + 2.0 ** -22 * (x.dtype == torch.float32) * s + 2.0 ** -38 * size.amax(1, keepdim=True) * w.abs().sum(1)[None] + 2.0 ** -133


def rounded(got, want, lim):
    """Every output is the rounding of some value within the bound (rounding is monotonic: between the roundings of the bound's ends)."""
    g, low, high = got.float(), (want - lim).float().to(got.dtype).float(), (want + lim).float().to(got.dtype).float()
    print("rounded elsewhere: %d of %d" % (((g < low) | (g > high)).sum(), g.numel()), flush=True)
    assert torch.isfinite(want).all() and ((g >= low) & (g <= high)).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("spread", [0, 16])
@pytest.mark.parametrize("bits,group,d_in,d_out,tokens", [(4, 128, 2048, 600, 65), (3, 128, 1280, 300, 300), (2, 256, 1024, 130, 700), (8, 128, 1024, 520, 200), (4, 64, 1024, 260, 100), (3, 32, 640, 70, 300), (4, 16, 1280, 300, 129),
                                                         (2, 48, 960, 200, 260), (8, 640, 1920, 300, 513)])
def test_groups_of_many_tokens_are_exact(ctx, lib, bits, group, d_in, d_out, tokens, spread, dtype):
    """Codes less zeros enter exactly and scales with all their bits, also where a row's scales are 2^-16 of each other and the channels of the smallest are the largest."""
    ng = d_in // group
    g = torch.Generator().manual_seed(bits + group)
    power = -spread * torch.rand(d_out, ng, generator=g) if spread else torch.zeros(d_out, ng)
    if spread:
        power[:] = power[:1].round()      # the same for all outputs, so that X can be large where scales are small
    scales = torch.exp2(power) * (0.01 + 0.02 * torch.rand(d_out, ng, generator=g))
    packed, w = weight(lib, ctx, d_out, d_in, bits, group, 31, scales)
    up, wu = weight(lib, ctx, d_out, d_in, bits, group, 32, scales)
    x = rows(tokens, d_in, torch.float32, 33, spread=0.5)
    if spread:
        x = x * torch.exp2(-power[0]).repeat_interleave(group)[None].cuda()
    x = x.to(dtype)
    want, lim = x.double() @ w.T, bound(x, w, ng)
    rounded(ctx.packed_linear(packed, x), want, lim)
    u, eu = x.double() @ wu.T, bound(x, wu, ng)
    rounded(ctx.packed_swiglu(packed, up, x), silu(want) * u, swiglu_bound(want, u, lim, eu))
