"""Linear layers on packed weights in 64 bits (torch, on the device), and the bound of their error."""
import torch

F64 = torch.float64


def weight(lib, ctx, d_out, d_in, bits, group, seed):
    """Codes, scales and zeros of any values, packed by the library; and the exact matrix in 64 bits."""
    g = torch.Generator().manual_seed(seed)
    ng = d_in // group if group else 1
    codes = torch.randint(0, 2 ** bits, (d_out, d_in), generator=g, dtype=torch.uint8).cuda()
    scales = torch.exp(0.7 * torch.randn(d_out, ng, generator=g) - 4).cuda()
    zeros = torch.randint(0, 2 ** bits, (d_out, ng), generator=g).float().cuda()
    packed = lib.PackedWeight(ctx.pack_codes(codes, bits), scales, zeros, d_in, bits, group)
    exact = ((codes.double().view(d_out, ng, -1) - zeros.double()[..., None]) * scales.double()[..., None]).view(d_out, d_in)
    return packed, exact


def bound(x, w, packed):
    """Of X W^T before its last rounding, per element.  With S = sum |x| |w| and R = sum |x| scale 2^(bits + 2):
      sums       a result is rounded at most d_in / 16 + 16 times (a matrix instruction adds 16 terms or more), each time by 2^-24 of what codes less zeros add up to, S at most.  Where codes enter
                 with an offset of up to 2^bits (bf16 X), its share is taken out again every 256 channels or fewer: 20 times 2^-24 of R more (codes, offset and zero are below 2^bits each)
      operands   weights scale (code - zero) in fp32 2^-23 of S; fp32 X in two half terms 2^-22 of S, the smallest channels to 2^-39 of the row's largest.  bf16 X of more
                 than 64 tokens and several scales a row: scale (code - zero) as half, the product of a scale as half and a whole number up to 255, exact as half: (1 + 2^-11)^2 - 1 < 2^-10 + 2^-22 of
                 S; scales down to 2^-13 of their row's largest (which is 1 .. 2) are normal halves, smaller ones off by 2^-25 at most, times 255"""
    d = packed.desc
    ng = packed.scales.numel() // d.d_out
    step = packed.scales.double().abs().view(d.d_out, ng).repeat_interleave(d.d_in // ng, 1)
    size = x.double().abs()
    s = size @ w.abs().T
    lim = (d.d_in / 16 + 16) * 2.0 ** -24 * s + 2.0 ** -21 * s + 2.0 ** -38 * size.amax(1, keepdim=True) * w.abs().sum(1)[None]
    if x.dtype == torch.bfloat16 and len(x) > 64 and ng > 1:
        lim = lim + (2.0 ** -10 + 2.0 ** -22) * s + 255 * 2.0 ** -24 * size.sum(1, keepdim=True) * (step.amax(1) * (step.amin(1) < 2.0 ** -13 * step.amax(1)))[None]
    return lim + 20 * 2.0 ** -24 * 2.0 ** (d.bits + 2) * (size @ step.T) if x.dtype == torch.bfloat16 else lim


def check(got, want, lim, telling=0.9):
    """Finite results within the bound and half a step of their type; at least `telling` of those that are not 0 are larger than the bound, so that zeros would fail."""
    half = torch.finfo(got.dtype).eps / 2
    lim = lim + half * (want.abs() + lim) + 2.0 ** -133
    err = (got.double() - want).abs()
    print("error over bound %.3f" % (err / lim).max().item(), flush=True)
    assert (err <= lim).all(), (err / lim).max().item()
    some = want != 0
    assert some.sum() < 20 or (want.abs() > lim)[some].double().mean() >= telling
