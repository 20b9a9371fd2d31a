"""Serving calls of more workgroups than one launch takes (GPU): of 2^32 work items and more the runtime starts what is left of their number modulo 2^32, and says nothing."""
import pytest
import torch

from tests import serving_ref as ref
from tests.test_gpu_kv_cache_append import i32

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


def test_row_tiles_of_more_workgroups_than_a_launch_takes(ctx, lib):
    """128 sequences of 40 new tokens and 65535 heads: the kernel for many rows would be asked for 9.7 million workgroups of 512."""
    S, N, H, pt = 128, 40, 65535, 64
    g = torch.Generator(device="cuda").manual_seed(4)
    data = torch.randint(0, 256, (1, lib.KVCache.page_bytes(H, 1, pt, 1)), generator=g, device="cuda", dtype=torch.uint8)
    lev, gr = H * pt * ref.padded(1), H * pt * 8
    k, v = data[0, :lev].view(H, pt, 32)[:, :, 0], data[0, lev:2 * lev].view(H, pt // 16, 32, 16)[:, :, 0].reshape(H, pt)
    kg, vg = (data[0, 2 * lev + i * gr:2 * lev + (i + 1) * gr].view(torch.float32).view(H, pt, 2) for i in range(2))
    for z in (kg, vg):
        z[..., 0] = 0.01
        z[..., 1] = 128
    key, val = ((x.double() - z[..., 1].double()) * z[..., 0].double() for x, z in ((k, kg), (v, vg)))
    lens = [N + b % 25 for b in range(S)]
    q = torch.randn(N * S, H, 1, generator=g, device="cuda").bfloat16()
    out = torch.full_like(q, 7)
    ctx.kv_cache_attention(lib.KVCache(data, H, 1, pt, 1), lib.KVBatch(i32(range(0, N * S + 1, N)), i32(lens), i32([[0]] * S)), q, out=out)
    torch.cuda.synchronize()
    place = torch.arange(pt, device="cuda")
    for b in (0, 1, 40, 77, 126, 127):
        rows = slice(N * b, N * b + N)
        x = q[rows].double() * key[None, :, :]
        seen = place[None] <= torch.arange(lens[b] - N, lens[b], device="cuda")[:, None]
        a = torch.softmax(x.masked_fill(~seen[:, None], -torch.inf), -1)
        o, size = (a * val[None]).sum(-1), (a * val[None].abs()).sum(-1)
        # probabilities in one half: 2^-11; scores of at most 7 with 5 operations, twice, the exponential and 64 tokens: below 2^-17 together
        assert ((out[rows, :, 0].double() - o).abs() <= 2.0 ** -8 * o.abs() + (2.0 ** -11 + 2.0 ** -17) * size).all(), b
