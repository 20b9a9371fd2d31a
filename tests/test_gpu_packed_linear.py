"""tboa_packed_linear and tboa_packed_swiglu against the exact matrices in 64 bits (GPU); the bounds are derived in tests/packed_ref.py."""
import pytest
import torch

from tests import packed_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx(lib):
    c = lib.Context()
    yield c
    c.close()


def rows(tokens, d, dtype, seed, spread=1.0):
    """Rows of different sizes, a few channels ten times as large."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(tokens, d, generator=g) * torch.exp(spread * torch.randn(tokens, 1, generator=g))
    x[:, ::max(d // 3, 1)] *= 10
    return x.to(dtype).cuda()


def silu(v):
    return v * torch.sigmoid(v)


def swiglu_bound(g, u, eg, eu):
    """silu has a slope of at most 1.1; its own four operations in fp32 (the exponential and the quotient 2^-22 each at most)."""
    return 1.1 * eg * (u.abs() + eu) + silu(g).abs() * eu + 2.0 ** -20 * (silu(g) * u).abs() + 2.0 ** -120


SHAPES = [
    # d_out, d_in, group
    (1, 1, 0), (5, 7, 0), (16, 32, 0), (17, 33, 0), (40, 256, 128), (64, 512, 64), (33, 320, 32), (48, 1000, 100), (70, 1000, 0), (130, 1024, 256), (31, 96, 96), (20, 90, 3), (37, 63, 7), (96, 1152, 128),
    (256, 2048, 128), (300, 640, 0), (9, 4096, 512), (200, 384, 16), (24, 72, 8), (50, 1920, 960),
]
TOKENS = [1, 2, 5, 16, 17, 40, 64, 65, 100, 129, 300]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("bits", [2, 3, 4, 8])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_sizes(ctx, lib, shape, bits, dtype):
    d_out, d_in, group = shape
    packed, w = ref.weight(lib, ctx, d_out, d_in, bits, group, d_in + bits)
    up, wu = ref.weight(lib, ctx, d_out, d_in, bits, group, d_in + bits + 50)
    for tokens in TOKENS:
        x, res = rows(tokens, d_in, dtype, tokens), rows(tokens, d_out, dtype, tokens + 1)
        print(shape, bits, dtype, tokens, flush=True)
        want, lim = x.double() @ w.T, ref.bound(x, w, packed)
        ref.check(ctx.packed_linear(packed, x), want, lim, telling=0.7)
        ref.check(ctx.packed_linear(packed, x, residual=res), want + res.double(), lim + 2.0 ** -24 * (want.abs() + res.double().abs()), telling=0.7)
        u, eu = x.double() @ wu.T, ref.bound(x, wu, up)
        ref.check(ctx.packed_swiglu(packed, up, x), silu(want) * u, swiglu_bound(want, u, lim, eu), telling=0.2)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("bits,group,d_in,d_out,tokens", [(4, 128, 4096, 1024, 1), (4, 128, 8192, 300, 16), (2, 0, 8192, 512, 3), (3, 128, 5120, 640, 64), (4, 128, 4096, 1536, 512), (2, 128, 2048, 4096, 700),
                                                         (8, 0, 2048, 1030, 1000), (3, 128, 1280, 2000, 2100), (4, 64, 11008, 260, 200), (4, 0, 28672, 64, 130)])
def test_layers(ctx, lib, bits, group, d_in, d_out, tokens, dtype):
    packed, w = ref.weight(lib, ctx, d_out, d_in, bits, group, 3)
    up, wu = ref.weight(lib, ctx, d_out, d_in, bits, group, 4)
    x, res = rows(tokens, d_in, dtype, 5), rows(tokens, d_out, dtype, 6)
    want, lim = x.double() @ w.T, ref.bound(x, w, packed)
    ref.check(ctx.packed_linear(packed, x, residual=res), want + res.double(), lim + 2.0 ** -24 * (want.abs() + res.double().abs()))
    u, eu = x.double() @ wu.T, ref.bound(x, wu, up)
    ref.check(ctx.packed_swiglu(packed, up, x), silu(want) * u, swiglu_bound(want, u, lim, eu), telling=0.3)


@pytest.mark.parametrize("tokens", [1, 20, 300])
@pytest.mark.parametrize("bits,group", [(2, 0), (3, 128), (4, 128), (8, 0), (4, 192), (4, 32)])
def test_of_a_quantized_layer(ctx, lib, bits, group, tokens):
    """Codes, scales and zeros as the quantizer leaves them, and the same products as from its dequantized matrix."""
    g = torch.Generator().manual_seed(bits)
    d_out, d_in = 96, 384
    w, x = (0.02 * torch.randn(d_out, d_in, generator=g)).cuda(), torch.randn(2000, d_in, generator=g).cuda()
    H, _ = ctx.build_hessian_linear(x)
    layer = ctx.quantize_layer(w, H, None, None, 1, bits=bits, block=d_out, group=group)
    packed = lib.PackedWeight.of(ctx, layer, bits, group)
    exact = ((layer["codes"].double().view(d_out, -1, group or d_in) - layer["zeros"].double().view(d_out, -1, 1)) * layer["scales"].double().view(d_out, -1, 1)).view(d_out, d_in)
    for dtype in (torch.bfloat16, torch.float32):
        t = x[:tokens].to(dtype)
        ref.check(ctx.packed_linear(packed, t), t.double() @ exact.T, ref.bound(t, exact, packed))


@pytest.mark.parametrize("tokens", [3, 40, 200])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("bits,group,d_in", [(4, 128, 1280), (2, 0, 1000), (3, 100, 500)])
def test_strides_and_alignments(ctx, lib, bits, group, d_in, dtype, tokens):
    """X, residual and Y as parts of wider tensors, aligned and not, of several leading dimensions; Y in the residual's place; what is beside Y stays."""
    packed, w = ref.weight(lib, ctx, 130, d_in, bits, group, 1)
    x, res = rows(tokens, d_in, dtype, 2), rows(tokens, 130, dtype, 3)
    base = ctx.packed_linear(packed, x, residual=res)
    ref.check(base, x.double() @ w.T + res.double(), ref.bound(x, w, packed) + 2.0 ** -24 * ((x.double() @ w.T).abs() + res.double().abs()))
    gated = ctx.packed_swiglu(packed, packed, x)
    for shift, pitch in ((0, d_in + 8), (8, d_in + 64), (1, d_in + 3), (3, d_in + 8)):
        wide = torch.full((tokens * pitch + shift,), float("nan"), dtype=dtype, device="cuda")[shift:].view(tokens, pitch)
        wide[:, :d_in] = x
        out = torch.full((tokens, 130 + pitch), 7.0, dtype=dtype, device="cuda")
        out[:, shift:shift + 130] = res
        got = ctx.packed_linear(packed, wide[:, :d_in], residual=out[:, shift:shift + 130], out=out[:, shift:shift + 130])
        torch.cuda.synchronize()
        assert torch.equal(got, base) and (out[:, :shift] == 7).all() and (out[:, shift + 130:] == 7).all()
        ctx.packed_swiglu(packed, packed, wide[:, :d_in], out=out[:, shift:shift + 130])
        assert torch.equal(out[:, shift:shift + 130], gated) and (out[:, :shift] == 7).all() and (out[:, shift + 130:] == 7).all()
    if tokens % 2 == 0:
        assert torch.equal(ctx.packed_linear(packed, x.view(2, tokens // 2, d_in), residual=res.view(2, tokens // 2, 130)).view(tokens, 130), base)


@pytest.mark.parametrize("tokens", [2, 30, 150])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("group", [0, 128])
def test_values_that_are_special(ctx, lib, group, dtype, tokens):
    """Rows of X far apart in size keep their own precision; infinities and NaN in a row reach that row and no other; a NaN scale its output and no other."""
    packed, w = ref.weight(lib, ctx, 50, 1024, 4, group, 9)
    x = rows(tokens, 1024, dtype, 1, spread=0.0)
    x[0] *= 2.0 ** 60
    x[1] *= 2.0 ** -60
    ref.check(ctx.packed_linear(packed, x), x.double() @ w.T, ref.bound(x, w, packed))
    x[0] = 0
    assert (ctx.packed_linear(packed, x)[0] == 0).all()
    base = ctx.packed_linear(packed, x)
    for bad in (float("inf"), float("nan")):
        y = x.clone()
        y[1, 700] = bad
        got = ctx.packed_linear(packed, y)
        assert not torch.isfinite(got[1]).any() and torch.equal(got[2:], base[2:]) and torch.equal(got[0], base[0])
    packed.scales.view(50, -1)[3, -1] = float("nan")
    got = ctx.packed_linear(packed, x)
    keep = torch.arange(50, device="cuda") != 3
    assert torch.isnan(got[1:, 3]).all() and torch.equal(got[:, keep], base[:, keep])


def test_far_offsets(ctx, lib):
    """Packed rows beyond 2^32 bytes, rows of X and Y beyond 2^32 bytes."""
    d_in, d_out, words = 16384, 540000, 2048
    raw = torch.randint(-2 ** 31, 2 ** 31 - 1, (d_out, words), dtype=torch.int32, device="cuda")
    scales, zeros = torch.rand(d_out, 1, device="cuda") + 0.5, torch.randint(0, 16, (d_out, 1), device="cuda").float()
    packed = lib.PackedWeight(raw, scales, zeros, d_in, 4)
    for tokens in (2, 70):
        x = rows(tokens, d_in, torch.bfloat16, 1)
        got = ctx.packed_linear(packed, x)
        for part in (slice(0, 40), slice(d_out - 40, d_out), slice(524280, 524300)):
            nibbles = (raw[part].view(-1, words, 1).long() >> (4 * torch.arange(8, device="cuda")) & 15).reshape(-1, d_in)
            w = (nibbles.double() - zeros[part].double()) * scales[part].double()
            some = lib.PackedWeight(raw[part].contiguous(), scales[part].contiguous(), zeros[part].contiguous(), d_in, 4)
            ref.check(got[:, part], x.double() @ w.T, ref.bound(x, w, some))
        del got
    del raw, packed
    packed, w = ref.weight(lib, ctx, 64, 256, 4, 128, 2)
    pitch = (1 << 30) + 64
    for tokens in (4, 80):
        big = torch.zeros(4 * pitch if tokens == 4 else (tokens - 1) * (1 << 25) + 256, dtype=torch.bfloat16, device="cuda")
        far = torch.as_strided(big, (tokens, 256), (pitch if tokens == 4 else 1 << 25, 1))
        far.copy_(rows(tokens, 256, torch.bfloat16, 7))
        x = far.contiguous()
        got = ctx.packed_linear(packed, far)
        ref.check(got, x.double() @ w.T, ref.bound(x, w, packed))
        y = torch.as_strided(big, (tokens, 64), (pitch if tokens == 4 else 1 << 25, 1))
        assert torch.equal(ctx.packed_linear(packed, x, out=y), got)
        del big, far, y


@pytest.mark.parametrize("tokens", [1, 50, 200])
def test_streams_and_contexts(lib, tokens):
    """A context on a stream of its own, beside one on the current stream, on the same weights."""
    side = torch.cuda.Stream()
    a, b = lib.Context(), lib.Context(stream=side)
    try:
        packed, w = ref.weight(lib, a, 200, 1024, 4, 128, 1)
        x = rows(tokens, 1024, torch.bfloat16, 2)
        want = a.packed_linear(packed, x)
        ref.check(want, x.double() @ w.T, ref.bound(x, w, packed))
        side.wait_stream(torch.cuda.current_stream())
        outs = []
        for _ in range(5):
            outs += [a.packed_linear(packed, x), b.packed_linear(packed, x)]
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        assert all(torch.equal(o, want) for o in outs)
    finally:
        a.close()
        b.close()


@pytest.mark.parametrize("tokens,d_out", [(1, 200), (30, 200), (70, 300), (300, 1000)])
def test_captured_and_replayed(lib, tokens, d_out):
    """Both calls in a graph over fixed buffers, replayed with eager calls of the same context between the replays."""
    stream = torch.cuda.Stream()
    ctx = lib.Context(stream=stream)
    try:
        with torch.cuda.stream(stream):
            (down, wd), (gate, wg), (up, wu) = ref.weight(lib, ctx, 640, d_out, 4, 0, 1), ref.weight(lib, ctx, d_out, 640, 3, 128, 2), ref.weight(lib, ctx, d_out, 640, 3, 128, 3)
            x, act, out = rows(tokens, 640, torch.bfloat16, 1), torch.empty(tokens, d_out, dtype=torch.bfloat16, device="cuda"), torch.empty(tokens, 640, dtype=torch.bfloat16, device="cuda")
            need = max(ctx.packed_workspace_bytes(t, tokens, torch.bfloat16) for t in (down, gate, up))
            if need:
                g = torch.cuda.CUDAGraph()
                with torch.cuda.graph(g, stream=stream):
                    if ctx.workspace_bytes() < need:
                        with pytest.raises(lib.TurboBoAError) as e:
                            for _ in range(1):
                                ctx.packed_swiglu(gate, up, x, out=act)
                                ctx.packed_linear(down, act, residual=x, out=out)
                        assert e.value.code == -3
                    out.zero_()
                ctx.reserve_workspace(need)
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=stream):
                ctx.packed_swiglu(gate, up, x, out=act)
                ctx.packed_linear(down, act, residual=x, out=out)
            for k in range(4):
                x.copy_(rows(tokens, 640, torch.bfloat16, 10 + k))
                want = ctx.packed_linear(down, ctx.packed_swiglu(gate, up, x), residual=x).clone()
                out.fill_(7)
                act.fill_(7)
                g.replay()
                stream.synchronize()
                assert torch.equal(out, want), k
                ctx.reserve_workspace(ctx.workspace_bytes() + (1 << 20))      # a growth leaves what the graph holds
    finally:
        ctx.close()


def test_refusals(ctx, lib):
    packed, _ = ref.weight(lib, ctx, 20, 64, 4, 32, 1)
    other, _ = ref.weight(lib, ctx, 20, 64, 3, 32, 1)
    x = rows(3, 64, torch.bfloat16, 1)
    for bad in (rows(3, 63, torch.bfloat16, 1), x.t(), rows(3, 64, torch.bfloat16, 1).cpu()):
        with pytest.raises(AssertionError):
            ctx.packed_linear(packed, bad)
    with pytest.raises(KeyError):
        ctx.packed_linear(packed, x.half())
    with pytest.raises(lib.TurboBoAError) as e:
        ctx.packed_linear(packed, x.double())
    assert e.value.code == -1
    for kw in (dict(residual=rows(3, 21, torch.bfloat16, 1)), dict(residual=rows(3, 20, torch.float32, 1)), dict(out=rows(2, 20, torch.bfloat16, 1)), dict(out=rows(3, 20, torch.float32, 1))):
        with pytest.raises(AssertionError):
            ctx.packed_linear(packed, x, **kw)
    with pytest.raises(lib.TurboBoAError) as e:
        ctx.packed_swiglu(packed, other, x)
    assert e.value.code == -1
    with pytest.raises(lib.TurboBoAError) as e:
        ctx.packed_linear(packed, x[:1].expand(3, 64))      # rows that overlap
    assert e.value.code == -1
    assert ctx.packed_linear(packed, x[:0]).shape == (0, 20) and ctx.packed_swiglu(packed, packed, x[:0]).shape == (0, 20)


@pytest.mark.parametrize("tokens", [33, 64])
@pytest.mark.parametrize("bits,group,d_in,d_out", [(4, 128, 8192, 100), (3, 128, 13824, 33), (2, 0, 9000, 4100), (8, 64, 2048, 8200), (4, 32, 3200, 640)])
def test_channels_shared_by_workgroups(ctx, lib, bits, group, d_in, d_out, tokens):
    """33 to 64 tokens, whose channels are split: results, the residual in its place, and no workspace beyond what is said to be needed."""
    packed, w = ref.weight(lib, ctx, d_out, d_in, bits, group, 12)
    x, res = rows(tokens, d_in, torch.bfloat16, 13), rows(tokens, d_out, torch.bfloat16, 14)
    want, lim = x.double() @ w.T + res.double(), ref.bound(x, w, packed)
    own = lib.Context()
    try:
        got = own.packed_linear(packed, x, residual=res)
        torch.cuda.synchronize()
        assert own.workspace_bytes() <= max(2 * own.packed_workspace_bytes(packed, tokens, torch.bfloat16), 1 << 20)
        ref.check(got, want, lim + 2.0 ** -24 * (want.abs() + 2 * res.double().abs()))
        out = res.clone()
        own.packed_linear(packed, x, residual=out, out=out)
        torch.cuda.synchronize()
        assert torch.equal(out, got)
    finally:
        own.close()
