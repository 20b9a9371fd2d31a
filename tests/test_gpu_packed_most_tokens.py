"""Calls of more tokens than tboa_packed_linear and tboa_packed_swiglu work off in one round, against the exact matrices in 64 bits (GPU); the bounds are derived in tests/packed_ref.py."""
import pytest
import torch

from tests import packed_ref as ref
from tests.test_gpu_packed_linear import rows, silu, swiglu_bound

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d_out,d_in,bits,group,tokens", [(4096, 4096, 4, 128, 8192 + 2048), (2048, 2048, 3, 128, 8192 + 300), (500, 640, 4, 0, 8192 + 1), (260, 384, 2, 48, 2 * 8192 + 65)])
def test_more_than_one_round(lib, d_out, d_in, bits, group, tokens, dtype):
    """On a context that has no workspace yet, so that what the call itself takes has to do; tokens on both sides of a round's end, and what is behind the outputs stays."""
    ctx = lib.Context()
    try:
        packed, w = ref.weight(lib, ctx, d_out, d_in, bits, group, 21)
        up, wu = ref.weight(lib, ctx, d_out, d_in, bits, group, 22)
        x, res = rows(tokens, d_in, dtype, 23), rows(tokens, d_out, dtype, 24)
        for gated in (False, True):
            own = lib.Context()
            out = torch.full((tokens + 8, d_out), 7.0, dtype=dtype, device="cuda")
            got = own.packed_swiglu(packed, up, x, out=out[:tokens]) if gated else own.packed_linear(packed, x, residual=res, out=out[:tokens])
            torch.cuda.synchronize()
            assert own.workspace_bytes() <= own.packed_workspace_bytes(packed, tokens, dtype) and (out[tokens:] == 7).all()
            for part in (slice(0, 300), slice(8000, 8500), slice(tokens - 300, tokens)):
                want, lim = x[part].double() @ w.T, ref.bound(x[part], w, packed)
                if gated:
                    u, eu = x[part].double() @ wu.T, ref.bound(x[part], wu, up)
                    ref.check(got[part], silu(want) * u, swiglu_bound(want, u, lim, eu), telling=0.3)
                else:
                    ref.check(got[part], want + res[part].double(), lim + 2.0 ** -24 * (want.abs() + res[part].double().abs()))
            own.close()
    finally:
        ctx.close()


def test_captured_with_what_is_said_to_be_needed(lib):
    """Several rounds in one graph, with the workspace that the query tells and no more; and a batch of fewer tokens, whose tiles are split, in another graph on the same workspace."""
    stream = torch.cuda.Stream()
    ctx = lib.Context(stream=stream)
    try:
        with torch.cuda.stream(stream):
            (gate, _), (up, _) = ref.weight(lib, ctx, 2048, 1024, 4, 128, 61), ref.weight(lib, ctx, 2048, 1024, 4, 128, 62)
            sizes = (8192 + 2048, 2048)
            ctx.reserve_workspace(ctx.packed_workspace_bytes(gate, sizes[0], torch.bfloat16))
            held = ctx.workspace_bytes()
            calls = []
            for tokens in sizes:
                x, act = rows(tokens, 1024, torch.bfloat16, 63), torch.empty(tokens, 2048, dtype=torch.bfloat16, device="cuda")
                g = torch.cuda.CUDAGraph()
                with torch.cuda.graph(g, stream=stream):
                    ctx.packed_swiglu(gate, up, x, out=act)
                calls.append((g, x, act))
            for k in range(3):
                for g, x, act in calls:
                    x.copy_(rows(len(x), 1024, torch.bfloat16, 70 + k))
                    want = ctx.packed_swiglu(gate, up, x).clone()
                    act.fill_(7)
                    g.replay()
                    stream.synchronize()
                    assert torch.equal(act, want), (k, len(x))
            assert ctx.workspace_bytes() == held
    finally:
        ctx.close()
