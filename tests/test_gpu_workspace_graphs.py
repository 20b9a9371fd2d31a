"""A context's workspace and the graphs that hold its address (GPU)."""
import numpy as np
import pytest
import torch

from tests.test_gpu_kv_cache_append import layout
from tests.test_gpu_serving import Step, captured

pytestmark = pytest.mark.gpu

MORE_THAN_ANY = 1 << 46


def refused(lib, call):
    with pytest.raises(lib.TurboBoAError) as e:
        call()
    assert e.value.code == -3
    return str(e.value)


def test_a_captured_call_without_room_is_refused(lib):
    """A call that has a smaller form than the one it would take: not recorded in it without a word."""
    d, hq, hkv, dh, length = 8192, 64, 8, 128, 256
    g = torch.Generator(device="cuda").manual_seed(1)
    X = torch.randn(1, length, d, generator=g, device="cuda").bfloat16()
    Wq, Wo = ((0.02 * torch.randn(d, d, generator=g, device="cuda")).bfloat16() for _ in "qo")
    Wk, Wv = ((0.02 * torch.randn(hkv * dh, d, generator=g, device="cuda")).bfloat16() for _ in "kv")
    call = lambda c: c.build_hessians(X, None, Wq, Wk, Wv, Wo, hq, hkv, dh, with_R_v=False, parts="qk")  # noqa: E731
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    ctx, roomy = lib.Context(stream=stream), lib.Context()
    try:
        want = call(roomy)
        torch.cuda.synchronize()
        refused(lib, lambda: ctx.reserve_workspace(MORE_THAN_ANY))
        ctx.reserve_workspace(256)      # the caller settles for little: the call takes its smaller form
        with torch.cuda.stream(stream):
            call(ctx)
        stream.synchronize()
        least = ctx.workspace_bytes()
        assert least < roomy.workspace_bytes()
        ctx.reserve_workspace(least + 256)      # there is room again, as far as the context knows
        mark = torch.zeros(1, device="cuda")

        def record():
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                mark.zero_()
                call(ctx)
        assert "captured" in refused(lib, record)
        with torch.cuda.stream(stream):
            got = call(ctx)
        torch.cuda.synchronize()
        assert ctx.workspace_bytes() == roomy.workspace_bytes() and torch.equal(got["Hout_q"], want["Hout_q"])
    finally:
        ctx.close()
        roomy.close()


def test_a_refused_growth_leaves_the_workspace_of_a_graph(lib):
    heads, rep, dh, pt = 2, 4, 128, 64
    lens = np.array([5, 300, 64])
    total, pages = layout(lens + 40, pt, 4)
    stream = torch.cuda.Stream()
    own, other = lib.Context(stream=stream), lib.Context()
    try:
        step = Step(lib, [1, 1, 1], lens, pages, total, heads, rep, dh, pt, 1, torch.bfloat16, 1)
        own.reserve_workspace(step.need(own))
        held = own.workspace_bytes()
        shadow = step.data.clone()
        torch.cuda.synchronize()
        graph = captured(lib, step, own, stream)
        refused(lib, lambda: own.reserve_workspace(MORE_THAN_ANY))
        assert own.workspace_bytes() == held
        for turn in range(3):
            lens = lens + 1
            step.fill(lens, turn)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            got = step.out.clone()
            want = step.run(other, data=shadow, out=torch.empty_like(step.out), turned=torch.empty_like(step.turned))
            torch.cuda.synchronize()
            assert torch.equal(got, want) and torch.equal(step.data, shadow)
            with torch.cuda.stream(stream):
                again = step.run(own, data=shadow, out=torch.empty_like(step.out), turned=torch.empty_like(step.turned))
            torch.cuda.synchronize()
            assert torch.equal(again, want) and own.workspace_bytes() == held
    finally:
        own.close()
        other.close()


def test_any_captured_call_keeps_its_workspace(lib):
    """A graph of a call that is no attention, replayed after the context's workspace has grown and what was free has been overwritten."""
    g = torch.Generator(device="cuda").manual_seed(2)
    X, W = torch.randn(70, 256, generator=g, device="cuda"), torch.randn(96, 256, generator=g, device="cuda")
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    own, other = lib.Context(stream=stream), lib.Context()
    try:
        with torch.cuda.stream(stream):
            own.linear_forward(X, W)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            out = own.linear_forward(X, W)
        held = own.workspace_bytes()
        for turn in range(3):
            own.reserve_workspace(held + ((turn + 1) << 20))
            filler = torch.full((held + (turn << 20),), 255, dtype=torch.uint8, device="cuda")
            X.normal_(generator=g)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            want = other.linear_forward(X, W)
            torch.cuda.synchronize()
            assert torch.equal(out, want) and (filler == 255).all()
    finally:
        own.close()
        other.close()
