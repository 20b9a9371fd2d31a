"""tboa_head_norm_rotate against the 64-bit form (GPU).  One fp32 operation is off by 2^-24 of its result; a result has at most eight of them (factor, two products of the norm, two of the
rotation, their sum, the rounding of the weight's product), each on terms no larger than |x|_2-scaled pairs, and one rounding to the output's type."""
import numpy as np
import pytest
import torch

from tests import serving_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx(lib):
    c = lib.Context()
    yield c
    c.close()


def table(n, rot, seed=0):
    a = np.arange(n)[:, None] * 10000.0 ** (-np.arange(rot // 2) * 2 / max(rot, 1))
    return torch.tensor(np.concatenate([np.cos(a), np.sin(a)], 1), dtype=torch.float32)


def close(got, want, x, w, tab, pos, adjacent, eps):
    """Element-wise: half a step of the type, and eight fp32 roundings of the pair's sizes."""
    size = np.abs(x.astype(np.float64))
    n = size if w is None else size / np.sqrt((size ** 2).mean(-1, keepdims=True) + eps) * np.abs(w)
    bound = n.copy()
    rot = 0 if tab is None else tab.shape[1]
    for i in range(rot // 2):
        a, b = (2 * i, 2 * i + 1) if adjacent else (i, i + rot // 2)
        bound[..., a] = bound[..., b] = n[..., a] + n[..., b]
    half = torch.finfo(got.dtype).eps / 2
    err = np.abs(got.double().cpu().numpy() - want)
    assert np.all(err <= half * np.abs(want) + (8 * 2.0 ** -24) * (1 + half) * bound + 2.0 ** -133), (err / (half * np.abs(want) + 8 * 2.0 ** -24 * bound + 1e-40)).max()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,hq,hk,dh,rot,adjacent,norm", [
    (1, 1, 1, 128, 128, False, True), (3, 64, 8, 128, 128, False, True), (17, 5, 3, 96, 96, True, True), (9, 4, 2, 64, 32, False, True), (5, 3, 1, 256, 256, True, False),
    (7, 10, 5, 100, 52, True, True), (4, 2, 2, 33, 10, False, True), (2, 3, 1, 1, 0, False, True), (6, 2, 1, 2, 2, True, False), (11, 2, 0, 80, 80, False, False), (300, 8, 8, 32, 16, False, True),
    (2, 3, 2, 192, 64, True, True), (3, 7, 2, 16, 16, True, True), (65, 3, 4, 48, 48, False, True)])
def test_against_the_plain_form(ctx, lib, dtype, T, hq, hk, dh, rot, adjacent, norm):
    g = torch.Generator().manual_seed(T * 1000 + dh)
    # a fused projection: queries, keys and something behind them in one row
    fused = (torch.randn(T, (hq + hk) * dh + 24, generator=g) * torch.exp(2 * torch.randn(T, 1, generator=g))).to(dtype).cuda()
    Q, K = fused[:, :hq * dh].view(T, hq, dh), fused[:, hq * dh:(hq + hk) * dh].view(T, hk, dh) if hk else None
    w = [(1 + 0.3 * torch.randn(dh, generator=g)).cuda() if norm else None for _ in "qk"]
    tab = table(5000, rot)
    pos = torch.randint(0, 5000, (T,), generator=g, dtype=torch.int32)
    rotation = lib.Rotation(tab.cuda(), adjacent=adjacent) if rot else None
    q, k = ctx.head_norm_rotate(Q, K, w[0], w[1], eps=1e-6, rotation=rotation, positions=pos.cuda())
    torch.cuda.synchronize()
    for got, x, ww in ((q, Q, w[0]), (k, K, w[1])):
        if x is None:
            continue
        x64, w64 = x.double().cpu().numpy(), None if ww is None else ww.double().cpu().numpy()
        want = ref.norm_rotate(x64, w64, 1e-6, tab.numpy() if rot else None, pos.numpy(), adjacent)
        close(got, want, x64, w64, tab.numpy() if rot else None, pos.numpy(), adjacent, 1e-6)
    # in place, and one side alone: the same bits
    copy = fused.clone()
    cq, ck = copy[:, :hq * dh].view(T, hq, dh), copy[:, hq * dh:(hq + hk) * dh].view(T, hk, dh) if hk else None
    ctx.head_norm_rotate(cq, ck, w[0], w[1], eps=1e-6, rotation=rotation, positions=pos.cuda(), out_q=cq, out_k=ck)
    alone, _ = ctx.head_norm_rotate(Q, None, w[0], None, eps=1e-6, rotation=rotation, positions=pos.cuda())
    torch.cuda.synchronize()
    assert torch.equal(cq, q) and torch.equal(alone, q) and (ck is None or torch.equal(ck, k))
    assert torch.equal(copy[:, (hq + hk) * dh:], fused[:, (hq + hk) * dh:])


def test_sizes_of_the_values(ctx, lib):
    """Rows of zeros, of values whose squares leave fp32, of values next to nothing, and with NaN or infinity (their own row alone)."""
    dh = 128
    X = torch.randn(6, 2, dh, generator=torch.Generator().manual_seed(3))
    X[0] = 0
    X[1] *= 1e30
    X[2] *= 1e-30
    X[3, 0, 5] = float("nan")
    X[4, 1, 7] = float("inf")
    for dtype in (torch.float32, torch.bfloat16):
        x = X.to(dtype)
        w = torch.ones(dh)
        q, _ = ctx.head_norm_rotate(x.cuda(), None, w.cuda(), None, eps=0.0 if dtype == torch.float32 else 1e-6)
        q = q.double().cpu().numpy()
        x64 = x.double().numpy()
        for r in (1, 2, 5):
            want = x64[r] / np.sqrt((x64[r] ** 2).mean(-1, keepdims=True) + (0.0 if dtype == torch.float32 else 1e-6))
            assert np.all(np.abs(q[r] - want) <= (torch.finfo(dtype).eps / 2 + 2.0 ** -21) * np.abs(want) + 2.0 ** -133)
        assert np.all(q[0] == 0) if dtype == torch.bfloat16 else np.isnan(q[0]).all()      # 0 / sqrt(0 + eps)
        assert np.isnan(q[3, 0]).all() and np.isfinite(q[3, 1]).all() and np.isfinite(q[4, 0]).all() and np.isnan(q[4, 1, 7])


def test_positions_outside_the_table(ctx, lib):
    X = torch.randn(4, 3, 100, device="cuda")
    for dh, rot in ((100, 52), (96, 32)):
        x = X[..., :dh].contiguous()
        tab = table(10, rot).cuda()
        pos = torch.tensor([-1, 0, 9, 10], dtype=torch.int32, device="cuda")
        y, _ = ctx.head_norm_rotate(x, None, rotation=lib.Rotation(tab), positions=pos)
        bad = torch.isnan(y[..., :rot]).all(-1).all(-1).tolist()
        assert bad == [True, False, False, True] and torch.equal(y[..., rot:], x[..., rot:]) and torch.isfinite(y[1:3]).all()


def test_refusals(ctx, lib):
    x = torch.zeros(2, 2, 64, device="cuda")
    pos = torch.zeros(2, dtype=torch.int32, device="cuda")
    with pytest.raises(lib.TurboBoAError):
        ctx.head_norm_rotate(torch.zeros(2, 1, 300, device="cuda"))
    with pytest.raises(lib.TurboBoAError):
        ctx.head_norm_rotate(x, rotation=lib.Rotation(table(4, 66).cuda()), positions=pos)
    with pytest.raises(lib.TurboBoAError):
        ctx.head_norm_rotate(x, rotation=lib.Rotation(torch.zeros(4, 5, device="cuda")), positions=pos)
    for eps in (-1.0, float("nan")):
        with pytest.raises(lib.TurboBoAError):
            ctx.head_norm_rotate(x, wq=torch.ones(64, device="cuda"), eps=eps)
    assert ctx.head_norm_rotate(x[:0])[0].shape == (0, 2, 64)
