"""Normalisation with the residual add (fpdt_tw_norm_*): oracle pins and refusals (no GPU), and GPU parity."""
import math

import numpy as np
import pytest
import torch

from oracle import tokenwise as otw
from paper_2408_16978_amd import tokenwise as TW

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


# ------------------------------------------------------------------ oracle pins (CPU)
@pytest.mark.parametrize("layer", [False, True])
def test_oracle_against_autograd_and_differences(layer):
    r = np.random.default_rng(3)
    S, W, B, dY, dR = (r.standard_normal(s) for s in ((5, 9), 9, 9, (5, 9), (5, 9)))
    out = otw.norm(S, W, B if layer else None, 1e-3, layer, dY, dR)
    s, w, b = (torch.tensor(a, requires_grad=True) for a in (S, W, B))
    y = torch.nn.functional.layer_norm(s, (9,), w, b, 1e-3) if layer else torch.nn.functional.rms_norm(s, (9,), w, 1e-3)
    ((y * torch.tensor(dY)).sum() + (s * torch.tensor(dR)).sum()).backward()
    np.testing.assert_allclose(out["Y"], y.detach().numpy(), rtol=1e-11, atol=1e-12)
    for k, t in (("dX", s), ("dW", w)) + ((("dB", b),) if layer else ()):
        np.testing.assert_allclose(out[k], t.grad.numpy(), rtol=1e-10, atol=1e-12, err_msg=k)
    loss = lambda S_, W_: (otw.norm(S_, W_, B if layer else None, 1e-3, layer)["Y"] * dY).sum() + (S_ * dR).sum()
    for at in ((0, 0), (3, 7)):
        d = np.zeros_like(S)
        d[at] = 1e-6
        assert abs((loss(S + d, W) - loss(S - d, W)) / 2e-6 - out["dX"][at]) < 1e-7


# ------------------------------------------------------------------ refusals (CPU)
def _fwd(**kw):
    a = dict(X=0x10000000, R=0x20000000, W=0x1000, B=None, S=0x30000000, Y=0x40000000, stats=0x50000000, rows=8, hidden=64, kind=0, eps=1e-5, dtype=1)
    a.update(kw)
    return TW.load().fpdt_tw_norm_fwd(*[a[k] for k in ("X", "R", "W", "B", "S", "Y", "stats", "rows", "hidden", "kind", "eps", "dtype")], None)


def _bwd(**kw):
    a = dict(S=0x10000000, W=0x1000, stats=0x2000, dY=0x20000000, dR=0x30000000, dX=0x40000000, dW=0x50000000, dB=None, rows=8, hidden=64, kind=0, dtype=1,
             ws=0x60000000, wsb=1 << 30)
    a.update(kw)
    return TW.load().fpdt_tw_norm_bwd(*[a[k] for k in ("S", "W", "stats", "dY", "dR", "dX", "dW", "dB", "rows", "hidden", "kind", "dtype", "ws", "wsb")], None)


@pytest.mark.parametrize("status,bad", [
    (1, dict(X=None)), (1, dict(W=None)), (1, dict(Y=None)), (1, dict(rows=0)), (1, dict(hidden=0)), (1, dict(hidden=-1)), (1, dict(kind=2)), (1, dict(dtype=7)),
    (1, dict(eps=-1.0)), (1, dict(eps=math.nan)), (1, dict(R=None)), (1, dict(B=0x1100)), (1, dict(X=0x10000001)), (1, dict(stats=0x50000002)),
    (1, dict(Y=0x10000002)), (1, dict(S=0x20000002)), (1, dict(Y=0x30000000)), (1, dict(W=0x40000000)), (1, dict(stats=0x40000000)), (1, dict(stats=0x1000)),
    (2, dict(hidden=16385)), (2, dict(rows=1 << 31))])
def test_forward_refused(status, bad):
    assert _fwd(**bad) == status and TW.fpdt_tw_last_error() != ""


@pytest.mark.parametrize("status,bad", [
    (1, dict(S=None)), (1, dict(W=None)), (1, dict(stats=None)), (1, dict(dY=None)), (1, dict(dX=None)), (1, dict(rows=0)), (1, dict(hidden=0)),
    (1, dict(kind=-1)), (1, dict(dtype=2)), (1, dict(dB=0x51000000)), (1, dict(dW=0x50000002)), (1, dict(dX=0x10000080)), (1, dict(dX=0x1000)),
    (1, dict(dX=0x2000)), (1, dict(dW=0x10000000)), (1, dict(kind=1, dB=0x50000080)), (1, dict(dW=0x60000000)), (1, dict(ws=0x20000000)), (1, dict(dW=0x2000)),
    (2, dict(hidden=16385)), (2, dict(rows=1 << 31)),
    (3, dict(ws=None)), (3, dict(ws=0x60000010)), (3, dict(wsb=8 * 64 * 4 - 1)), (3, dict(kind=1, wsb=2 * 8 * 64 * 4 - 1))])
def test_backward_refused(status, bad):
    assert _bwd(**bad) == status and TW.fpdt_tw_last_error() != ""


def test_workspace_bytes_and_binding():
    W = TW.fpdt_tw_norm_bwd_workspace_bytes
    assert W(8, 64, TW.FPDT_TW_RMSNORM) == 8 * 64 * 4 and W(8, 64, TW.FPDT_TW_LAYERNORM) == 2 * 8 * 64 * 4
    assert W(1 << 20, 4096) <= 1024 * 4096 * 4
    assert W(0, 64) == W(8, 0) == W(8, 16385) == W(8, 64, 5) == W(1 << 31, 64) == 0
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError, match="current device"):
        TW.fpdt_tw_norm_fwd(x, None, x[0], None, None, x.clone(), None, 1e-5)


def test_workspace_is_what_the_backward_writes():
    """16 MiB for each of the sums at most, whatever the width (64 MiB were asked for at 16384 columns); as many workgroups as the widest launch of either
    type has: as many as registers hold at once of 6 waves a SIMD with one access a lane (groups of 4 waves 6 a compute unit, of 8 three), or of 4 with more
    (of 8 waves two, of 12 or 16 one)."""
    W = TW.fpdt_tw_norm_bwd_workspace_bytes
    for hidden in range(1, 16385):
        assert 0 < W(1 << 20, hidden) <= 1 << 24 and W(1 << 20, hidden, TW.FPDT_TW_LAYERNORM) == 2 * W(1 << 20, hidden), hidden
        assert W(5, hidden) == 5 * hidden * 4
    groups = lambda hidden: W(1 << 20, hidden) // (4 * hidden)
    assert [groups(h) for h in (64, 4096, 8192, 12288, 16384)] == [1536, 768, 512, 256, 256]


# ------------------------------------------------------------------ GPU parity
# (a lane of a wave, a quarter wave, several waves; cut-off accesses; one row; every shape of the kernels; the widest)
SIZES = [(1, 1), (3, 5), (1, 4096), (67, 64), (1030, 128), (17, 129), (130, 513), (300, 512), (41, 1000), (2100, 257), (65, 2048), (33, 2560), (37, 4096), (9, 4099),
         (11, 8192), (5, 12000), (3, 16384),
         (70, 200), (50, 384), (2101, 640), (1101, 2560), (40, 5120), (19, 6001), (1027, 1536)]


def _make(rows, hidden, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda *s: torch.randn(*s, device="cuda", generator=g)
    return [t.to(DT[dtype]) for t in (n(rows, hidden) * 2 + n(hidden), n(rows, hidden), 1 + 0.2 * n(hidden), n(hidden), n(rows, hidden), n(rows, hidden))]


def _close(name, got, ref, budget):
    err = np.abs(got.double().cpu().numpy() - ref) / (budget + 1e-300)
    assert err.max() <= 1.0, (name, err.max())


@pytest.mark.gpu
@pytest.mark.parametrize("rows,hidden", SIZES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layer", [False, True])
def test_gpu_forward_and_backward_match_the_oracle(rows, hidden, dtype, layer):
    print("[case] norm", rows, hidden, dtype, layer, flush=True)
    kind, eps, half = (TW.FPDT_TW_LAYERNORM if layer else TW.FPDT_TW_RMSNORM), 1e-5, HALF_STEP[dtype]
    X, R, W, B, dY, dR = _make(rows, hidden, dtype, hidden)
    B = B if layer else None
    S, Y, stats = torch.empty_like(X), torch.empty_like(X), torch.empty((2 if layer else 1, rows), device="cuda")
    TW.fpdt_tw_norm_fwd(X, R, W, B, S, Y, stats, eps, kind)
    torch.cuda.synchronize()
    f64 = lambda t: None if t is None else t.double().cpu().numpy()
    assert torch.equal(S, (X.float() + R.float()).to(X.dtype))
    ref = otw.norm(f64(S), f64(W), f64(B), eps, layer)
    # Sums of `hidden` terms: at most 64 in a lane, 6 + 16 steps over lanes and waves, so 90 roundings of 2^-24 relative to the
    # sum of sizes: 2^-17 of the mean size for the mean, 2^-18 of rstd (half that of the mean square, one root, one quotient);
    # three more products.  2^-17 covers rstd's and the products' share.
    slop = 2.0 ** -17
    s, w = np.abs(f64(S)), np.abs(f64(W))
    size, rstd = s.mean(axis=1, keepdims=True) if layer else 0.0, ref["stats"][-1][:, None]
    # (an error of the mean moves the mean square by its own square only, but with few channels by what rstd makes of it)
    worst = slop * (np.abs(ref["U"]) + rstd * size) * w
    _close("Y", Y, ref["Y"], worst + slop * np.abs(ref["Y"]) + half * np.abs(ref["Y"]))
    _close("rstd", stats[-1], ref["stats"][-1], slop * (ref["stats"][-1] + (ref["stats"][-1] ** 3) * (slop * size[:, 0]) ** 2 * 4 if layer else ref["stats"][-1]))
    if layer:
        _close("mean", stats[0], ref["stats"][0], slop * size[:, 0])
    # backward, by the statistics that the forward left
    dX, dW, dB = torch.empty_like(X), torch.full((hidden,), 0.5, device="cuda"), torch.full((hidden,), -0.5, device="cuda") if layer else None
    ws = torch.empty(TW.fpdt_tw_norm_bwd_workspace_bytes(rows, hidden, kind), dtype=torch.uint8, device="cuda")
    TW.fpdt_tw_norm_bwd(S, W, stats, dY, dR, dX, dW, dB, kind, ws)
    torch.cuda.synchronize()
    st = f64(stats)
    ref = otw.norm(f64(S), f64(W), None, eps, layer, f64(dY), f64(dR), st)
    H, U = np.abs(f64(dY) * f64(W)), np.abs(ref["U"]) + (st[1][:, None] * np.abs(st[0][:, None]) * 2.0 ** -6 if layer else 0.0)
    mean = lambda a: a.mean(axis=1, keepdims=True)
    budget = slop * st[-1][:, None] * (H + (mean(H) if layer else 0.0) + U * mean(H * U)) + slop * np.abs(f64(dR))
    _close("dX", dX, ref["dX"], budget + half * np.abs(ref["dX"]))
    # rows of a workgroup in a row, 16 groups, 64 workgroups of 1024 in a wave of the last sum, 16 waves
    chain = 2.0 ** -24 * (rows / 1024 + 16 + 64 + 16 + 4)
    _close("dW", dW, 0.5 + ref["dW"], chain * (0.5 + (np.abs(f64(dY)) * U).sum(axis=0)))
    if layer:
        _close("dB", dB, -0.5 + ref["dB"], chain * (0.5 + np.abs(f64(dY)).sum(axis=0)))
    # the same bits again, without dR and without sums where they are not wanted; sums alone do not change dX
    dX2, dW2 = torch.empty_like(X), torch.full((hidden,), 0.5, device="cuda")
    TW.fpdt_tw_norm_bwd(S, W, stats, dY, dR, dX2, dW2, None, kind, ws)
    assert torch.equal(dX2, dX) and torch.equal(dW2, dW)
    TW.fpdt_tw_norm_bwd(S, W, stats, dY, None, dX2, None, None, kind)
    torch.cuda.synchronize()
    ref0 = ref["dX"] - f64(dR)
    _close("dX without dR", dX2, ref0, budget + half * np.abs(ref0))
    if layer:
        dB2 = torch.full((hidden,), -0.5, device="cuda")
        TW.fpdt_tw_norm_bwd(S, W, stats, dY, dR, dX2, None, dB2, kind, ws)
        torch.cuda.synchronize()
        assert torch.equal(dB2, dB)


@pytest.mark.gpu
@pytest.mark.parametrize("hidden", [3, 7, 100, 520, 1001, 2560, 5120, 12000, 16383])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gpu_means_of_equal_values_are_that_value(hidden, dtype):
    """Rows of one whole number each, whose sums are whole numbers below 2^24 and so exact in fp32 in any order: a quotient rounded once is
    the number itself, so no deviation is left (LAYERNORM: Y = B, whatever eps makes of a deviation), and a mean square of 1024 or 9 gives its root.
    Backward, equal gradients on a row without deviation: nothing is left of them."""
    value = torch.tensor([1000.0, -1000.0, 3.0, 0.0, 1.0], device="cuda")
    X = value[:, None].expand(-1, hidden).to(DT[dtype]).contiguous()
    W, B = torch.full((hidden,), 1.5, device="cuda").to(DT[dtype]), torch.randn(hidden, device="cuda").to(DT[dtype])
    Y, stats = torch.empty_like(X), torch.empty(2, len(value), device="cuda")
    TW.fpdt_tw_norm_fwd(X, None, W, B, None, Y, stats, 1e-5, TW.FPDT_TW_LAYERNORM)
    torch.cuda.synchronize()
    assert torch.equal(stats[0], value) and torch.equal(Y, B.expand_as(Y))
    one = torch.ones_like(W)
    dY, dX = X.clone(), torch.empty_like(X)
    TW.fpdt_tw_norm_bwd(X, one, stats, dY, None, dX, None, None, TW.FPDT_TW_LAYERNORM)
    torch.cuda.synchronize()
    assert (dX == 0).all()
    # RMSNORM without eps: the mean square is the number's square, and rstd one over the number
    size = torch.tensor([32.0, -32.0, 3.0, 2.0 ** -60, 1.0], device="cuda")
    X = size[:, None].expand(-1, hidden).to(DT[dtype]).contiguous()
    TW.fpdt_tw_norm_fwd(X, None, one, None, None, Y, stats[0], 0.0)
    torch.cuda.synchronize()
    assert torch.equal(stats[0], 1.0 / size.abs()) and torch.equal(Y, torch.sign(size)[:, None].expand_as(Y).to(Y.dtype))


@pytest.mark.gpu
@pytest.mark.parametrize("hidden", [1, 77, 520, 2560, 4096, 16384])
@pytest.mark.parametrize("eps", [0.0, 1e-5, 0.25])
def test_gpu_rstd_is_rounded_once(hidden, eps):
    """Rows of whole numbers, whose squares' sums fp32 holds: rstd is the fp32 number next to 1 / sqrt(sum / hidden + eps).  And where there is none next to it: no
    square at all, squares below the normal numbers, a sum that is infinite."""
    g = torch.Generator(device="cuda").manual_seed(hidden)
    X = torch.randint(-7, 8, (600, hidden), device="cuda", generator=g).float()
    X[:, 0] = torch.randint(1, 100, (600,), device="cuda", generator=g).float()
    W, Y, stats = torch.ones(hidden, device="cuda"), torch.empty_like(X), torch.empty(600, device="cuda")
    TW.fpdt_tw_norm_fwd(X, None, W, None, None, Y, stats, eps)
    torch.cuda.synchronize()
    total = X.double().square().sum(1).cpu().numpy()
    assert total.max() < 2 ** 24
    want = (1.0 / np.sqrt(total / hidden + float(np.float32(eps)))).astype(np.float32)
    assert np.array_equal(stats.cpu().numpy(), want)
    X = X[:4].zero_()
    X[1], X[2], X[3, 0] = 2.0 ** -68, 3e38, math.inf
    TW.fpdt_tw_norm_fwd(X, None, W, None, None, Y[:4], stats[:4], 0.0)
    torch.cuda.synchronize()
    # (2^-136 is held to 13 bits, half a step of which is 2^-14 of it, half that of its root)
    assert stats[0] == math.inf and abs(stats[1].item() * 2.0 ** -68 - 1) <= 2.0 ** -14 and stats[2] == 0 and stats[3] == 0


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [1, 37, 500])
@pytest.mark.parametrize("layer", [False, True])
def test_gpu_sums_over_rows_of_a_workgroup_each_are_rounded_once(rows, layer):
    """Rows of several waves, no more of them than workgroups: a partial sum is one row's dY (U is 1), so dW and dB are sums of fp32 numbers, added in 64 bits
    and rounded once: half a step, and 2^-40 of the sum of sizes for the sums themselves."""
    hidden, kind = 4096, TW.FPDT_TW_LAYERNORM if layer else TW.FPDT_TW_RMSNORM
    g = torch.Generator(device="cuda").manual_seed(rows)
    S, W, stats = torch.ones(rows, hidden, device="cuda"), torch.ones(hidden, device="cuda"), torch.zeros(2 if layer else 1, rows, device="cuda")
    stats[-1] = 1.0
    dY, dX = torch.randn(rows, hidden, device="cuda", generator=g), torch.empty_like(S)
    was = torch.randn(2, hidden, device="cuda", generator=g)
    dW, dB = was[0].clone(), was[1].clone() if layer else None
    ws = torch.empty(TW.fpdt_tw_norm_bwd_workspace_bytes(rows, hidden, kind), dtype=torch.uint8, device="cuda")
    TW.fpdt_tw_norm_bwd(S, W, stats, dY, None, dX, dW, dB, kind, ws)
    torch.cuda.synchronize()
    for got, before in ((dW, was[0]), (dB, was[1])) if layer else ((dW, was[0]),):
        want = before.double() + dY.double().sum(0)
        assert ((got.double() - want).abs() <= 2.0 ** -24 * want.abs() + 2.0 ** -40 * dY.double().abs().sum(0)).all()


@pytest.mark.gpu
@pytest.mark.parametrize("hidden", [64, 1001, 2048, 2056, 4096, 6144, 8192, 12288, 16384])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gpu_workspace_of_the_size_asked_for_and_no_more(hidden, dtype):
    """More rows than there are workgroups (where a wave or less has a row, more than their rows): the bytes behind the workspace stay, and the sums of
    small whole numbers, which fp32 adds exactly in any order, are all there."""
    rows = 1600 if hidden > 1024 else 20000
    g = torch.Generator(device="cuda").manual_seed(hidden)
    S = torch.ones(rows, hidden, dtype=DT[dtype], device="cuda")
    dY = torch.randint(-2, 3, (rows, hidden), device="cuda", generator=g).to(DT[dtype])
    W, stats, dX = torch.ones(hidden, dtype=DT[dtype], device="cuda"), torch.zeros(2, rows, device="cuda"), torch.empty_like(S)
    stats[1] = 1.0
    need = TW.fpdt_tw_norm_bwd_workspace_bytes(rows, hidden, TW.FPDT_TW_LAYERNORM)
    room = torch.full((need + 4096,), 77, dtype=torch.uint8, device="cuda")
    dW, dB = torch.zeros(hidden, device="cuda"), torch.zeros(hidden, device="cuda")
    TW.fpdt_tw_norm_bwd(S, W, stats, dY, None, dX, dW, dB, TW.FPDT_TW_LAYERNORM, room[:need])
    torch.cuda.synchronize()
    want = dY.double().sum(0)
    assert (room[need:] == 77).all() and torch.equal(dW.double(), want) and torch.equal(dB.double(), want)
    with pytest.raises(TW.FpdtTwError) as e:
        TW.fpdt_tw_norm_bwd(S, W, stats, dY, None, dX, dW, dB, TW.FPDT_TW_LAYERNORM, room[:need - 1])
    assert e.value.status == 3


@pytest.mark.gpu
@pytest.mark.parametrize("hidden", [8, 100, 129, 1000, 4096, 12000])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gpu_in_place_without_residual_and_off_alignment(hidden, dtype):
    rows = 21
    X, R, W, B, dY, dR = _make(rows, hidden, dtype, 5)
    Y, S, stats = torch.empty_like(X), torch.empty_like(X), torch.empty(rows, device="cuda")
    TW.fpdt_tw_norm_fwd(X, R, W, None, S, Y, stats, 1e-6)
    # S in X's place and Y in R's; then S nowhere
    X2, R2 = X.clone(), R.clone()
    TW.fpdt_tw_norm_fwd(X2, R2, W, None, X2, R2, None, 1e-6)
    assert torch.equal(X2, S) and torch.equal(R2, Y)
    X2, R2 = X.clone(), R.clone()
    TW.fpdt_tw_norm_fwd(X2, R2, W, None, None, X2, None, 1e-6)
    assert torch.equal(X2, Y) and torch.equal(R2, R)
    # no residual: the norm of S itself
    TW.fpdt_tw_norm_fwd(S.clone(), None, W, None, None, X2, None, 1e-6)
    assert torch.equal(X2, Y)
    # everything one element behind a boundary
    def off(t):
        b = torch.zeros(t.numel() + 2, dtype=t.dtype, device="cuda")
        v = b[1:-1].view(t.shape)
        v.copy_(t)
        return v, b
    (X3, _), (R3, _), (W3, _), (S3, sb), (Y3, yb) = (off(t) for t in (X, R, W, S * 0, Y * 0))
    TW.fpdt_tw_norm_fwd(X3, R3, W3, None, S3, Y3, None, 1e-6)
    assert torch.equal(S3, S) and torch.equal(Y3, Y)
    assert sb[0] == sb[-1] == yb[0] == yb[-1] == 0
    ws = torch.empty(TW.fpdt_tw_norm_bwd_workspace_bytes(rows, hidden), dtype=torch.uint8, device="cuda")
    dX, dW = torch.empty_like(X), torch.zeros(hidden, device="cuda")
    TW.fpdt_tw_norm_bwd(S, W, stats, dY, dR, dX, dW, None, workspace=ws)
    for name in ("S", "dY", "dR"):
        t = {"S": S.clone(), "dY": dY.clone(), "dR": dR.clone()}
        TW.fpdt_tw_norm_bwd(t["S"], W, stats, t["dY"], t["dR"], t[name], None, None)
        assert torch.equal(t[name], dX), name
    (S4, _), (dY4, _), (dR4, _), (dX4, xb), (dW4, wb) = (off(t) for t in (S, dY, dR, dX * 0, dW * 0))
    TW.fpdt_tw_norm_bwd(S4, W3, stats, dY4, dR4, dX4, dW4, None, workspace=ws)
    torch.cuda.synchronize()
    assert torch.equal(dX4, dX) and torch.equal(dW4, dW) and xb[0] == xb[-1] == wb[0] == wb[-1] == 0


@pytest.mark.gpu
@pytest.mark.parametrize("layer", [False, True])
def test_gpu_constant_huge_and_not_finite_rows(layer):
    """A constant row has no deviation (LAYERNORM: 0 times W, plus B); a large offset does not cancel; what is not finite stays
    within its row."""
    kind, hidden = (TW.FPDT_TW_LAYERNORM if layer else TW.FPDT_TW_RMSNORM), 520
    X = torch.randn(6, hidden, device="cuda")
    X[1] = 3.0
    X[2] += 4096.0
    X[3, 7] = math.inf
    X[4, 100] = math.nan
    X[5] = 0.0
    W, B = torch.rand(hidden, device="cuda") + 0.5, torch.randn(hidden, device="cuda")
    Y, stats = torch.empty_like(X), torch.empty((2 if layer else 1, 6), device="cuda")
    TW.fpdt_tw_norm_fwd(X, None, W, B if layer else None, None, Y, stats, 1e-5, kind)
    torch.cuda.synchronize()
    good = [0, 1, 2, 5]
    ref = otw.norm(X[good].double().cpu().numpy(), W.double().cpu().numpy(), B.double().cpu().numpy() if layer else None, 1e-5, layer)
    # row 2 (LAYERNORM): the mean is right to 2^-17 of 4096 = 2^-5 at worst (test above); what the lanes' sums of 32 terms and six
    # steps over lanes make of it, 38 roundings of 2^-24 of 4096: 2^-6.7, of a deviation of 1; U W + B within that and W < 1.5
    tol = np.array([1e-5, 1e-5, 1.5 * 38 * 2.0 ** -12 if layer else 1e-5, 1e-5])[:, None] * (1 + np.abs(ref["Y"]))
    assert (np.abs(Y[good].double().cpu().numpy() - ref["Y"]) <= tol).all()
    if layer:
        assert (Y[1] - B).abs().max() <= 1e-4 and torch.equal(Y[5], B)
    else:
        assert (Y[5] == 0).all()
    assert not torch.isfinite(Y[4]).any()


@pytest.mark.gpu
def test_gpu_captured_and_two_streams():
    """Forward and backward captured, replayed with eager work between; two backwards at once on two streams, each with its
    own workspace, give the bits of one alone."""
    rows, hidden = 700, 1000
    X, R, W, _, dY, dR = _make(rows, hidden, "bf16", 9)
    def buffers():
        return dict(S=torch.empty_like(X), Y=torch.empty_like(X), stats=torch.empty(rows, device="cuda"), dX=torch.empty_like(X), dW=torch.zeros(hidden, device="cuda"),
                    ws=torch.empty(TW.fpdt_tw_norm_bwd_workspace_bytes(rows, hidden), dtype=torch.uint8, device="cuda"))
    def step(b, stream=None):
        TW.fpdt_tw_norm_fwd(X, R, W, None, b["S"], b["Y"], b["stats"], 1e-5, stream=stream)
        TW.fpdt_tw_norm_bwd(b["S"], W, b["stats"], dY, dR, b["dX"], b["dW"], None, workspace=b["ws"], stream=stream)
    a, b, c = buffers(), buffers(), buffers()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(a)
    for _ in range(3):
        X.normal_()
        dY.normal_()
        graph.replay()
        step(b)
        torch.cuda.synchronize()
        assert all(torch.equal(a[k], b[k]) for k in ("S", "Y", "stats", "dX", "dW"))
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for t in (b, c):
        t["dW"].zero_()
    a["dW"].zero_()
    torch.cuda.synchronize()
    step(b, streams[0])
    step(c, streams[1])
    torch.cuda.synchronize()
    step(a)
    torch.cuda.synchronize()
    assert all(torch.equal(a[k], t[k]) for t in (b, c) for k in ("Y", "dX", "dW"))
