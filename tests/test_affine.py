"""Products with bias, activation and residual or gate behind them (fpdt_tw_affine_*): oracle pins and refusals (no GPU), and GPU parity."""
import os
import re
import subprocess
import tempfile

import numpy as np
import pytest
import torch

from oracle import tokenwise as otw
from paper_2408_16978_amd import build as lib_build
from paper_2408_16978_amd import tokenwise as TW

ACT = {"none": TW.FPDT_TW_ACT_NONE, "gelu": TW.FPDT_TW_ACT_GELU, "silu": TW.FPDT_TW_ACT_SILU}
HALF = 2.0 ** -8  # a rounding to bf16


# ------------------------------------------------------------------ oracle pins (CPU)
@pytest.mark.parametrize("act", ["none", "gelu", "silu"])
@pytest.mark.parametrize("join", ["none", "add", "times"])
def test_oracle_against_autograd_and_differences(act, join):
    r = np.random.default_rng(3)
    X, W, B, R, dY = (r.standard_normal(s) for s in ((5, 7), (6, 7), 6, (5, 6), (5, 6)))
    x, w, b, res = (torch.tensor(a, requires_grad=True) for a in (X, W, B, R))
    z = x @ w.T + b
    z.retain_grad()
    y = {"none": lambda v: v, "gelu": torch.nn.functional.gelu, "silu": torch.nn.functional.silu}[act](z)
    y = y + res if join == "add" else y * res if join == "times" else y
    (y * torch.tensor(dY)).sum().backward()
    out = otw.affine(X, W, B, None if join == "none" else R, act, join == "times")
    back = otw.affine_behind_bwd(out["Z"], R, dY, act, join == "times")
    np.testing.assert_allclose(out["Y"], y.detach().numpy(), rtol=1e-11, atol=1e-12)
    np.testing.assert_allclose(back["dZ"], z.grad.numpy(), rtol=1e-10, atol=1e-12)
    np.testing.assert_allclose(back["dB"], b.grad.numpy(), rtol=1e-10, atol=1e-12)
    if join != "none":
        np.testing.assert_allclose(back["dR"], res.grad.numpy(), rtol=1e-10, atol=1e-12)
    lin = otw.linear(X, W, back["dZ"])
    np.testing.assert_allclose(lin["dW"], w.grad.numpy(), rtol=1e-10, atol=1e-12)
    for i in (0, 4):
        d = np.zeros(6)
        d[i] = 1e-6
        loss = lambda b_: (otw.affine(X, W, b_, None if join == "none" else R, act, join == "times")["Y"] * dY).sum()
        assert abs((loss(B + d) - loss(B - d)) / 2e-6 - back["dB"][i]) < 1e-7


# ------------------------------------------------------------------ refusals (CPU)
def _fwd(**kw):
    a = dict(X=0x10000000, W=0x20000000, B=0x1000, R=0x30000000, Z=0x40000000, Y=0x50000000, rows=8, n_in=64, n_out=32, act=1, join=0, ws=0x60000000, wsb=1 << 30)
    a.update(kw)
    return TW.load().fpdt_tw_affine_fwd(*[a[k] for k in ("X", "W", "B", "R", "Z", "Y", "rows", "n_in", "n_out", "act", "join", "ws", "wsb")], None)


def _bwd(**kw):
    a = dict(Z=0x10000000, R=0x20000000, dY=0x30000000, dZ=0x40000000, dR=0x50000000, dB=0x60000000, rows=8, n_out=32, act=1, join=1, offsets=None, experts=1, ws=0x70000000,
             wsb=1 << 30)
    a.update(kw)
    return TW.load().fpdt_tw_affine_bwd(*[a[k] for k in ("Z", "R", "dY", "dZ", "dR", "dB", "rows", "n_out", "act", "join", "offsets", "experts", "ws", "wsb")], None)


@pytest.mark.parametrize("status,bad", [
    (1, dict(X=None)), (1, dict(W=None)), (1, dict(Y=None)), (1, dict(rows=0)), (1, dict(n_in=0)), (1, dict(n_out=-8)), (1, dict(act=3)), (1, dict(act=-1)), (1, dict(join=2)),
    (1, dict(join=1, R=None)), (1, dict(Y=0x50000001)), (1, dict(B=0x1001)), (1, dict(X=0x10000002)), (1, dict(W=0x20000008)), (1, dict(Y=0x40000010)), (1, dict(Y=0x10000010)),
    (1, dict(Z=0x30000000)), (1, dict(Y=0x30000010)), (1, dict(Y=0x60000000)), (1, dict(Z=0x20000010)), (1, dict(Y=0x1000)), (1, dict(X=0x60000000)),
    (2, dict(rows=1 << 31)), (2, dict(n_in=(1 << 22) + 8)), (2, dict(n_out=(1 << 22) + 8)), (3, dict(ws=None)), (3, dict(ws=0x60000010)), (3, dict(wsb=255))])
def test_forward_refused(status, bad):
    assert _fwd(**bad) == status and TW.fpdt_tw_last_error() != ""


@pytest.mark.parametrize("status,bad", [
    (1, dict(dY=None)), (1, dict(Z=None)), (1, dict(dZ=None)), (1, dict(R=None)), (1, dict(rows=0)), (1, dict(n_out=0)), (1, dict(act=7)), (1, dict(join=-1)),
    (1, dict(join=0)), (1, dict(experts=0)), (1, dict(experts=2)), (1, dict(join=0, act=0, dR=None, dZ=None, dB=None)), (1, dict(dB=0x60000002)), (1, dict(dZ=0x40000001)),
    (1, dict(offsets=0x1002)), (1, dict(dZ=0x50000000)), (1, dict(dZ=0x10000010)), (1, dict(dB=0x30000000)), (1, dict(dR=0x70000000)), (1, dict(offsets=0x40000000, experts=4)),
    (2, dict(rows=1 << 31)), (2, dict(n_out=(1 << 22) + 1)), (2, dict(offsets=0x1000, experts=1025)), (3, dict(ws=None)), (3, dict(ws=0x70000080)), (3, dict(wsb=100))])
def test_backward_refused(status, bad):
    assert _bwd(**bad) == status and TW.fpdt_tw_last_error() != ""


def test_workspace_bytes_and_binding():
    F, B = TW.fpdt_tw_affine_workspace_bytes, TW.fpdt_tw_affine_bwd_workspace_bytes
    assert F(0, 8, 8) == F(8, 0, 8) == F(8, 8, 0) == F(1 << 31, 8, 8) == F(8, (1 << 22) + 1, 8) == F(8, 1 << 32, 8) == 0
    assert B(0, 8) == B(8, 0) == B(8, 8, 0) == B(8, 8, 1025) == B(1 << 31, 8) == B(8, (1 << 32) + 8) == 0
    # copies only where rows are no multiple of 16 bytes, of 32768 rows of X at a time
    assert F(1 << 20, 64, 256) < 1 << 28 and F(1 << 20, 4095, 256) - F(1 << 15, 4095, 256) < 1 << 28
    assert B(1 << 20, 4096) <= 2049 * 4096 * 4
    x = torch.zeros(4, 8, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="current device"):
        TW.fpdt_tw_affine_fwd(x, x, None, None, None, x.clone())
    with pytest.raises(ValueError, match="current device"):
        TW.fpdt_tw_affine_bwd(x, None, x, x, None, None)


@pytest.mark.parametrize("source,count,requests", [("tw_affine.hip", 15, 15), ("tw_experts_gemm.hip", 12, 27), ("tw_experts_gemm_bwd.hip", 8, 0)])
def test_compiler_moves_no_accumulator(source, count, requests):
    """As for the other products: from the first MFMA of a tile loop to the wait behind its last one no instruction of the compiler's may touch an accumulation
    register, and every address that a copy takes from scalar registers is in some.  What joins a whole tile is requested in front of the last two stages by as many
    loads as the wait for the last copies counts: four rows of accumulator tiles of four accesses (256, 192 and 128 rows), two of four (64 rows), four of two (128 columns),
    in one block of instructions for each tile loop."""
    with tempfile.TemporaryDirectory() as d:
        out = os.path.join(d, "x.s")
        subprocess.run([lib_build.HIPCC] + lib_build.FLAGS + ["-S", "--cuda-device-only", os.path.join(lib_build.SRC_DIR, source), "-o", out], check=True, capture_output=True)
        with open(out) as f:
            text = f.read()
    kernels = [k for k in re.findall(r"^(_ZN\S*):(.*?)^\.Lfunc_end", text, re.S | re.M) if "global_load_lds" in k[1]]
    assert len(kernels) == count
    for name, k in kernels:
        loops = False  # from an MFMA on, until the wait
        for line in (line.split(";")[0].strip() for line in k.splitlines()):
            if "v_mfma" in line:
                loops = True
            elif line == "s_nop 15":
                loops = False
            assert not (loops and ("accvgpr" in line or "scratch" in line)), (name, line)
            assert not re.match(r"s_mov_b64 s\[[0-9:]+\], v", line), (name, line)
        assert not loops, name
    found = 0
    for _, k in kernels:
        lines = [x for x in (line.split(";")[0].strip() for line in k.splitlines()) if x]
        starts = [i for i, x in enumerate(lines) if x.startswith(".LBB")] + [len(lines)]
        for a, b in zip(starts, starts[1:]):
            loads = sum(x.startswith("global_load_dwordx4") for x in lines[a:b])
            found += loads in (8, 16) and not any("accvgpr_read" in x for x in lines[a:b])
    assert found == requests


# ------------------------------------------------------------------ parity (GPU)
def f64(t):
    return None if t is None else t.double().cpu().numpy()


def _make(rows, n_in, n_out, seed, std=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    half = lambda *s, std=1.0: (torch.randn(*s, device="cuda", generator=g) * std).to(torch.bfloat16)
    return half(rows, n_in, std=std), half(n_out, n_in, std=n_in ** -0.5), half(n_out), half(rows, n_out), half(rows, n_out)


def budget_fwd(X, W, B, R, ref, act, times, k):
    """z: k products that fp32 holds exactly, their sums and the bias's: k + 2 roundings of 2^-24 of the sum of sizes at most.  The activation's slope is at
    most 1.13; it is right to 2^-20 of its value and what the exponential makes of its argument's roundings (z^2 / 2 or z, three of 2^-24: 2^-23 (1 + z^2) at
    most), and 2^-22 more for the joining operation; then one rounding to bf16."""
    size = np.abs(f64(X)) @ np.abs(f64(W)).T + (0.0 if B is None else np.abs(f64(B)))
    dz = (k + 2) * 2.0 ** -24 * size
    y = np.abs(otw.activation(ref["Z"], act)[0])
    dy = (1.0 if act == "none" else 1.13) * dz + (2.0 ** -20 + 2.0 ** -23 * (1 + ref["Z"] ** 2)) * y
    r = 0.0 if R is None else np.abs(f64(R))
    dy = dy * r if times and R is not None else dy
    return dz + HALF * np.abs(ref["Z"]), dy + (HALF + 2.0 ** -22) * np.abs(ref["Y"]) + 2.0 ** -22 * (y + r) * (R is not None)


def _close(name, got, ref, tol):
    off = np.abs(f64(got) - ref)
    assert np.isfinite(f64(got)).all() and (off <= tol).all(), (name, off.max(), (off - tol).max())


SIZES = [(1, 8, 8), (1, 1, 1), (3, 7, 5), (16, 64, 32), (17, 72, 40), (64, 32, 256), (65, 63, 129), (33, 129, 77), (130, 257, 264), (257, 520, 300), (300, 96, 515), (16, 2048, 512),
         (5, 4000, 136), (700, 1000, 1032)]


@pytest.mark.gpu
@pytest.mark.parametrize("rows,n_in,n_out", SIZES)
@pytest.mark.parametrize("act", ["none", "gelu", "silu"])
def test_gpu_forward(rows, n_in, n_out, act):
    X, W, B, R, _ = _make(rows, n_in, n_out, rows + n_in)
    ws = torch.empty(TW.fpdt_tw_affine_workspace_bytes(rows, n_in, n_out), dtype=torch.uint8, device="cuda")
    for b, r, times, keep in ((None, None, False, False), (B, R, False, True), (B, R, True, True), (None, R, True, False), (B, None, False, True)):
        print("[case] affine", rows, n_in, n_out, act, b is not None, r is not None, times, flush=True)
        Y, Z = (torch.full((rows, n_out), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        TW.fpdt_tw_affine_fwd(X, W, b, r, Z if keep else None, Y, ACT[act], TW.FPDT_TW_JOIN_TIMES if times else TW.FPDT_TW_JOIN_ADD, ws)
        torch.cuda.synchronize()
        ref = otw.affine(f64(X), f64(W), f64(b), f64(r), act, times)
        tz, ty = budget_fwd(X, W, b, r, ref, act, times, n_in)
        _close("Y", Y, ref["Y"], ty)
        if keep:
            _close("Z", Z, ref["Z"], tz)
        else:
            assert torch.isnan(Z).all()
        # the same bits again; in R's place
        Y2 = torch.empty_like(Y) if r is None else r.clone()
        TW.fpdt_tw_affine_fwd(X, W, b, None if r is None else Y2, None, Y2, ACT[act], TW.FPDT_TW_JOIN_TIMES if times else TW.FPDT_TW_JOIN_ADD, ws)
        torch.cuda.synchronize()
        assert torch.equal(Y2, Y)


def reference(X, W, B, R, act, times):
    """The forward in 64 bits on the GPU, with what budget_fwd allows (sizes that numpy's erf would take long for)."""
    z = X.double() @ W.double().t() + (0.0 if B is None else B.double())
    y = {"none": lambda v: v, "gelu": lambda v: v * torch.special.erfc(-v / 2 ** 0.5) / 2, "silu": lambda v: v * torch.sigmoid(v)}[act](z)
    dz = (X.shape[1] + 2) * 2.0 ** -24 * (X.double().abs() @ W.double().abs().t() + (0.0 if B is None else B.double().abs()))
    dy = 1.13 * dz + (2.0 ** -20 + 2.0 ** -23 * (1 + z * z)) * y.abs()
    r = None if R is None else R.double()
    if r is not None:
        y, dy = (y * r, dy * r.abs()) if times else (y + r, dy + 2.0 ** -22 * (y.abs() + r.abs()))
    return y, dy + (HALF + 2.0 ** -22) * y.abs(), z, dz + HALF * z.abs()


@pytest.mark.gpu
@pytest.mark.parametrize("rows,n_out", [(4096, 4096), (2500, 4104), (1500, 6144), (600, 1024), (16001, 1280)])
@pytest.mark.parametrize("n_in", [8, 40, 64, 72, 128, 136, 192, 200, 264, 448, 1000])
def test_gpu_forward_of_large_tiles(rows, n_out, n_in):
    """Tiles of every height, whole and cut off, over one, two and three stages of k, whole and cut off: what joins a tile is requested in front of the last two."""
    X, W, B, R, _ = _make(rows, n_in, n_out, n_in)
    ws = torch.empty(TW.fpdt_tw_affine_workspace_bytes(rows, n_in, n_out), dtype=torch.uint8, device="cuda")
    print("[case] large tiles", rows, n_in, n_out, flush=True)
    for b, r, act, times in ((B, R, "silu", True), (None, R, "none", False), (B, None, "gelu", False)):
        Y, Z = (torch.full((rows, n_out), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        TW.fpdt_tw_affine_fwd(X, W, b, r, Z, Y, ACT[act], TW.FPDT_TW_JOIN_TIMES if times else TW.FPDT_TW_JOIN_ADD, ws)
        y, ty, z, tz = reference(X, W, b, r, act, times)
        assert bool(((Y.double() - y).abs() <= ty).all()) and bool(((Z.double() - z).abs() <= tz).all()), (act, times)


@pytest.mark.gpu
@pytest.mark.parametrize("n_in,n_out", [(64, 48), (63, 47)])
def test_gpu_forward_off_alignment_and_no_further(n_in, n_out):
    """B, R, Z and Y one element behind a boundary (X and W too, where they are copied); what lies around them stays."""
    rows = 70
    X, W, B, R, _ = _make(rows, n_in, n_out, 3)
    need = TW.fpdt_tw_affine_workspace_bytes(rows, n_in, n_out)
    room = torch.full((need + 512,), 77, dtype=torch.uint8, device="cuda")
    Y, Z = torch.empty_like(R), torch.empty_like(R)
    TW.fpdt_tw_affine_fwd(X, W, B, R, Z, Y, ACT["gelu"], TW.FPDT_TW_JOIN_TIMES, room[:need])
    def off(t):
        b = torch.full((t.numel() + 2,), 9.0, dtype=t.dtype, device="cuda")
        v = b[1:-1].view(t.shape)
        v.copy_(t)
        return v, b
    (B2, _), (R2, _), (Y2, yb), (Z2, zb) = (off(t) for t in (B, R, Y * 0, Z * 0))
    X2, W2 = (X, W) if n_in % 8 == 0 else (off(X)[0], off(W)[0])
    TW.fpdt_tw_affine_fwd(X2, W2, B2, R2, Z2, Y2, ACT["gelu"], TW.FPDT_TW_JOIN_TIMES, room[:need])
    torch.cuda.synchronize()
    assert torch.equal(Y2, Y) and torch.equal(Z2, Z) and all(b[0] == b[-1] == 9 for b in (yb, zb)) and (room[need:] == 77).all()
    with pytest.raises(TW.FpdtTwError) as e:
        TW.fpdt_tw_affine_fwd(X, W, B, R, Z, Y, ACT["gelu"], TW.FPDT_TW_JOIN_TIMES, room[:need - 1])
    assert e.value.status == 3


@pytest.mark.gpu
def test_gpu_activations_over_all_of_bf16():
    """Every finite bf16 number as z (one product with 1): the activation is right to 2^-20 + 2^-23 (1 + z^2) of its value before it is rounded (SILU:
    |z| for z^2), in the tails too, until the share that it multiplies z with is below the smallest normal number (|z| < 128 there); infinities and NaN go where
    the formulas send them."""
    z = torch.arange(1 << 16, dtype=torch.int32, device="cuda").to(torch.int16).view(torch.bfloat16)
    X = torch.zeros(1 << 16, 8, dtype=torch.bfloat16, device="cuda")
    X[:, 0] = torch.where(torch.isfinite(z), z, torch.zeros_like(z))
    W = torch.zeros(8, 8, dtype=torch.bfloat16, device="cuda")
    W[0, 0] = 1.0
    ws = torch.empty(TW.fpdt_tw_affine_workspace_bytes(1 << 16, 8, 8), dtype=torch.uint8, device="cuda")
    Y, dZ = torch.empty_like(X), torch.empty_like(X)
    Z = X.clone()
    one = torch.ones_like(X)
    for act in ("gelu", "silu"):
        TW.fpdt_tw_affine_fwd(X, W, None, None, None, Y, ACT[act], workspace=ws)
        TW.fpdt_tw_affine_bwd(Z, None, one, dZ, None, None, ACT[act])
        torch.cuda.synchronize()
        x = f64(X[:, 0])
        y, slope = otw.activation(x, act)
        low = 2.0 ** -126 * 128
        grows = np.minimum(np.abs(x) if act == "silu" else x * x, 2.0 ** 14)
        assert (np.abs(f64(Y[:, 0]) - y) <= (HALF + 2.0 ** -20 + 2.0 ** -23 * (1 + grows) * (x < 0)) * np.abs(y) + low).all(), act
        # a slope is a sum of two terms of |x| and less
        ok = np.abs(x) < 1e18
        assert (np.abs(f64(dZ[:, 0]) - slope) <= HALF * np.abs(slope) + 2.0 ** -20 * np.minimum(1 + np.abs(x), 64) * np.exp(-np.minimum(np.abs(x), 80) / 2) + 2.0 ** -20 * np.abs(slope) + low)[ok].all(), act
    # not finite: in the bias, so that a product of it with 0 is not made
    X = torch.zeros(1, 8, dtype=torch.bfloat16, device="cuda")
    B = torch.tensor([float("inf"), float("nan"), 0, 1, 2, 3, 4, 5], device="cuda").bfloat16()
    for act in ("none", "gelu", "silu"):
        TW.fpdt_tw_affine_fwd(X, W, B, None, None, Y[:1], ACT[act], workspace=ws)
        torch.cuda.synchronize()
        assert Y[0, 0] == float("inf") and torch.isnan(Y[0, 1]) and torch.isfinite(Y[0, 2:]).all()


def budget_bwd(Z, R, dY, ref, act, times, slice_rows):
    """Slopes and activations are right to 2^-20 (1 + |z|) and 2^-20 of their value; products 2^-22; one rounding.  The columns' sums: a rounding of
    2^-24 of the sum of sizes for each row of a workgroup's slice and 32 for what its threads have, then 64 bits and one rounding."""
    g = np.abs(f64(dY)) * (np.abs(f64(R)) if times else 1.0)
    dz = 2.0 ** -20 * g * (1 + (0.0 if Z is None else np.minimum(np.abs(f64(Z)), 64))) + 2.0 ** -22 * np.abs(ref["dZ"])
    return dz, dz + HALF * np.abs(ref["dZ"]), dz.sum(axis=0) + (slice_rows + 34) * 2.0 ** -24 * np.abs(ref["dZ"]).sum(axis=0)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,n_out", [(1, 1), (1, 8), (3, 5), (16, 64), (33, 77), (70, 2048), (64, 2050), (1000, 264), (5000, 40), (300, 4100)])
@pytest.mark.parametrize("act", ["none", "gelu", "silu"])
@pytest.mark.parametrize("times", [False, True])
def test_gpu_backward(rows, n_out, act, times):
    g = torch.Generator(device="cuda").manual_seed(rows + n_out)
    Z, R, dY = ((torch.randn(rows, n_out, device="cuda", generator=g) * s).to(torch.bfloat16) for s in (2.0, 1.0, 0.1))
    if not times:
        R = None
    if act == "none" and not times:
        Z = None
    join = TW.FPDT_TW_JOIN_TIMES if times else TW.FPDT_TW_JOIN_ADD
    ref = otw.affine_behind_bwd(f64(Z), f64(R), f64(dY), act, times)
    ws = torch.empty(TW.fpdt_tw_affine_bwd_workspace_bytes(rows, n_out), dtype=torch.uint8, device="cuda")
    dZ, dR, dB = torch.empty_like(dY), torch.empty_like(dY) if times else None, torch.full((n_out,), 0.5, device="cuda")
    TW.fpdt_tw_affine_bwd(Z, R, dY, dZ, dR, dB, ACT[act], join, workspace=ws)
    torch.cuda.synchronize()
    _, tz, tb = budget_bwd(Z, R, dY, ref, act, times, 64)
    _close("dZ", dZ, ref["dZ"], tz + 2.0 ** -126)
    _close("dB", dB, 0.5 + ref["dB"], tb + 2.0 ** -24 * np.abs(0.5 + ref["dB"]))
    if times:
        _close("dR", dR, ref["dR"], (HALF + 2.0 ** -19) * np.abs(ref["dR"]) + 2.0 ** -126)
    # the same bits without the sums, in Z's place and in dY's (dR in R's); the sums alone
    for k in (0, 1):
        z, d, r = None if Z is None else Z.clone(), dY.clone(), None if R is None else R.clone()
        out = z if k == 0 and z is not None else d
        TW.fpdt_tw_affine_bwd(z, r, d, out, r, None, ACT[act], join)
        torch.cuda.synchronize()
        assert torch.equal(out, dZ) and (r is None or torch.equal(r, dR))
    if Z is None:
        dB2 = torch.full((1, n_out), 0.5, device="cuda")
        TW.fpdt_tw_affine_bwd(None, None, dY, None, None, dB2, workspace=ws)
        torch.cuda.synchronize()
        assert torch.equal(dB2[0], dB)


@pytest.mark.gpu
@pytest.mark.parametrize("n_out", [40, 2056])
def test_gpu_backward_of_experts_rows(n_out):
    """Experts whose rows end within a slice, that have none, or all; rows without an expert are left as they were."""
    for counts in ([3, 0, 70, 0, 0, 1, 130, 0], [0, 0, 0, 0], [0, 300], [1] * 200, [0] * 500 + [97] + [0] * 523):
        used, E = sum(counts), len(counts)
        rows = used + 5
        g = torch.Generator(device="cuda").manual_seed(E)
        Z, R, dY = ((torch.randn(rows, n_out, device="cuda", generator=g) * s).to(torch.bfloat16) for s in (2.0, 1.0, 0.1))
        ends = np.concatenate([[0], np.cumsum(counts)])
        offsets = torch.tensor(ends, dtype=torch.int32, device="cuda")
        need = TW.fpdt_tw_affine_bwd_workspace_bytes(rows, n_out, E)
        room = torch.full((need + 256,), 77, dtype=torch.uint8, device="cuda")
        dZ, dR = torch.full_like(dY, 9.0), torch.full_like(dY, 9.0)
        dB = torch.randn(E, n_out, device="cuda", generator=g)
        was = f64(dB)
        TW.fpdt_tw_affine_bwd(Z, R, dY, dZ, dR, dB, ACT["gelu"], TW.FPDT_TW_JOIN_TIMES, offsets, room[:need])
        torch.cuda.synchronize()
        ref = otw.affine_behind_bwd(f64(Z), f64(R), f64(dY), "gelu", True)
        raw, tz, _ = budget_bwd(Z, R, dY, ref, "gelu", True, 64)
        _close("dZ", dZ[:used], ref["dZ"][:used], tz[:used])
        assert (dZ[used:] == 9).all() and (dR[used:] == 9).all() and (room[need:] == 77).all()
        for e in range(E):
            part = slice(ends[e], ends[e + 1])
            want = was[e] + ref["dZ"][part].sum(axis=0)
            _close("dB", dB[e], want, raw[part].sum(axis=0) + 98 * 2.0 ** -24 * np.abs(ref["dZ"][part]).sum(axis=0) + 2.0 ** -24 * np.abs(want))


@pytest.mark.gpu
def test_gpu_backward_matches_differences_of_the_forward():
    """The gradient of sum(dY Y) with respect to the bias, against differences of the forward, whose z is exact here (sums of small whole numbers): a step of
    2^-4 in b, Y rounded to bf16 at both ends, and the third derivative's share of the step."""
    rows, n = 512, 8
    X, W = torch.zeros(rows, 8, dtype=torch.bfloat16, device="cuda"), torch.zeros(n, 8, dtype=torch.bfloat16, device="cuda")
    X[:, 0] = (torch.arange(rows, device="cuda") % 33 - 16).float().div(8).bfloat16()
    W[:, 0] = 1.0
    ws = torch.empty(TW.fpdt_tw_affine_workspace_bytes(rows, 8, n), dtype=torch.uint8, device="cuda")
    wb = torch.empty(TW.fpdt_tw_affine_bwd_workspace_bytes(rows, n), dtype=torch.uint8, device="cuda")
    dY = torch.ones(rows, n, dtype=torch.bfloat16, device="cuda")
    for act in ("gelu", "silu"):
        ys = []
        for b in (2.0 ** -4, -2.0 ** -4, 0.0):
            Y, Z = torch.empty_like(dY), torch.empty_like(dY)
            TW.fpdt_tw_affine_fwd(X, W, torch.full((n,), b, device="cuda").bfloat16(), None, Z, Y, ACT[act], workspace=ws)
            ys.append(f64(Y))
        dB, dZ = torch.zeros(n, device="cuda"), torch.empty_like(dY)
        TW.fpdt_tw_affine_bwd(Z, None, dY, dZ, None, dB, ACT[act], workspace=wb)
        torch.cuda.synchronize()
        # |Y| <= 2.1: half a step is 2^-7 at most and 2^-8 |y| each; |act'''| < 2, times h^2 / 6
        tol = (HALF * (np.abs(ys[0]) + np.abs(ys[1])).sum(axis=0) / 2 ** -3 + rows * 2 * 2.0 ** -8 / 6)
        assert (np.abs((ys[0] - ys[1]).sum(axis=0) / 2 ** -3 - f64(dB)) <= tol).all()


@pytest.mark.gpu
@pytest.mark.parametrize("rows,n_in,n_out", [(270000, 64, 8192), (33000, 1001, 513), (40000, 63, 8)])
def test_gpu_forward_of_many_rows(rows, n_in, n_out):
    """Outputs of more than 2^31 elements; X copied in pieces of 32768 rows: rows at the ends and around what separates them."""
    X, W, B, R, _ = _make(rows, n_in, n_out, 1)
    ws = torch.empty(TW.fpdt_tw_affine_workspace_bytes(rows, n_in, n_out), dtype=torch.uint8, device="cuda")
    TW.fpdt_tw_affine_fwd(X, W, B, R, None, R, ACT["silu"], TW.FPDT_TW_JOIN_ADD, ws)
    Y = R
    _, _, _, R, _ = _make(rows, n_in, n_out, 1)
    torch.cuda.synchronize()
    at = torch.tensor([0, 1, 32767, 32768, rows // 2, rows - 257, rows - 1], device="cuda")
    ref = otw.affine(f64(X[at]), f64(W), f64(B), f64(R[at]), "silu")
    _close("Y", Y[at], ref["Y"], budget_fwd(X[at], W, B, R[at], ref, "silu", False, n_in)[1])


@pytest.mark.gpu
def test_gpu_two_streams_and_captured():
    """Calls on two streams at once, each with its own workspace, give the bits of one alone; captured and replayed with new inputs."""
    rows, n_in, n_out = 500, 1000, 1032
    X, W, B, R, dY = _make(rows, n_in, n_out, 4)
    def buffers():
        return dict(Y=torch.empty_like(R), Z=torch.empty_like(R), dZ=torch.empty_like(R), dR=torch.empty_like(R), dB=torch.zeros(n_out, device="cuda"),
                    ws=torch.empty(TW.fpdt_tw_affine_workspace_bytes(rows, n_in, n_out), dtype=torch.uint8, device="cuda"),
                    wb=torch.empty(TW.fpdt_tw_affine_bwd_workspace_bytes(rows, n_out), dtype=torch.uint8, device="cuda"))
    def step(b, stream=None):
        TW.fpdt_tw_affine_fwd(X, W, B, R, b["Z"], b["Y"], ACT["gelu"], TW.FPDT_TW_JOIN_TIMES, b["ws"], stream=stream)
        TW.fpdt_tw_affine_bwd(b["Z"], R, dY, b["dZ"], b["dR"], b["dB"], ACT["gelu"], TW.FPDT_TW_JOIN_TIMES, workspace=b["wb"], stream=stream)
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
        assert all(torch.equal(a[k], b[k]) for k in ("Y", "Z", "dZ", "dR", "dB"))
    for t in (a, b, c):
        t["dB"].zero_()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    step(b, streams[0])
    step(c, streams[1])
    torch.cuda.synchronize()
    step(a)
    torch.cuda.synchronize()
    assert all(torch.equal(a[k], t[k]) for t in (b, c) for k in ("Y", "Z", "dZ", "dR", "dB"))


@pytest.mark.gpu
@pytest.mark.parametrize("n_out", [40, 2056, 77])
@pytest.mark.parametrize("counts,first", [([5, 40, 0, 60], 10), ([5, 40, 0, 60], 16), ([0, 0, 30, 1], 64), ([70, 0, 90], 100), ([1] * 50, 130), ([0, 0], 30), ([100], 7), ([64], 64)])
def test_gpu_backward_of_experts_that_begin_behind_other_rows(n_out, counts, first):
    """A part of sorted offsets, the first of them not 0: within a slice of rows (64 of them at 40 and 77 columns, 16 at 2056), at its end, some slices in.  The rows in front
    (and behind) are another's: not read (they hold NaN), not written, in no sum."""
    E, used = len(counts), sum(counts)
    ends = first + np.concatenate([[0], np.cumsum(counts)])
    rows = first + used + 9
    g = torch.Generator(device="cuda").manual_seed(first)
    Z, R, dY = ((torch.randn(rows, n_out, device="cuda", generator=g) * s).to(torch.bfloat16) for s in (2.0, 1.0, 0.1))
    every = torch.tensor([0, first // 2] + list(ends) + [rows], dtype=torch.int32, device="cuda")  # (those of all experts)
    offsets, mine = every[2:-1], slice(first, first + used)
    ref = otw.affine_behind_bwd(f64(Z), f64(R), f64(dY), "gelu", True)
    raw, tz, _ = budget_bwd(Z, R, dY, ref, "gelu", True, 64)
    plain = f64(dY)
    for t in (Z, R, dY):
        t[:first], t[first + used:] = float("nan"), float("nan")
    ws = torch.empty(TW.fpdt_tw_affine_bwd_workspace_bytes(rows, n_out, E), dtype=torch.uint8, device="cuda")
    dZ, dR = torch.full_like(dY, 9.0), torch.full_like(dY, 9.0)
    dB = torch.randn(E, n_out, device="cuda", generator=g)
    sums, was = dB.clone(), f64(dB)
    TW.fpdt_tw_affine_bwd(Z, R, dY, dZ, dR, dB, ACT["gelu"], TW.FPDT_TW_JOIN_TIMES, offsets, ws)
    TW.fpdt_tw_affine_bwd(None, None, dY, None, None, sums, offsets=offsets, workspace=ws)
    torch.cuda.synchronize()
    _close("dZ", dZ[mine], ref["dZ"][mine], tz[mine] + 2.0 ** -126)
    _close("dR", dR[mine], ref["dR"][mine], (HALF + 2.0 ** -19) * np.abs(ref["dR"][mine]) + 2.0 ** -126)
    for t in (dZ, dR):
        assert (t[:first] == 9).all() and (t[first + used:] == 9).all()
    for e in range(E):
        part = slice(ends[e], ends[e + 1])
        want = was[e] + ref["dZ"][part].sum(axis=0)
        _close("dB", dB[e], want, raw[part].sum(axis=0) + 98 * 2.0 ** -24 * np.abs(ref["dZ"][part]).sum(axis=0) + 2.0 ** -24 * np.abs(want))
        want = was[e] + plain[part].sum(axis=0)
        _close("sums alone", sums[e], want, 98 * 2.0 ** -24 * np.abs(plain[part]).sum(axis=0) + 2.0 ** -24 * np.abs(want))
