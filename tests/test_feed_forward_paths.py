"""Loops and launches of the feed-forward kernels (csrc/tw_affine.hip) that short cases do not reach, each with the rule that sends its sizes there: several steps of four rows in the
backward, few rows over every number of pipelined steps, products with some or all tiles divided along k.  Against 64 bits on the GPU."""
import pytest
import torch

import launch_rules
from paper_2408_16978_amd import tokenwise as TW
from test_affine import ACT, HALF, _make, reference

ADD, TIMES = TW.FPDT_TW_JOIN_ADD, TW.FPDT_TW_JOIN_TIMES


def within(name, got, want, tol):
    off = (got.double() - want).abs()
    assert bool(torch.isfinite(got).all()) and bool((off <= tol).all()), (name, float(off.max()), float((off - tol).max()))


# ------------------------------------------------------------------ backward: slices of many rows
def walk(rows, n_out):
    """(threads along the columns, rows side by side, rows of a slice) of the backward: lanes_of and slice_of of csrc/tw_affine.hip."""
    accesses, cols = -(-n_out // 8), 8
    while cols < 32 and cols < accesses:
        cols *= 2
    if accesses >= 32:
        threads = {c: -(-accesses // c) * c for c in (256, 128, 64, 32)}
        cols = next((c for c, t in threads.items() if t * 8 <= accesses * 9), min(threads, key=threads.get))
    lines, wide = 256 // cols, -(-n_out // (cols * 8))
    most = 1536 // wide if wide < 1536 else 1
    piece = -(-rows // most)
    return cols, lines, -(-piece // lines) * lines if piece > 2 * lines else 2 * lines


LONG = [(8000, 10240), (9001, 4104), (300001, 40), (200003, 77), (20001, 2050), (5003, 14336)]


@pytest.mark.parametrize("rows,n_out", LONG)
def test_long_slices_take_steps_of_four_rows_and_a_rest(rows, n_out):
    _, lines, piece = walk(rows, n_out)
    slices = -(-rows // piece)
    assert TW.fpdt_tw_affine_bwd_workspace_bytes(rows, n_out) == (slices + 1) * n_out * 4 // 256 * 256 + 256 * ((slices + 1) * n_out * 4 % 256 > 0)
    assert piece >= 6 * lines and piece // lines % 4 != 0 and slices > 100


def test_sums_of_long_slices_take_steps_of_eight():
    assert sum(-(-rows // walk(rows, n)[2]) > 7 * 32 + 32 for rows, n in LONG) >= 3


def back(Z, R, dY, act, times):
    """dZ, its allowance, dR, its allowance, and of each dZ the error before it is rounded: slopes are right to 2^-20 (1 + |z|), activations to 2^-20 of their value and what the
    exponential makes of its argument's roundings (2^-23 (1 + z^2)), products to 2^-22; one rounding."""
    g = dY.double()
    dz, raw, dr, tr = g, torch.zeros_like(g), None, None
    if Z is not None:
        z = Z.double().requires_grad_()
        y = {"none": lambda v: v * 1.0, "gelu": lambda v: v * torch.special.erfc(-v / 2 ** 0.5) / 2, "silu": lambda v: v * torch.sigmoid(v)}[act](z)
        slope, = torch.autograd.grad(y.sum(), z)
        z, y = z.detach(), y.detach()
        if times:
            dr = g * y
            tr = (HALF + 2.0 ** -20 + 2.0 ** -22 + 2.0 ** -23 * (1 + z * z)) * dr.abs() + 2.0 ** -126
            g = g * R.double()
        dz = g * slope
        raw = 2.0 ** -20 * g.abs() * (1 + z.abs().clamp(max=64)) + 2.0 ** -22 * dz.abs()
    return dz, raw, dr, tr


KINDS = [("gelu", False), ("silu", True), ("none", True), ("none", False)]


def tensors(rows, n_out, act, times, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    Z, R, dY = ((torch.randn(rows, n_out, device="cuda", generator=g) * s).to(torch.bfloat16) for s in (2.0, 1.0, 0.1))
    return Z if act != "none" or times else None, R if times else None, dY


@pytest.mark.gpu
@pytest.mark.parametrize("rows,n_out", LONG)
@pytest.mark.parametrize("act,times", KINDS)
def test_gpu_backward_of_long_slices(rows, n_out, act, times):
    Z, R, dY = tensors(rows, n_out, act, times, rows)
    join = TIMES if times else ADD
    ws = torch.empty(TW.fpdt_tw_affine_bwd_workspace_bytes(rows, n_out), dtype=torch.uint8, device="cuda")
    dZ, dR = torch.full_like(dY, float("nan")), torch.full_like(dY, float("nan")) if times else None
    dB = torch.full((n_out,), 0.5, device="cuda")
    print("[case] long slices", rows, n_out, act, times, flush=True)
    TW.fpdt_tw_affine_bwd(Z, R, dY, dZ, dR, dB, ACT[act], join, workspace=ws)
    torch.cuda.synchronize()
    dz, raw, dr, tr = back(Z, R, dY, act, times)
    within("dZ", dZ, dz, raw + HALF * dz.abs() + 2.0 ** -126)
    if times:
        within("dR", dR, dr, tr)
    # a rounding for each of a thread's rows and for each thread beside it, then in 64 bits and once more
    _, lines, piece = walk(rows, n_out)
    want = 0.5 + dz.sum(0)
    within("dB", dB, want, raw.sum(0) + (piece / lines + lines + 1) * 2.0 ** -24 * dz.abs().sum(0) + 2.0 ** -24 * want.abs())
    del dz, raw, dr, tr
    # in Z's place, in dY's, in R's (dR in another one): the same bits; the sums alone too
    for places in ("zr", "dz" if times else "d", "rd" if times else "z"):
        t = {"z": None if Z is None else Z.clone(), "r": None if R is None else R.clone(), "d": dY.clone()}
        out = t[places[0]] if t[places[0]] is not None else t["d"]
        other = t[places[1]] if times else None
        sums = torch.full((n_out,), 0.5, device="cuda")
        TW.fpdt_tw_affine_bwd(t["z"], t["r"], t["d"], out, other, sums, ACT[act], join, workspace=ws)
        torch.cuda.synchronize()
        assert torch.equal(out, dZ) and torch.equal(sums, dB) and (other is None or torch.equal(other, dR)), places
    if Z is None:
        sums = torch.full((n_out,), 0.5, device="cuda")
        TW.fpdt_tw_affine_bwd(None, None, dY, None, None, sums, workspace=ws)
        torch.cuda.synchronize()
        assert torch.equal(sums, dB)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,n_out", LONG)
@pytest.mark.parametrize("act,times", [("gelu", False), ("silu", True)])
def test_gpu_backward_of_experts_in_long_slices(rows, n_out, act, times):
    """Experts that end anywhere within a step of four rows, that have none, and one of many slices; rows in front of the first and behind the last are nobody's."""
    Z, R, dY = tensors(rows, n_out, act, times, rows + 1)
    cuts = torch.randint(11, rows // 2, (40,), generator=torch.Generator().manual_seed(n_out)).sort().values
    ends = torch.cat([cuts, cuts[-1:], torch.tensor([rows - 5])])
    offsets, E = ends.to(torch.int32).cuda(), len(ends) - 1
    first, last = int(ends[0]), int(ends[-1])
    ws = torch.empty(TW.fpdt_tw_affine_bwd_workspace_bytes(rows, n_out, E), dtype=torch.uint8, device="cuda")
    dZ, dR = torch.full_like(dY, 9.0), torch.full_like(dY, 9.0) if times else None
    dB = torch.randn(E, n_out, device="cuda", generator=torch.Generator(device="cuda").manual_seed(5))
    was = dB.double()
    print("[case] experts in long slices", rows, n_out, act, times, flush=True)
    TW.fpdt_tw_affine_bwd(Z, R, dY, dZ, dR, dB, ACT[act], TIMES if times else ADD, offsets, ws)
    torch.cuda.synchronize()
    dz, raw, dr, tr = back(Z, R, dY, act, times)
    mine = slice(first, last)
    within("dZ", dZ[mine], dz[mine], (raw + HALF * dz.abs() + 2.0 ** -126)[mine])
    if times:
        within("dR", dR[mine], dr[mine], tr[mine])
    for t in (dZ, dR):
        assert t is None or bool((t[:first] == 9).all() and (t[last:] == 9).all())
    _, lines, piece = walk(rows, n_out)
    for e in range(E):
        part = slice(int(ends[e]), int(ends[e + 1]))
        want = was[e] + dz[part].sum(0)
        within("dB of %d" % e, dB[e], want, raw[part].sum(0) + (piece / lines + lines + 1) * 2.0 ** -24 * dz[part].abs().sum(0) + 2.0 ** -24 * want.abs())


# ------------------------------------------------------------------ few rows
def steps_of(n_in):
    """Pipelined steps (two units of 64 k each) of the eight waves: few_rows of csrc/tw_affine.h."""
    units = -(-n_in // 64)
    each = -(-units // 8)
    return [max(min(min(w * each + each, units), n_in // 64) - w * each, 0) // 2 for w in range(8)]


FEW_IN = (1024, 1096, 2048, 3080, 4096, 5128, 8800)


def test_few_rows_cover_every_way_through_the_pipeline():
    assert {s for n in FEW_IN for s in steps_of(n)} >= {0, 1, 2, 3, 4, 5, 9}


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [1, 16, 17, 20, 32, 33, 48, 64])
@pytest.mark.parametrize("n_in", FEW_IN)
@pytest.mark.parametrize("n_out", [40, 515, 1001])
def test_gpu_few_rows(rows, n_in, n_out):
    """One, two and four tiles of rows; outputs in pieces of 16 bytes and not; B, R, Z and Y one element behind a boundary; in R's place."""
    assert rows <= 64 and n_in % 8 == 0 and rows * n_in * n_out <= 544 << 20  # (few_pays)
    X, W, B, R, _ = _make(rows, n_in, n_out, n_in + rows)
    ws = torch.empty(TW.fpdt_tw_affine_workspace_bytes(rows, n_in, n_out), dtype=torch.uint8, device="cuda")

    def off(t):
        b = torch.full((t.numel() + 2,), 9.0, dtype=t.dtype, device="cuda")
        v = b[1:-1].view(t.shape)
        v.copy_(t)
        return v, b

    for b, r, act, join in ((B, R, "silu", TIMES), (None, R, "none", ADD), (B, None, "gelu", ADD)):
        Y, Z = (torch.full((rows, n_out), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        TW.fpdt_tw_affine_fwd(X, W, b, r, Z, Y, ACT[act], join, ws)
        y, ty, z, tz = reference(X, W, b, r, act, join == TIMES)
        within("Y", Y, y, ty)
        within("Z", Z, z, tz)
        (Y2, yb), (Z2, zb) = off(Y * 0), off(Z * 0)
        TW.fpdt_tw_affine_fwd(X, W, None if b is None else off(b)[0], None if r is None else off(r)[0], Z2, Y2, ACT[act], join, ws)
        assert torch.equal(Y2, Y) and torch.equal(Z2, Z) and all(t[0] == 9 and t[-1] == 9 for t in (yb, zb))
        if r is not None:
            Y3 = r.clone()
            TW.fpdt_tw_affine_fwd(X, W, b, Y3, None, Y3, ACT[act], join, ws)
            assert torch.equal(Y3, Y)


@pytest.mark.gpu
@pytest.mark.parametrize("counts", [(16, 0, 5, 33), (64,), (1, 2, 30, 7), (20, 20, 20)])
@pytest.mark.parametrize("n_in", [1024, 2048, 3080, 8800])
@pytest.mark.parametrize("n_out", [40, 520])
def test_gpu_few_rows_of_experts_off_alignment(counts, n_in, n_out):
    """Every number of steps; B, R, Z and Y one element behind a boundary, which the rows of an expert's tensors may be."""
    E, used = len(counts), sum(counts)
    ends = [sum(counts[:e]) for e in range(E + 1)]
    offsets = torch.tensor(ends, dtype=torch.int32, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(n_in)
    bf = lambda *s, std=1.0: (torch.randn(*s, device="cuda", generator=g) * std).to(torch.bfloat16)
    X, W, B, R = bf(used, n_in), bf(E, n_out, n_in, std=n_in ** -0.5), bf(E, n_out), bf(used, n_out)

    def off(t):
        b = torch.full((t.numel() + 2,), 9.0, dtype=t.dtype, device="cuda")
        v = b[1:-1].view(t.shape)
        v.copy_(t)
        return v, b

    for r, act, join in ((R, "silu", TIMES), (None, "gelu", ADD)):
        (Y, yb), (Z, zb) = off(torch.zeros_like(R)), off(torch.zeros_like(R))
        TW.fpdt_tw_experts_affine_fwd(X, W, off(B)[0], None if r is None else off(r)[0], Z, Y, offsets, ACT[act], join)
        torch.cuda.synchronize()
        assert all(t[0] == 9 and t[-1] == 9 for t in (yb, zb))
        for e in range(E):
            at = slice(ends[e], ends[e + 1])
            y, ty, z, tz = reference(X[at], W[e], B[e], None if r is None else r[at], act, join == TIMES)
            within("Y of %d" % e, Y[at], y, ty)
            within("Z of %d" % e, Z[at], z, tz)


# ------------------------------------------------------------------ products with divided tiles
DIVIDED = [((81, 88, 1240), (1, 4, "divided")), ((95, 164, 1792), (1, 4, "divided")), ((100, 183, 737), (1, 4, "divided")), ((579, 904, 712), (2, 2, "divided")),
           ((607, 565, 880), (2, 2, "divided")), ((2226, 264, 1584), (2, 4, "divided")), ((2763, 309, 1336), (2, 4, "divided")), ((132, 4440, 3240), (3, 4, "divided")),
           ((132, 3761, 4246), (3, 4, "divided")), ((405, 4264, 3096), (4, 4, "divided")), ((405, 3277, 4960), (4, 4, "divided")), ((4193, 4056, 608), (2, 2, "mixed")),
           ((4457, 3734, 610), (2, 2, "mixed")), ((2497, 3320, 3824), (2, 4, "mixed")), ((2524, 3249, 3816), (2, 4, "mixed")), ((3814, 4368, 840), (4, 4, "mixed")),
           ((4041, 4334, 888), (4, 4, "mixed"))]


def test_products_run_divided():
    for size, plan in DIVIDED:
        assert launch_rules.product(*size) == plan, size


@pytest.mark.gpu
@pytest.mark.parametrize("size", [s for s, _ in DIVIDED], ids=str)
def test_gpu_forward_with_divided_tiles(size):
    """Some workgroups leave sums of their range of k and others do what is behind their whole tile, with a gate, a residual in Y's place, and Z."""
    rows, n_out, n_in = size
    X, W, B, R, _ = _make(rows, n_in, n_out, rows)
    ws = torch.empty(TW.fpdt_tw_affine_workspace_bytes(rows, n_in, n_out), dtype=torch.uint8, device="cuda")
    ws.fill_(255)  # (sums that nobody wrote are NaN)
    print("[case] divided tiles", size, flush=True)
    for b, r, act, join in ((B, R, "silu", TIMES), (None, R, "none", ADD), (B, None, "gelu", ADD)):
        Y, Z = (torch.full((rows, n_out), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        TW.fpdt_tw_affine_fwd(X, W, b, r, Z, Y, ACT[act], join, ws)
        y, ty, z, tz = reference(X, W, b, r, act, join == TIMES)
        within("Y", Y, y, ty)
        within("Z", Z, z, tz)
        if r is not None:
            Y2 = r.clone()
            TW.fpdt_tw_affine_fwd(X, W, b, Y2, None, Y2, ACT[act], join, ws)
            assert torch.equal(Y2, Y)
