"""Tokens sorted by expert and back (fpdt_tw_experts_*), the experts' products, and a feed-forward block made of them: refusals (no GPU), and GPU parity."""
import numpy as np
import pytest
import torch

from oracle import tokenwise as otw
from paper_2408_16978_amd import tokenwise as TW

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
ACT = {"none": TW.FPDT_TW_ACT_NONE, "gelu": TW.FPDT_TW_ACT_GELU, "silu": TW.FPDT_TW_ACT_SILU}


# ------------------------------------------------------------------ refusals (CPU)
L = lambda name: getattr(TW.load(), "fpdt_tw_experts_" + name)


def _call(name, order, base, **kw):
    assert not set(kw) - set(order)
    return L(name)(*[dict(base, **kw)[k] for k in order], None)


SORT = ("expert", "offsets", "place", "rows", "top", "experts", "ws", "wsb")
ROWS = ("rows", "top", "hidden", "dtype")
PTRS = dict(zip(("a", "b", "c", "d", "e", "f", "g", "h"), range(0x10000000, 0x90000000, 0x10000000)))


@pytest.mark.parametrize("status,bad", [
    (1, dict(expert=None)), (1, dict(offsets=None)), (1, dict(place=None)), (1, dict(rows=0)), (1, dict(top=0)), (1, dict(experts=0)), (1, dict(expert=0x10000002)),
    (1, dict(place=0x10000004)), (1, dict(offsets=0x30000000)), (1, dict(ws=0x30000000)), (2, dict(experts=1025)), (2, dict(rows=1 << 31)), (2, dict(rows=1 << 30, top=2)),
    (3, dict(ws=None)), (3, dict(ws=0x40000010)), (3, dict(wsb=255))])
def test_sort_refused(status, bad):
    base = dict(expert=PTRS["a"], offsets=PTRS["b"], place=PTRS["c"], rows=100, top=2, experts=8, ws=PTRS["d"], wsb=1 << 20)
    assert _call("sort", SORT, base, **bad) == status and TW.fpdt_tw_last_error() != ""


@pytest.mark.parametrize("status,bad", [(1, dict(X=None)), (1, dict(place=None)), (1, dict(Xs=None)), (1, dict(rows=-1)), (1, dict(hidden=0)), (1, dict(dtype=2)), (1, dict(X=0x10000001)),
                                        (1, dict(Xs=0x10000010)), (1, dict(Xs=0x20000010)), (2, dict(rows=1 << 31)), (2, dict(hidden=(1 << 28) + 1)), (2, dict(rows=1 << 30, top=2))])
def test_gather_refused(status, bad):
    base = dict(X=PTRS["a"], place=PTRS["b"], Xs=PTRS["c"], R=PTRS["d"], rows=64, top=2, hidden=64, dtype=1)
    assert _call("gather_fwd", ("X", "place", "Xs") + ROWS, base, **bad) == status and TW.fpdt_tw_last_error() != ""
    assert _call("gather_bwd", ("X", "place", "R", "Xs") + ROWS, base, **bad) == status and TW.fpdt_tw_last_error() != ""


@pytest.mark.parametrize("status,bad", [(1, dict(Ys=None)), (1, dict(weight=None)), (1, dict(place=None)), (1, dict(Y=None)), (1, dict(top=0)), (1, dict(weight=0x20000002)),
                                        (1, dict(Y=0x10000010)), (1, dict(Y=0x20000000)), (1, dict(Y=0x40000010)), (2, dict(rows=1 << 30, top=2))])
def test_combine_refused(status, bad):
    base = dict(Ys=PTRS["a"], weight=PTRS["b"], place=PTRS["c"], R=PTRS["d"], Y=PTRS["e"], rows=64, top=2, hidden=64, dtype=1)
    assert _call("combine_fwd", ("Ys", "weight", "place", "R", "Y") + ROWS, base, **bad) == status and TW.fpdt_tw_last_error() != ""


@pytest.mark.parametrize("status,bad", [
    (1, dict(place=None)), (1, dict(dY=None)), (1, dict(dYs=None, dweight=None)), (1, dict(Ys=None)), (1, dict(weight=None)), (1, dict(dYs=0x10000010)), (1, dict(dYs=0x40000000)),
    (1, dict(dweight=0x20000000)), (1, dict(dweight=0x50000000)), (1, dict(dweight=0x60000002)), (1, dict(dtype=-1)), (2, dict(hidden=1 << 29))])
def test_combine_bwd_refused(status, bad):
    base = dict(Ys=PTRS["a"], weight=PTRS["b"], place=PTRS["c"], dY=PTRS["d"], dYs=PTRS["e"], dweight=PTRS["f"], rows=64, top=2, hidden=64, dtype=1)
    assert _call("combine_bwd", ("Ys", "weight", "place", "dY", "dYs", "dweight") + ROWS, base, **bad) == status and TW.fpdt_tw_last_error() != ""


@pytest.mark.parametrize("status,bad", [
    (1, dict(X=None)), (1, dict(W=None)), (1, dict(Y=None)), (1, dict(offsets=None)), (1, dict(rows=0)), (1, dict(experts=0)), (1, dict(act=4)), (1, dict(join=3)), (1, dict(join=1, R=None)),
    (1, dict(X=0x10000008)), (1, dict(W=0x20000002)), (1, dict(Y=0x60000001)), (1, dict(Y=0x10000000)), (1, dict(Z=0x40000000)), (1, dict(Y=0x50000000)), (1, dict(Z=0x70000000)),
    (2, dict(n_in=60)), (2, dict(n_out=62)), (2, dict(experts=1025)), (2, dict(rows=1 << 31)), (2, dict(n_out=1 << 23))])
def test_products_refused(status, bad):
    base = dict(X=PTRS["a"], W=PTRS["b"], B=PTRS["c"], R=PTRS["d"], Z=PTRS["e"], Y=PTRS["f"], offsets=PTRS["g"], rows=64, experts=4, n_in=64, n_out=64, act=1, join=0)
    order = ("X", "W", "B", "R", "Z", "Y", "offsets", "rows", "experts", "n_in", "n_out", "act", "join")
    assert _call("affine_fwd", order, base, **bad) == status and TW.fpdt_tw_last_error() != ""


@pytest.mark.parametrize("status,bad", [
    (1, dict(X=None)), (1, dict(W=None)), (1, dict(dY=None)), (1, dict(offsets=None)), (1, dict(dY=0x30000008)), (1, dict(dX=0x10000000)), (1, dict(dX=0x40000001)),
    (1, dict(dW=0x20000000)), (1, dict(dW=0x50000002)), (1, dict(dW=0x60000000)), (1, dict(n_in=0)), (2, dict(n_in=12)), (2, dict(experts=2000))])
def test_products_bwd_refused(status, bad):
    base = dict(X=PTRS["a"], W=PTRS["b"], dY=PTRS["c"], dX=PTRS["d"], dW=PTRS["e"], offsets=PTRS["f"], rows=64, experts=4, n_in=64, n_out=64)
    assert _call("linear_bwd", ("X", "W", "dY", "dX", "dW", "offsets", "rows", "experts", "n_in", "n_out"), base, **bad) == status and TW.fpdt_tw_last_error() != ""


def test_workspace_bytes_and_binding():
    S = TW.fpdt_tw_experts_sort_workspace_bytes
    assert S(0, 8) == S(8, 0) == S(1 << 31, 8) == S(8, 1025) == S(8, (1 << 32) + 8) == 0
    assert S(1, 1) == 256 and S(1 << 30, 1024) <= 256 * 1024 * 4
    i = torch.zeros(4, 2, dtype=torch.int32)
    with pytest.raises(ValueError, match="current device"):
        TW.fpdt_tw_experts_sort(i, torch.zeros(9, dtype=torch.int32), i.clone(), torch.zeros(256, dtype=torch.uint8))


# ------------------------------------------------------------------ parity (GPU)
def f64(t):
    return None if t is None else t.double().cpu().numpy()


def _close(name, got, ref, tol):
    off = np.abs(f64(got) - ref)
    assert np.isfinite(f64(got)).all() and (off <= tol).all(), (name, off.max(), (off - tol).max())


def sort(expert, experts):
    rows, top = expert.shape
    offsets, place = torch.full((experts + 1,), -7, dtype=torch.int32, device="cuda"), torch.full_like(expert, -7)
    need = TW.fpdt_tw_experts_sort_workspace_bytes(rows * top, experts)
    room = torch.full((need + 256,), 77, dtype=torch.uint8, device="cuda")
    TW.fpdt_tw_experts_sort(expert, offsets, place, room[:need])
    torch.cuda.synchronize()
    assert (room[need:] == 77).all()
    return offsets, place


@pytest.mark.gpu
@pytest.mark.parametrize("rows,top,experts", [(1, 1, 1), (1, 8, 8), (16, 2, 8), (63, 1, 3), (65, 1, 64), (1000, 8, 64), (1024, 1, 1024), (1025, 7, 100), (4096, 2, 8), (4097, 2, 8), (8191, 1, 5),
                                              (30001, 2, 8), (32768, 2, 16), (60000, 8, 256), (100003, 6, 1000), (700001, 1, 33)])
def test_gpu_sort(rows, top, experts):
    """Whole numbers, equal to the definition's: random choices, all to one expert, none to any, numbers that are no expert's, in order, and one expert twice."""
    g = torch.Generator(device="cuda").manual_seed(rows)
    some = torch.randint(-2, experts + 2, (rows, top), device="cuda", generator=g).to(torch.int32)
    cases = [some, torch.full_like(some, experts - 1), torch.full_like(some, -1), (torch.arange(rows * top, device="cuda") * experts // (rows * top)).view(rows, top).to(torch.int32)]
    far = some.clone()
    far[::3] = 2 ** 31 - 1
    far[1::3] = -2 ** 31
    for expert in cases + [far]:
        offsets, place = sort(expert, experts)
        want_offsets, want_place = otw.experts_sort(expert.cpu().numpy(), experts)
        assert np.array_equal(offsets.cpu().numpy(), want_offsets) and np.array_equal(place.cpu().numpy(), want_place)


def chosen(rows, top, experts, seed, lost=0.1):
    g = torch.Generator(device="cuda").manual_seed(seed)
    e = torch.rand(rows, experts, device="cuda", generator=g).topk(min(top, experts), 1).indices.to(torch.int32)
    e = e.repeat(1, -(-top // e.shape[1]))[:, :top]  # (more than there are experts: some twice)
    return torch.where(torch.rand(rows, top, device="cuda", generator=g) < lost, -1, e).contiguous()


@pytest.mark.gpu
@pytest.mark.parametrize("rows,top,experts,hidden", [(1, 1, 1, 1), (3, 2, 4, 7), (16, 2, 8, 64), (37, 8, 64, 520), (50, 3, 2, 2048), (33, 9, 16, 2056), (200, 4, 8, 1001), (1030, 6, 16, 100),
                                                     (20, 2, 8, 16390)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gpu_rows_to_experts_and_back(rows, top, experts, hidden, dtype):
    g = torch.Generator(device="cuda").manual_seed(hidden)
    make = lambda *s: torch.randn(*s, device="cuda", generator=g).to(DT[dtype])
    half = HALF_STEP[dtype]
    expert = chosen(rows, top, experts, rows)
    offsets, place = sort(expert, experts)
    used, p = int(offsets[-1]), place.cpu().numpy()
    X, R, dY, Ys, dXs = make(rows, hidden), make(rows, hidden), make(rows, hidden), make(rows * top, hidden), make(rows * top, hidden)
    weight = torch.rand(rows, top, device="cuda", generator=g)
    print("[case] rows", rows, top, experts, hidden, dtype, flush=True)
    # to the experts: exact, and what has no assignment stays
    Xs = torch.full_like(Ys, 9.0)
    TW.fpdt_tw_experts_gather_fwd(X, place, Xs)
    torch.cuda.synchronize()
    want = np.full((rows * top, hidden), 9.0)
    for t, j in zip(*np.nonzero(p >= 0)):
        want[p[t, j]] = f64(X[t])
    assert np.array_equal(f64(Xs), want) and (Xs[used:] == 9).all()
    # sums on the way back: a rounding of 2^-24 of the sum of sizes for each term, and one more of the result
    here = (p >= 0)[..., None]
    def sums(values, w):
        terms = np.where(here, f64(values)[np.maximum(p, 0)], 0.0) * (1.0 if w is None else f64(w)[..., None])
        return terms.sum(axis=1), np.abs(terms).sum(axis=1)
    for w, r in ((None, None), (None, R), (weight, None), (weight, R)):
        values = dXs if w is None else Ys
        ref, size = sums(values, w)
        ref, size = (ref, size) if r is None else (ref + f64(r), size + np.abs(f64(r)))
        for out in (torch.full_like(X, float("nan")), None if r is None else r.clone()):
            if out is None:
                continue
            joins = None if r is None else r if torch.isnan(out).any() else out
            if w is None:
                TW.fpdt_tw_experts_gather_bwd(values, place, joins, out)
            else:
                TW.fpdt_tw_experts_combine_fwd(values, w, place, joins, out)
            torch.cuda.synchronize()
            _close("sum", out, ref, half * np.abs(ref) + (top + 2) * 2.0 ** -24 * size)
    # gradient of the weighted sum
    dYs, dweight = torch.full_like(Ys, 9.0), torch.full_like(weight, float("nan"))
    TW.fpdt_tw_experts_combine_bwd(Ys, weight, place, dY, dYs, dweight)
    torch.cuda.synchronize()
    want, dots, size = np.full((rows * top, hidden), 9.0), np.zeros((rows, top)), np.zeros((rows, top))
    for t, j in zip(*np.nonzero(p >= 0)):
        want[p[t, j]] = f64(weight[t, j]) * f64(dY[t])
        dots[t, j], size[t, j] = (f64(dY[t]) * f64(Ys[p[t, j]])).sum(), np.abs(f64(dY[t]) * f64(Ys[p[t, j]])).sum()
    _close("dYs", dYs, want, (half + 2.0 ** -24) * np.abs(want) * (want != 9.0))
    # the terms of a lane, then six steps over the lanes
    _close("dweight", dweight, dots, (hidden / 64 + 8 + 7) * 2.0 ** -24 * size)
    assert (dYs[used:] == 9).all() and (dweight[place < 0] == 0).all()
    # one of them alone, and in Ys's place: the same bits
    alone, dw = torch.full_like(Ys, 9.0), torch.empty_like(weight)
    TW.fpdt_tw_experts_combine_bwd(None, weight, place, dY, alone, None)
    TW.fpdt_tw_experts_combine_bwd(Ys, None, place, dY, None, dw)
    there = Ys.clone()
    dw2 = torch.empty_like(weight)
    TW.fpdt_tw_experts_combine_bwd(there, weight, place, dY, there, dw2)
    torch.cuda.synchronize()
    assert torch.equal(alone, dYs) and torch.equal(dw, dweight) and torch.equal(dw2, dweight) and torch.equal(there[:used], dYs[:used]) and torch.equal(there[used:], Ys[used:])


@pytest.mark.gpu
def test_gpu_places_beyond_and_values_not_finite():
    """A place outside the rows counts as none; what is not finite where nothing is sent reaches nothing."""
    rows, top, hidden = 10, 2, 100
    place = torch.arange(20, dtype=torch.int32, device="cuda").view(rows, top)
    place[3] = torch.tensor([20, 2 ** 31 - 1], dtype=torch.int32)
    place[4] = torch.tensor([-2 ** 31, -5], dtype=torch.int32)
    Ys, weight, Y = torch.randn(20, hidden, device="cuda"), torch.rand(rows, top, device="cuda"), torch.empty(rows, hidden, device="cuda")
    Ys[6:10] = float("nan")
    weight[3:5] = float("inf")
    TW.fpdt_tw_experts_combine_fwd(Ys, weight, place, None, Y)
    room = torch.full((22, hidden), 9.0, device="cuda")
    dw = torch.empty_like(weight)
    TW.fpdt_tw_experts_gather_fwd(Y, place, room[1:21])
    TW.fpdt_tw_experts_combine_bwd(Ys, weight, place, Y, room[1:21], dw)
    torch.cuda.synchronize()
    assert (Y[3:5] == 0).all() and torch.isfinite(Y).all() and (dw[3:5] == 0).all()
    assert (room[0] == 9).all() and (room[21] == 9).all() and (room[7:11] == 9).all() and torch.isfinite(room).all()


@pytest.mark.gpu
def test_gpu_rows_of_more_than_32_bits_of_elements():
    """300000 rows of 8192: the last ones come and go right."""
    rows, hidden = 300000, 8192
    X = torch.zeros(rows, hidden, dtype=torch.bfloat16, device="cuda")
    X[:, 0] = (torch.arange(rows, device="cuda") % 251).bfloat16()
    X[:, -1] = (torch.arange(rows, device="cuda") % 241).bfloat16()
    place = torch.arange(rows - 1, -1, -1, dtype=torch.int32, device="cuda")[:, None].contiguous()
    Xs, one = torch.empty_like(X), torch.ones(rows, 1, device="cuda")
    TW.fpdt_tw_experts_gather_fwd(X, place, Xs)
    torch.cuda.synchronize()
    assert torch.equal(Xs[:, 0], X[:, 0].flip(0)) and torch.equal(Xs[:, -1], X[:, -1].flip(0))
    Y, dw = torch.empty_like(X), torch.empty_like(one)
    TW.fpdt_tw_experts_combine_fwd(Xs, one, place, None, Y)
    assert torch.equal(Y, X)
    TW.fpdt_tw_experts_combine_bwd(Xs, one, place, X, Xs, dw)
    torch.cuda.synchronize()
    assert torch.equal(dw[:, 0], X[:, 0].float() ** 2 + X[:, -1].float() ** 2) and torch.equal(Xs[0], X[-1])




@pytest.mark.gpu
@pytest.mark.parametrize("counts,n_in,n_out", [([1], 8, 8), ([3, 0, 5], 64, 32), ([0, 0, 70, 64, 1], 72, 136), ([130, 65, 0, 257, 2], 256, 264), ([0, 400], 520, 88), ([1] * 70, 40, 48),
                                               ([0] * 60 + [33] + [0] * 30 + [2, 0, 40], 96, 64), ([5] * 300, 64, 128), ([0, 0], 64, 64), ([1000, 900, 30], 1024, 520)])
@pytest.mark.parametrize("act,join", [("none", None), ("gelu", "add"), ("silu", "times")])
def test_gpu_products_of_experts(counts, n_in, n_out, act, join):
    """Every expert's rows against its own product in 64 bits, forward and backward; rows without an expert are left as they were."""
    E, used = len(counts), sum(counts)
    rows, ends = used + 3, np.concatenate([[0], np.cumsum(counts)])
    offsets = torch.tensor(ends, dtype=torch.int32, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(E + n_in)
    bf = lambda *s, std=1.0: (torch.randn(*s, device="cuda", generator=g) * std).to(torch.bfloat16)
    X, W, B, R, dY = bf(rows, n_in), bf(E, n_out, n_in, std=n_in ** -0.5), bf(E, n_out), bf(rows, n_out), bf(rows, n_out, std=0.1)
    print("[case] products", E, used, n_in, n_out, act, join, flush=True)
    Y, Z = (torch.full((rows, n_out), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    r, code = R if join else None, TW.FPDT_TW_JOIN_TIMES if join == "times" else TW.FPDT_TW_JOIN_ADD
    TW.fpdt_tw_experts_affine_fwd(X, W, B, r, Z, Y, offsets, ACT[act], code)
    dX, dW = torch.full_like(X, 9.0), torch.randn(E, n_out, n_in, device="cuda", generator=g)
    was = dW.clone()
    TW.fpdt_tw_experts_linear_bwd(X, W, dY, dX, dW, offsets)
    torch.cuda.synchronize()
    for t in (Y, Z, dX):
        assert (t[used:] == 9).all()
    import test_affine
    for e in range(E):
        a, b = ends[e], ends[e + 1]
        if a == b:
            assert torch.equal(dW[e], was[e])
            continue
        ref = otw.affine(f64(X[a:b]), f64(W[e]), f64(B[e]), None if r is None else f64(r[a:b]), act, join == "times")
        tz, ty = test_affine.budget_fwd(X[a:b], W[e], B[e], None if r is None else r[a:b], ref, act, join == "times", n_in)
        _close("Y", Y[a:b], ref["Y"], ty)
        _close("Z", Z[a:b], ref["Z"], tz)
        lin = otw.linear(f64(X[a:b]), f64(W[e]), f64(dY[a:b]))
        size = np.abs(f64(dY[a:b]))
        _close("dX", dX[a:b], lin["dX"], (n_out + 2) * 2.0 ** -24 * (size @ np.abs(f64(W[e]))) + 2.0 ** -8 * np.abs(lin["dX"]))
        _close("dW", dW[e], f64(was[e]) + lin["dW"], (b - a + 2) * 2.0 ** -24 * (size.T @ np.abs(f64(X[a:b])) + np.abs(f64(was[e]))))
    # one of the two alone, and Y in R's place: the same bits
    dX2, dW2, Y2 = torch.full_like(X, 9.0), was.clone(), Y.clone() if r is None else r.clone()
    TW.fpdt_tw_experts_linear_bwd(X, W, dY, dX2, None, offsets)
    TW.fpdt_tw_experts_linear_bwd(X, W, dY, None, dW2, offsets)
    TW.fpdt_tw_experts_affine_fwd(X, W, B, None if r is None else Y2, None, Y2, offsets, ACT[act], code)
    torch.cuda.synchronize()
    assert torch.equal(dX2, dX) and torch.equal(dW2, dW) and torch.equal(Y2[:used], Y[:used])


@pytest.mark.gpu
@pytest.mark.parametrize("counts,n_in,n_out", [((700, 130, 70, 0, 300, 257), 136, 8192), ((1000, 1, 513, 2000), 64, 4096), ((600,) * 6 + (190, 60), 200, 4104), ((3000, 2000), 520, 2048)])
def test_gpu_products_of_experts_in_large_tiles(counts, n_in, n_out):
    """Tiles of 256 rows and what an expert's last rows make of them, with a gate and without; forward and backward against 64 bits on the GPU."""
    import test_affine
    E, rows, ends = len(counts), sum(counts), np.concatenate([[0], np.cumsum(counts)])
    offsets = torch.tensor(ends, dtype=torch.int32, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(n_in)
    bf = lambda *s, std=1.0: (torch.randn(*s, device="cuda", generator=g) * std).to(torch.bfloat16)
    X, W, B, R, dY = bf(rows, n_in), bf(E, n_out, n_in, std=n_in ** -0.5), bf(E, n_out), bf(rows, n_out), bf(rows, n_out, std=0.1)
    print("[case] large tiles of experts", counts, n_in, n_out, flush=True)
    dX, dW = torch.full_like(X, 9.0), torch.zeros(E, n_out, n_in, device="cuda")
    TW.fpdt_tw_experts_linear_bwd(X, W, dY, dX, dW, offsets)
    for r, act, code in ((R, "silu", TW.FPDT_TW_JOIN_TIMES), (None, "gelu", TW.FPDT_TW_JOIN_ADD)):
        Y, Z = (torch.full((rows, n_out), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        TW.fpdt_tw_experts_affine_fwd(X, W, B, r, Z, Y, offsets, ACT[act], code)
        for e in range(E):
            at = slice(int(ends[e]), int(ends[e + 1]))
            y, ty, z, tz = test_affine.reference(X[at], W[e], B[e], None if r is None else r[at], act, r is not None)
            assert bool(((Y[at].double() - y).abs() <= ty).all()) and bool(((Z[at].double() - z).abs() <= tz).all()), (e, act)
    for e in range(E):
        at = slice(int(ends[e]), int(ends[e + 1]))
        x, d, w = X[at].double(), dY[at].double(), W[e].double()
        want = d @ w
        assert bool(((dX[at].double() - want).abs() <= (n_out + 2) * 2.0 ** -24 * (d.abs() @ w.abs()) + 2.0 ** -8 * want.abs()).all()), e
        assert bool(((dW[e].double() - d.t() @ x).abs() <= (counts[e] + 2) * 2.0 ** -24 * (d.abs().t() @ x.abs())).all()), e


@pytest.mark.gpu
@pytest.mark.parametrize("counts", [(0, 3, 17, 0, 40, 4), (64,), (0, 64, 0, 0), (1,) * 60, (16, 16, 16, 16)])
@pytest.mark.parametrize("n_in,n_out", [(8, 24), (72, 40), (520, 136), (2056, 1000), (4096, 512)])
def test_gpu_few_rows_of_experts(counts, n_in, n_out):
    """Up to 64 rows in all, and up to 64 of one expert: 16 at a time, the last ones fewer."""
    import test_affine
    E, used, ends = len(counts), sum(counts), np.concatenate([[0], np.cumsum(counts)])
    rows = min(64, used + 2)
    offsets = torch.tensor(ends, dtype=torch.int32, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(n_in)
    bf = lambda *s, std=1.0: (torch.randn(*s, device="cuda", generator=g) * std).to(torch.bfloat16)
    X, W, B, R = bf(rows, n_in), bf(E, n_out, n_in, std=n_in ** -0.5), bf(E, n_out), bf(rows, n_out)
    for r, act, code in ((R, "silu", TW.FPDT_TW_JOIN_TIMES), (None, "gelu", TW.FPDT_TW_JOIN_ADD)):
        Y, Z = (torch.full((rows, n_out), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        TW.fpdt_tw_experts_affine_fwd(X, W, B, r, Z, Y, offsets, ACT[act], code)
        for e in range(E):
            at = slice(int(ends[e]), int(ends[e + 1]))
            y, ty, z, tz = test_affine.reference(X[at], W[e], B[e], None if r is None else r[at], act, r is not None)
            assert bool(((Y[at].double() - y).abs() <= ty).all()) and bool(((Z[at].double() - z).abs() <= tz).all()), (e, act)
        assert (Y[used:] == 9).all() and (Z[used:] == 9).all()


@pytest.mark.gpu
def test_gpu_offsets_that_are_none():
    """Offsets below 0, beyond the rows or descending: no row outside the tensors is read or written, and what is in order is right."""
    E, rows, n = 4, 100, 64
    g = torch.Generator(device="cuda").manual_seed(1)
    bf = lambda *s: torch.randn(*s, device="cuda", generator=g).to(torch.bfloat16)
    X, W, dY = bf(rows, n), bf(E, n, n), bf(rows, n)
    room = torch.full((rows + 2, n), 9.0, dtype=torch.bfloat16, device="cuda")
    for ends in ([-5, 30, 20, 60, 2 ** 31 - 1], [-2 ** 31] * 5, [50, 40, 30, 20, 10], [0, 2 ** 30, 5, 2 ** 30, 7]):
        offsets = torch.tensor(ends, dtype=torch.int32, device="cuda")
        room.fill_(9.0)
        dW, dB = torch.zeros(E, n, n, device="cuda"), torch.zeros(E, n, device="cuda")
        TW.fpdt_tw_experts_affine_fwd(X, W, None, None, None, room[1:-1], offsets)
        TW.fpdt_tw_experts_linear_bwd(X, W, dY, torch.empty_like(X), dW, offsets)
        wb = torch.empty(TW.fpdt_tw_affine_bwd_workspace_bytes(rows, n, E), dtype=torch.uint8, device="cuda")
        TW.fpdt_tw_affine_bwd(X, None, dY, torch.empty_like(X), None, dB, ACT["gelu"], offsets=offsets, workspace=wb)
        torch.cuda.synchronize()
        assert (room[0] == 9).all() and (room[-1] == 9).all()
    offsets = torch.tensor([-5, 30, 30, 60, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    TW.fpdt_tw_experts_affine_fwd(X, W, None, None, None, room[1:-1], offsets)
    Y = torch.empty(rows, n, dtype=torch.bfloat16, device="cuda")
    TW.fpdt_tw_experts_affine_fwd(X, W, None, None, None, Y, torch.tensor([0, 30, 30, 60, rows], dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    assert torch.equal(room[1:-1], Y)


@pytest.mark.gpu
@pytest.mark.parametrize("nm,nf,lines", [(256, 512, 9), (100, 300, 4)])
def test_gpu_benchmark_of_the_block(monkeypatch, capsys, nm, nf, lines):
    """Each operation is timed; of widths that experts do not take, the dense ones."""
    import json
    import sys

    from paper_2408_16978_amd import bench_tokenwise as bench
    common = ("--rows 64 --n-model %d --n-ffn %d --n-qkv 300 --head-dim 50 --vocab 512 --chunks 1 --iters 1" % (nm, nf)).split()
    counts = []
    for more in ([], ["--feed-forward"]):
        monkeypatch.setattr(sys, "argv", ["bench"] + common + more)
        bench.main()
        out = [json.loads(l) for l in capsys.readouterr().out.splitlines()]
        assert all(l["ms"] > 0 for l in out)
        counts.append(len(out))
    assert counts[1] - counts[0] == lines


# ------------------------------------------------------------------ a block of them
class Block:
    """y = x + dropout(sum_j w_j (silu(xs W1^T) * (xs W3^T)) W2^T): the buffers, and forward and backward as a training step calls them."""

    def __init__(self, rows, top, E, n, f, seed=11):
        g = torch.Generator(device="cuda").manual_seed(seed)
        bf = lambda *s, std=1.0: (torch.randn(*s, device="cuda", generator=g) * std).to(torch.bfloat16)
        e = lambda *s, dt=torch.bfloat16: torch.zeros(*s, dtype=dt, device="cuda")
        self.rows, self.top, self.E, wide = rows, top, E, rows * top
        self.W1, self.W3, self.W2 = bf(E, f, n, std=n ** -0.5), bf(E, f, n, std=n ** -0.5), bf(E, n, f, std=f ** -0.5)
        self.x, self.dy, self.weight, self.expert = bf(rows, n), bf(rows, n), torch.rand(rows, top, device="cuda", generator=g), chosen(rows, top, E, seed)
        self.offsets, self.place, self.step = e(E + 1, dt=torch.int32), e(rows, top, dt=torch.int32), e(1, dt=torch.int64)
        self.xs, self.u, self.z, self.h, self.ys, self.sum, self.y = e(wide, n), e(wide, f), e(wide, f), e(wide, f), e(wide, n), e(rows, n), e(rows, n)
        self.dsum, self.dys, self.dh, self.dz, self.du, self.dxs, self.dxs3, self.dx = e(rows, n), e(wide, n), e(wide, f), e(wide, f), e(wide, f), e(wide, n), e(wide, n), e(rows, n)
        self.dweight = e(rows, top, dt=torch.float32)
        self.dW1, self.dW3, self.dW2 = (torch.zeros_like(w, dtype=torch.float32) for w in (self.W1, self.W3, self.W2))
        self.ws = e(TW.fpdt_tw_experts_sort_workspace_bytes(wide, E), dt=torch.uint8)

    def run(self, stream=None):
        o, p, more = self.offsets, self.place, dict(stream=stream)
        drop = dict(p=0.1, seed=21, step_dev=self.step, stream=stream)
        TW.fpdt_tw_experts_sort(self.expert, o, p, self.ws, **more)
        TW.fpdt_tw_experts_gather_fwd(self.x, p, self.xs, **more)
        TW.fpdt_tw_experts_affine_fwd(self.xs, self.W3, None, None, None, self.u, o, **more)
        TW.fpdt_tw_experts_affine_fwd(self.xs, self.W1, None, self.u, self.z, self.h, o, ACT["silu"], TW.FPDT_TW_JOIN_TIMES, **more)
        TW.fpdt_tw_experts_affine_fwd(self.h, self.W2, None, None, None, self.ys, o, **more)
        TW.fpdt_tw_experts_combine_fwd(self.ys, self.weight, p, None, self.sum, **more)
        TW.fpdt_tw_dropout_fwd(self.sum, self.x, self.y, **drop)
        # and back
        TW.fpdt_tw_dropout_bwd(self.dy, self.dsum, **drop)
        TW.fpdt_tw_experts_combine_bwd(self.ys, self.weight, p, self.dsum, self.dys, self.dweight, **more)
        TW.fpdt_tw_experts_linear_bwd(self.h, self.W2, self.dys, self.dh, self.dW2, o, **more)
        TW.fpdt_tw_affine_bwd(self.z, self.u, self.dh, self.dz, self.du, None, ACT["silu"], TW.FPDT_TW_JOIN_TIMES, o, **more)
        TW.fpdt_tw_experts_linear_bwd(self.xs, self.W1, self.dz, self.dxs, self.dW1, o, **more)
        TW.fpdt_tw_experts_linear_bwd(self.xs, self.W3, self.du, self.dxs3, self.dW3, o, **more)
        TW.fpdt_tw_experts_gather_bwd(self.dxs, p, self.dy, self.dx, **more)
        TW.fpdt_tw_experts_gather_bwd(self.dxs3, p, self.dx, self.dx, **more)

    OUT = ("y", "dx", "dweight", "dW1", "dW3", "dW2")

    def reference(self):
        """The same by torch's autograd in 64 bits."""
        x, w = self.x.double().requires_grad_(), self.weight.double().requires_grad_()
        W1, W3, W2 = (t.double().requires_grad_() for t in (self.W1, self.W3, self.W2))
        total = torch.zeros_like(x)
        for e in range(self.E):
            t, j = torch.nonzero(self.expert == e, as_tuple=True)
            h = torch.nn.functional.silu(x[t] @ W1[e].t()) * (x[t] @ W3[e].t())
            total = total.index_add(0, t, (h @ W2[e].t()) * w[t, j][:, None])
        kept, scale = otw.dropout_kept(x.numel(), 0, 0.1, 21, int(self.step))
        y = x + total * torch.tensor(kept.reshape(x.shape) * scale, device="cuda")
        y.backward(self.dy.double())
        return dict(y=y.detach(), dx=x.grad, dweight=w.grad, dW1=W1.grad, dW3=W3.grad, dW2=W2.grad)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,top,E,n,f", [(300, 2, 8, 256, 512), (1, 1, 4, 64, 64), (77, 3, 5, 136, 72)])
def test_gpu_block_of_experts(rows, top, E, n, f):
    """Forward and backward against autograd in 64 bits.  Seven tensors on the way are rounded to bf16 (2^-8 at most, 2^-9.8 of the values in the root mean
    square): 2^-8.3 of an output's norm for those of them that reach it and for its own; twice that is allowed."""
    b = Block(rows, top, E, n, f)
    b.step.fill_(4)
    b.run()
    torch.cuda.synchronize()
    for k, want in b.reference().items():
        got = getattr(b, k).double()
        assert float((got - want).norm()) <= 2 * 2.0 ** -8.3 * float(want.norm()) + 1e-30, k


@pytest.mark.gpu
def test_gpu_block_captured_with_other_routes():
    """Captured once; replayed with other tokens, other choices of experts (all to one, none at all) and other steps of dropout, with eager work between: the
    bits of the eager call, whatever the offsets have become."""
    a, b = Block(200, 2, 6, 128, 192), Block(200, 2, 6, 128, 192)
    a.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.run()
    for k in range(4):
        for t in (a, b):
            g = torch.Generator(device="cuda").manual_seed(k)
            t.x.normal_(generator=g)
            t.dy.normal_(generator=g)
            t.expert.copy_(chosen(200, 2, 6, k) if k < 2 else torch.full_like(t.expert, 3 if k == 2 else -1))
            t.step.fill_(k)
            for w in (t.dW1, t.dW3, t.dW2):
                w.zero_()
        graph.replay()
        b.run()
        torch.cuda.synchronize()
        for name in Block.OUT:
            assert torch.equal(getattr(a, name), getattr(b, name)), (k, name)
    assert torch.equal(a.y, a.x) and torch.equal(a.dx, a.dy) and (a.dweight == 0).all() and (a.dW1 == 0).all()


@pytest.mark.gpu
def test_gpu_blocks_on_two_streams():
    """Two blocks at once on two streams: the bits of each alone."""
    blocks, alone = [Block(150, 2, 4, 128, 136, s) for s in (1, 2)], [Block(150, 2, 4, 128, 136, s) for s in (1, 2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for b, s in zip(blocks, streams):
        b.run(s)
    torch.cuda.synchronize()
    for a, b in zip(alone, blocks):
        a.run()
        torch.cuda.synchronize()
        for name in Block.OUT:
            assert torch.equal(getattr(a, name), getattr(b, name)), name


@pytest.mark.parametrize("top", [1, 2])
def test_one_tensor_in_three_places_is_refused(top):
    """An output may be the residual, or Ys, and nothing else with it: rows are read by place and written by token (or the other way round), so a tensor that is all three
    would be read by some workgroups behind what others wrote."""
    a, b, c, d = PTRS["a"], PTRS["b"], PTRS["c"], PTRS["d"]
    sizes = (64, top, 64, 1)
    assert L("gather_bwd")(a, c, a, a, *sizes, None) == 1 and TW.fpdt_tw_last_error() != ""
    assert L("combine_fwd")(a, b, c, a, a, *sizes, None) == 1 and TW.fpdt_tw_last_error() != ""
    assert L("combine_fwd")(d, a, c, a, a, *sizes, None) == 1 and L("combine_fwd")(d, b, a, a, a, *sizes, None) == 1
    assert L("combine_bwd")(a, b, c, a, a, None, *sizes, None) == 1 and TW.fpdt_tw_last_error() != ""
    assert L("combine_bwd")(a, a, c, d, a, None, *sizes, None) == 1 and L("combine_bwd")(a, b, a, d, a, None, *sizes, None) == 1


@pytest.mark.gpu
@pytest.mark.parametrize("rows,top", [((1 << 24) + 5, 4), ((1 << 26) + 3, 1), (3000001, 6), (5000011, 2)])
def test_gpu_more_rows_than_one_turn_of_a_grid(rows, top):
    """Narrow rows, more of them than the largest grid has waves (2^22) or workgroups (2^20), and more than a launch takes (2^32 threads; one of more is cut off without an error): small whole numbers, weights of
    1/2, 1 and 2, so that every product and sum is exact."""
    hidden = 8
    g = torch.Generator(device="cuda").manual_seed(top)
    taken = lambda t, index: torch.cat([t[i] for i in index.split(1 << 22)])  # (one index call of torch's over 2^26 rows and more is cut off at that)
    small = lambda n: torch.randint(-8, 9, (n, hidden), device="cuda", generator=g, dtype=torch.int8).to(torch.bfloat16)
    place = torch.randperm(rows * top, device="cuda", generator=g, dtype=torch.int32).view(rows, top)
    place[::7, 0] = -1
    there = (place >= 0)[..., None]
    at = place.clamp(min=0).long()
    X, R, Ys = small(rows), small(rows), small(rows * top)
    weight = torch.randint(-1, 2, (rows, top), device="cuda", generator=g).float().exp2()
    print("[case] rows of several turns", rows, top, flush=True)
    # to their places
    Xs = torch.full_like(Ys, 9.0)
    TW.fpdt_tw_experts_gather_fwd(X, place, Xs)
    want = torch.full_like(Ys, 9.0)
    for j in range(top):
        sent = there[:, j, 0]
        want[at[sent, j]] = taken(X, sent.nonzero()[:, 0])
    assert torch.equal(Xs, want)
    del Xs, want
    # and back
    Y, Y2 = torch.full_like(X, float("nan")), torch.full_like(X, float("nan"))
    TW.fpdt_tw_experts_combine_fwd(Ys, weight, place, R, Y)
    TW.fpdt_tw_experts_gather_bwd(Ys, place, None, Y2)
    total, plain = R.float(), torch.zeros(rows, hidden, device="cuda")
    for j in range(top):
        y = torch.where(there[:, j], taken(Ys, at[:, j]).float(), 0.0)
        total += y * weight[:, j, None]
        plain += y
    assert torch.equal(Y.float(), total) and torch.equal(Y2.float(), plain)
    del Y, Y2, total, plain
    # the gradient
    dYs, dweight = torch.full_like(Ys, 9.0), torch.full_like(weight, float("nan"))
    TW.fpdt_tw_experts_combine_bwd(Ys, weight, place, X, dYs, dweight)
    want = torch.full_like(Ys, 9.0)
    for j in range(top):
        sent = there[:, j, 0]
        want[at[sent, j]] = (taken(X, sent.nonzero()[:, 0]).float() * weight[sent, j, None]).bfloat16()
        dots = torch.where(sent, (X.float() * taken(Ys, at[:, j]).float()).sum(1), 0.0)
        assert torch.equal(dweight[:, j], dots)
    assert torch.equal(dYs, want)


def test_more_tiles_than_a_launch_has_are_refused():
    """1024 experts of 2^22 columns are 2^24 tiles in any of their shapes: workgroups of 256 threads, 2^32 in all, of which none beyond that would run."""
    far = {k: (i + 1) << 42 for i, k in enumerate("abcdefg")}
    sizes = dict(rows=1024, experts=1024)
    order = ("X", "W", "B", "R", "Z", "Y", "offsets", "rows", "experts", "n_in", "n_out", "act", "join")
    base = dict(X=far["a"], W=far["b"], B=None, R=None, Z=None, Y=far["c"], offsets=far["d"], n_in=8, n_out=1 << 22, act=0, join=0, **sizes)
    assert _call("affine_fwd", order, base) == 2 and TW.fpdt_tw_last_error() != ""
    back = ("X", "W", "dY", "dX", "dW", "offsets", "rows", "experts", "n_in", "n_out")
    base = dict(X=far["a"], W=far["b"], dY=far["c"], dX=None, dW=None, offsets=far["d"], **sizes)
    assert _call("linear_bwd", back, base, dX=far["e"], n_in=1 << 22, n_out=8) == 2
    for n_in, n_out in ((8, 1 << 22), (1 << 22, 8)):
        assert _call("linear_bwd", back, base, dW=far["f"], n_in=n_in, n_out=n_out) == 2 and TW.fpdt_tw_last_error() != ""


@pytest.mark.gpu
@pytest.mark.parametrize("counts", [(2 ** 31 - 1,), (2 ** 30, 0, 5, 2 ** 29 + 77, 2 ** 28, 2 ** 27 - 100)])
def test_gpu_products_of_as_many_rows_as_there_may_be(counts):
    """Narrow rows, 2^31 - 1 of them: tiles of 256 rows where those of 128 would be more than a launch has.  Small whole numbers, so that the products are exact."""
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 120 << 30:
        pytest.skip("needs 120 GB")
    rows, E, n = 2 ** 31 - 1, len(counts), 8
    ends = np.concatenate([[0], np.cumsum(counts)])
    offsets = torch.tensor(ends, dtype=torch.int32, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(E)
    small = lambda *s: torch.randint(-4, 5, s, device="cuda", generator=g, dtype=torch.int8).to(torch.bfloat16)
    period = (1 << 22) + 9
    some, W = small(period, n), small(E, n, n)
    X, Y = torch.empty(rows, n, dtype=torch.bfloat16, device="cuda"), torch.full((rows, n), 9.0, dtype=torch.bfloat16, device="cuda")
    for r in range(0, rows, period):
        X[r:r + period] = some[:min(period, rows - r)]
    print("[case] as many rows as there may be", counts, flush=True)
    for back in (False, True):
        if back:  # dX, with X for dY
            got = torch.full_like(Y, 9.0)
            TW.fpdt_tw_experts_linear_bwd(Y, W, X, got, None, offsets)
        else:
            got = Y
            TW.fpdt_tw_experts_affine_fwd(X, W, None, None, None, got, offsets)
        torch.cuda.synchronize()
        by_expert = [(some.float() @ (W[e].float() if back else W[e].float().t())).bfloat16() for e in range(E)]
        for e in range(E):
            for r in range(int(ends[e]) // period * period, int(ends[e + 1]), period):
                a, b = max(r, int(ends[e])), min(r + period, int(ends[e + 1]))
                assert a >= b or torch.equal(got[a:b], by_expert[e][a - r:b - r]), (back, e, a)
        assert (got[int(ends[-1]):] == 9).all()


@pytest.mark.gpu
@pytest.mark.parametrize("counts,first,n_in,n_out", [([3, 0, 70, 17], 5, 72, 40), ([65, 130, 1], 64, 136, 264), ([300, 257, 190], 33, 200, 4104), ([4, 0, 9, 16], 7, 1032, 136)])
def test_gpu_group_of_experts_between_rows_that_are_not_finite(counts, first, n_in, n_out):
    """A part of sorted offsets, the first of them not 0, and NaN in the rows around them and in those of one of the experts: forward (tiles and few rows), dX and dW of the others are what they
    are on their own, and the rows around stay as they were."""
    import test_affine
    E, used = len(counts), sum(counts)
    rows, ends = first + used + 6, first + np.concatenate([[0], np.cumsum(counts)])
    every = torch.tensor([0] + list(ends) + [rows], dtype=torch.int32, device="cuda")
    offsets = every[1:-1]
    g = torch.Generator(device="cuda").manual_seed(n_in)
    bf = lambda *s, std=1.0: (torch.randn(*s, device="cuda", generator=g) * std).to(torch.bfloat16)
    X, W, B, R, dY = bf(rows, n_in), bf(E, n_out, n_in, std=n_in ** -0.5), bf(E, n_out), bf(rows, n_out), bf(rows, n_out, std=0.1)
    bad = slice(int(ends[E - 2]), int(ends[E - 1]))  # the last but one
    for t in (X, R, dY):
        t[:first], t[first + used:], t[bad] = float("nan"), float("inf"), float("nan")
    print("[case] group of experts", counts, first, n_in, n_out, flush=True)
    Y, Z = (torch.full((rows, n_out), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    TW.fpdt_tw_experts_affine_fwd(X, W, B, R, Z, Y, offsets, ACT["silu"], TW.FPDT_TW_JOIN_TIMES)
    dX, dW = torch.full_like(X, 9.0), torch.zeros(E, n_out, n_in, device="cuda")
    TW.fpdt_tw_experts_linear_bwd(X, W, dY, dX, dW, offsets)
    torch.cuda.synchronize()
    for t in (Y, Z, dX):
        assert (t[:first] == 9).all() and (t[first + used:] == 9).all()
    for e in range(E):
        at = slice(int(ends[e]), int(ends[e + 1]))
        if at == bad:
            assert torch.isnan(Y[at]).all() and torch.isnan(dX[at]).all()
            continue
        y, ty, z, tz = test_affine.reference(X[at], W[e], B[e], R[at], "silu", True)
        assert bool(((Y[at].double() - y).abs() <= ty).all()) and bool(((Z[at].double() - z).abs() <= tz).all()), e
        x, d, w = X[at].double(), dY[at].double(), W[e].double()
        want = d @ w
        assert bool(((dX[at].double() - want).abs() <= (n_out + 2) * 2.0 ** -24 * (d.abs() @ w.abs()) + 2.0 ** -8 * want.abs()).all()), e
        assert bool(((dW[e].double() - d.t() @ x).abs() <= (counts[e] + 2) * 2.0 ** -24 * (d.abs().t() @ x.abs())).all()), e


@pytest.mark.gpu
@pytest.mark.parametrize("rows,top,experts", [(2 ** 31 - 1, 1, 3), ((1 << 28) + 3, 7, 1000)])
def test_gpu_sort_of_as_many_assignments_as_there_may_be(rows, top, experts):
    """Places of every piece of the assignments continue those of the pieces before it."""
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB")
    g = torch.Generator(device="cuda").manual_seed(top)
    piece = torch.randint(-1, experts, ((1 << 24) + 11,), device="cuda", generator=g, dtype=torch.int32)
    n = rows * top
    expert = torch.empty(n, dtype=torch.int32, device="cuda")
    for a in range(0, n, len(piece)):
        expert[a:a + len(piece)] = piece[:min(len(piece), n - a)]
    print("[case] sort", rows, top, experts, flush=True)
    offsets, place = sort(expert.view(rows, top), experts)
    place = place.view(-1)
    # within a piece: what comes before in the order of experts, then as they come
    def ranks(some):
        order = torch.where(some < 0, experts, some).sort(stable=True).indices
        counts = torch.bincount((some + 1).long(), minlength=experts + 1)[1:]
        starts = torch.cat([counts.new_zeros(1), counts.cumsum(0)])
        rank = torch.empty(len(some), dtype=torch.int64, device="cuda")
        rank[order] = torch.arange(len(some), device="cuda")
        return rank - starts[some.clamp(min=0).long()], counts
    rank, counts = ranks(piece)
    last, rest = ranks(piece[:n % len(piece)])
    total = counts * (n // len(piece)) + rest
    want = torch.cat([total.new_zeros(1), total.cumsum(0)])
    assert torch.equal(offsets.long(), want)
    before = want[:-1].clone()
    for a in range(0, n, len(piece)):
        some, r = (piece, rank) if a + len(piece) <= n else (piece[:n - a], last)
        assert torch.equal(place[a:a + len(some)].long(), torch.where(some < 0, -1, before[some.clamp(min=0).long()] + r)), a
        before += counts
