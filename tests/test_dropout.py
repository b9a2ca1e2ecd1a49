"""Dropout with the residual add (fpdt_tw_dropout_*): the generator's published vectors, refusals (no GPU), and GPU parity."""
import math

import numpy as np
import pytest
import torch

from oracle import tokenwise as otw
from paper_2408_16978_amd import tokenwise as TW

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


# ------------------------------------------------------------------ the generator (CPU)
def test_oracle_gives_the_published_vectors():
    """Known answers of Philox4x32-10, as its authors published them with the method."""
    ones = 0xffffffff
    for counter, key, want in (([0] * 4, [0] * 2, "6627e8d5 e169c58d bc57ac4c 9b00dbd8"), ([ones] * 4, [ones] * 2, "408f276d 41c83b0e a20bc7c6 6d5451fd"),
                               ([0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344], [0xa4093822, 0x299f31d0], "d16cfe09 94fdcceb 5001e420 24126ea1")):
        assert " ".join("%08x" % w for w in otw.philox(np.array([counter]), key)[0]) == want


def test_oracle_keeps_the_share_and_not_the_same_twice():
    n = 1 << 16
    kept, scale = otw.dropout_kept(n, 0, 0.25, 7, 3)
    # a binomial share: five deviations
    assert abs(kept.mean() - 0.75) < 5 * math.sqrt(0.25 * 0.75 / n) and scale == 65536 / 49152
    others = [otw.dropout_kept(n, 0, 0.25, 8, 3)[0], otw.dropout_kept(n, 0, 0.25, 7, 4)[0], otw.dropout_kept(n, 1, 0.25, 7, 3)[0], otw.dropout_kept(n, 0, 0.25, 7 + (1 << 40), 3)[0]]
    for o in others:
        assert abs((kept == o).mean() - (0.75 ** 2 + 0.25 ** 2)) < 5 * 0.5 / math.sqrt(n)
    assert np.array_equal(otw.dropout_kept(100, 37, 0.25, 7, 3)[0], kept[37:137])


# ------------------------------------------------------------------ refusals (CPU)
def _fwd(**kw):
    a = dict(X=0x10000000, R=0x20000000, Y=0x30000000, n=1000, first=0, p=0.1, seed=1, step=1, step_dev=None, dtype=1)
    a.update(kw)
    return TW.load().fpdt_tw_dropout_fwd(*[a[k] for k in ("X", "R", "Y", "n", "first", "p", "seed", "step", "step_dev", "dtype")], None)


@pytest.mark.parametrize("status,bad", [
    (1, dict(X=None)), (1, dict(Y=None)), (1, dict(n=0)), (1, dict(n=-1)), (1, dict(first=-1)), (1, dict(p=-0.1)), (1, dict(p=1.5)), (1, dict(p=math.nan)), (1, dict(dtype=2)),
    (1, dict(X=0x10000001)), (1, dict(R=0x20000001)), (1, dict(Y=0x30000002, dtype=0)), (1, dict(step_dev=0x40000004)), (1, dict(Y=0x10000010)), (1, dict(Y=0x20000010)),
    (1, dict(step_dev=0x30000010)), (2, dict(first=1 << 62)), (2, dict(n=1 << 61)), (2, dict(first=(1 << 62) - 1000))])
def test_forward_refused(status, bad):
    assert _fwd(**bad) == status and TW.fpdt_tw_last_error() != ""


def test_backward_and_binding_refused():
    L = TW.load()
    assert L.fpdt_tw_dropout_bwd(None, 0x1000, 8, 0, 0.1, 1, 1, None, 1, None) == 1 and L.fpdt_tw_dropout_bwd(0x1000, 0x1008, 8, 0, 0.1, 1, 1, None, 1, None) == 1
    with pytest.raises(ValueError, match="current device"):
        TW.fpdt_tw_dropout_fwd(torch.zeros(8), None, torch.zeros(8), 0.1, 1)


@pytest.mark.gpu
def test_gpu_binding_refused():
    x, y = torch.zeros(8, device="cuda"), torch.zeros(8, device="cuda")
    for bad, what in ((dict(R=torch.zeros(9, device="cuda")), ValueError), (dict(R=x.bfloat16()), TypeError), (dict(Y=torch.zeros(16, device="cuda")[::2]), ValueError),
                      (dict(seed=-1), ValueError), (dict(seed=1 << 64), ValueError), (dict(step=1 << 63), TW.FpdtTwError), (dict(first=1 << 62), TW.FpdtTwError),
                      (dict(first=-1), TW.FpdtTwError), (dict(X=x.half(), Y=y.half()), TypeError), (dict(step_dev=torch.zeros(2, dtype=torch.int64, device="cuda")), ValueError),
                      (dict(step_dev=torch.zeros(1, device="cuda")), TypeError)):
        a = dict(X=x, R=None, Y=y, p=0.1, seed=1)
        a.update(bad)
        with pytest.raises(what):
            TW.fpdt_tw_dropout_fwd(**a)


# ------------------------------------------------------------------ parity (GPU)
def f64(t):
    return t.double().cpu().numpy()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,first", [(1, 0), (1, 7), (7, 1), (8, 0), (8, 3), (15, 5), (2048, 0), (2049, 8), (4095, (1 << 32) * 8 - 11), (100003, (1 << 62) - 100004)])
@pytest.mark.parametrize("p", [0.1, 0.5])
def test_gpu_against_oracle(dtype, n, first, p):
    """fp32 product and sum (two roundings of 2^-24 of the sizes), rounded once; what is dropped is exactly 0, or R itself."""
    seed, step = 0x123456789abcdef0 + n, -5 if n == 2048 else n
    g = torch.Generator(device="cuda").manual_seed(n)
    X, R = (torch.randn(n, device="cuda", generator=g).to(DT[dtype]) for _ in range(2))
    kept, scale = otw.dropout_kept(n, first, p, seed, step)
    Y = torch.empty_like(X)
    for r in (None, R):
        TW.fpdt_tw_dropout_fwd(X, r, Y, p, seed, step, first)
        torch.cuda.synchronize()
        want = np.where(kept, f64(X) * scale, 0.0)
        size = np.abs(want) + (0.0 if r is None else np.abs(f64(r)))
        want = want if r is None else want + f64(r)
        assert (np.abs(f64(Y) - want) <= HALF_STEP[dtype] * np.abs(want) + 2.0 ** -22 * size).all()
        assert np.array_equal(f64(Y)[~kept], np.zeros((~kept).sum()) if r is None else f64(R)[~kept])
    dX = torch.empty_like(X)
    TW.fpdt_tw_dropout_bwd(X, dX, p, seed, step, first)
    TW.fpdt_tw_dropout_fwd(X, None, Y, p, seed, step, first)
    assert torch.equal(dX, Y)


@pytest.mark.gpu
def test_gpu_ends_of_p_and_what_is_not_finite():
    X, R, Y = torch.randn(1000, device="cuda"), torch.randn(1000, device="cuda"), torch.empty(1000, device="cuda")
    TW.fpdt_tw_dropout_fwd(X, R, Y, 0.0, 1)
    assert torch.equal(Y, X + R)
    TW.fpdt_tw_dropout_fwd(X, R, Y, 1.0, 1)
    assert torch.equal(Y, R)
    TW.fpdt_tw_dropout_fwd(X, None, Y, 1.0, 1)
    assert (Y == 0).all()
    kept = torch.tensor(otw.dropout_kept(1000, 0, 0.5, 9, 2)[0], device="cuda")
    X[::2], X[1::2] = math.inf, math.nan
    TW.fpdt_tw_dropout_fwd(X, R, Y, 0.5, 9, 2)
    assert torch.equal(Y[~kept], R[~kept]) and not torch.isfinite(Y[kept]).any()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gpu_in_place_chunks_and_off_alignment(dtype):
    """In X's place and in R's; a sequence in chunks is the whole; tensors one element behind a boundary."""
    n = 5001
    X, R, Y = (torch.randn(n, device="cuda").to(DT[dtype]) for _ in range(3))
    TW.fpdt_tw_dropout_fwd(X, R, Y, 0.3, 5, 6)
    for place in (0, 1):
        t = [X.clone(), R.clone()]
        TW.fpdt_tw_dropout_fwd(t[0], t[1], t[place], 0.3, 5, 6)
        assert torch.equal(t[place], Y) and torch.equal(t[1 - place], (X, R)[1 - place])
    parts = torch.full((n + 2,), 9.0, device="cuda").to(DT[dtype])
    for a, b in ((0, 1), (1, 1003), (1003, 4097), (4097, n)):
        TW.fpdt_tw_dropout_fwd(X[a:b], R[a:b], parts[1 + a:1 + b], 0.3, 5, 6, first=a)
    torch.cuda.synchronize()
    assert torch.equal(parts[1:-1], Y) and parts[0] == parts[-1] == 9


@pytest.mark.gpu
def test_gpu_more_than_32_bits_of_elements():
    """2^32 + 40 elements of bf16: the last ones are those of their own numbers."""
    n = (1 << 32) + 40
    X = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    TW.fpdt_tw_dropout_fwd(X, None, X, 0.5, 11, 1)
    for a in (0, (1 << 32) - 30):
        kept, scale = otw.dropout_kept(60, a, 0.5, 11, 1)
        assert np.array_equal(f64(X[a:a + 60]), kept * scale)
    share = X.view(torch.int16)[: 1 << 32].ne(0).sum().item() / 2 ** 32
    assert abs(share - 0.5) < 5 * 0.5 / 2 ** 16


@pytest.mark.gpu
def test_gpu_captured_step_and_another_stream():
    """A captured call reads its step from the device at every replay; a call on another stream gives the same."""
    X, Y, Z = torch.randn(3000, device="cuda"), torch.empty(3000, device="cuda"), torch.empty(3000, device="cuda")
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        TW.fpdt_tw_dropout_fwd(X, None, Y, 0.4, 3, step=77, step_dev=step)
    seen = []
    for k in (5, -1, 5):
        step.fill_(k)
        X.normal_(generator=torch.Generator(device="cuda").manual_seed(1))
        graph.replay()
        TW.fpdt_tw_dropout_fwd(X, None, Z, 0.4, 3, step=k)
        torch.cuda.synchronize()
        assert torch.equal(Y, Z)
        seen.append(Y.clone())
    assert torch.equal(seen[0], seen[2]) and not torch.equal(seen[0], seen[1])
    s = torch.cuda.Stream()
    TW.fpdt_tw_dropout_fwd(X, None, Y, 0.4, 3, step=5, stream=s)
    s.synchronize()
    assert torch.equal(Y, seen[0])
