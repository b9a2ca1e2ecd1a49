"""Rotary positions and the split of the QKV product (fpdt_tw_rope_*): oracle pins, frequencies and refusals (no GPU), and
GPU parity against the oracle."""
import math

import numpy as np
import pytest
import torch

from oracle import tokenwise as otw
from paper_2408_16978_amd import tokenwise as TW

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


# ------------------------------------------------------------------ oracle pins (CPU)
@pytest.mark.parametrize("interleaved", [False, True])
def test_oracle_is_an_isometry_that_sees_position_differences_only(interleaved):
    r = np.random.default_rng(1)
    q, k = r.standard_normal((1, 1, 12)), r.standard_normal((1, 1, 12))
    f = otw.rope_freqs(8, 100.0)
    turn = lambda x, p: otw.rope(x, [p], f, interleaved=interleaved)
    assert np.allclose(np.linalg.norm(turn(q, 77)), np.linalg.norm(q))
    assert np.array_equal(turn(q, 77)[..., 8:], q[..., 8:])
    for shift in (1, 50):
        assert np.allclose((turn(q, 9) * turn(k, 4)).sum(), (turn(q, 9 + shift) * turn(k, 4 + shift)).sum())
    # a quarter turn by hand: pair 0 has the frequency 1
    x = np.zeros((1, 1, 4))
    x[0, 0, 0] = 1.0
    y = otw.rope(x, [1], [math.pi / 2, 0.0], interleaved=interleaved)
    assert np.allclose(y[0, 0], [0, 1, 0, 0] if interleaved else [0, 0, 1, 0])


@pytest.mark.parametrize("interleaved", [False, True])
def test_oracle_gradient_is_the_transpose(interleaved):
    r = np.random.default_rng(2)
    x, g = r.standard_normal((3, 2, 10)), r.standard_normal((3, 2, 10))
    f, pos = otw.rope_freqs(6, 50.0), [5, 0, 123]
    fwd = lambda t: (otw.rope(t, pos, f, 1.3, interleaved) * g).sum()
    back = otw.rope(g, pos, f, 1.3, interleaved, inverse=True)
    for at in np.ndindex(x.shape):  # linear: differences of any size are exact
        d = np.zeros_like(x)
        d[at] = 1.0
        assert abs(fwd(x + d) - fwd(x) - back[at]) < 1e-10


# ------------------------------------------------------------------ frequencies (host logic)
def test_frequencies():
    F = TW.fpdt_tw_rope_freqs
    plain = F(64, 500000.0).numpy()
    np.testing.assert_allclose(plain, otw.rope_freqs(64, 500000.0), rtol=1e-14)
    np.testing.assert_allclose(F(64, 500000.0, TW.FPDT_TW_ROPE_LINEAR, 4.0).numpy(), plain / 4, rtol=1e-14)
    raised = F(64, 500000.0, TW.FPDT_TW_ROPE_RAISED, 4.0).numpy()
    assert raised[0] == 1.0 and abs(raised[-1] * 4 / plain[-1] - 1) < 1e-12 and (raised[1:] < plain[1:]).all()
    parts = F(64, 500000.0, TW.FPDT_TW_ROPE_PARTS, 8.0, 8192.0, 1.0, 4.0).numpy()
    turns = 8192 * plain / (2 * math.pi)
    fast, slow = turns >= 4, turns <= 1
    assert fast.any() and slow.any() and (~fast & ~slow).any()
    np.testing.assert_allclose(parts[fast], plain[fast], rtol=1e-14)
    np.testing.assert_allclose(parts[slow], plain[slow] / 8, rtol=1e-14)
    mix = (turns - 1) / 3
    np.testing.assert_allclose(parts, np.where(fast, plain, np.where(slow, plain / 8, mix * plain + (1 - mix) * plain / 8)), rtol=1e-14)
    assert F(2, 10000.0, TW.FPDT_TW_ROPE_RAISED, 4.0).tolist() == [1.0]
    for bad in (dict(rot=0), dict(rot=7), dict(rot=-2), dict(base=0.0), dict(base=math.inf), dict(base=math.nan), dict(scaling=4), dict(scaling=-1),
                dict(scaling=1, factor=0.0), dict(scaling=2, factor=math.nan), dict(scaling=3, factor=2.0, context=0.0),
                dict(scaling=3, factor=2.0, context=8.0, low=4.0, high=4.0), dict(scaling=3, factor=2.0, context=8.0, low=math.nan)):
        with pytest.raises(TW.FpdtTwError) as e:
            F(**dict(dict(rot=8, base=100.0), **bad))
        assert e.value.status == 1, bad
    assert TW.load().fpdt_tw_rope_freqs(8, 100.0, 0, 1.0, 0.0, 0.0, 1.0, None) == 1


# ------------------------------------------------------------------ refusals (CPU)
def _status(**kw):
    """Status of calls with places that are no memory, none of which gets as far as a launch."""
    a = dict(Q=0x10000000, qr=512, K=0x20000000, kr=256, V=0x30000000, vr=256, Qo=0x40000000, qor=512, Ko=0x50000000, kor=256, Vo=0x60000000, vor=256,
             pos=None, pos0=0, freqs=0x1000, amp=1.0, rows=4, Hq=4, Hkv=2, D=128, rot=128, layout=0, dtype=1)
    a.update(kw)
    L = TW.load()
    args = [a[k] for k in ("Q", "qr", "K", "kr", "V", "vr", "Qo", "qor", "Ko", "kor", "Vo", "vor", "pos", "pos0", "freqs", "amp", "rows", "Hq", "Hkv",
                           "D", "rot", "layout", "dtype")]
    got = L.fpdt_tw_rope_fwd(*args, None)
    back = L.fpdt_tw_rope_bwd(*args, None)
    assert got == back
    return got


@pytest.mark.parametrize("bad", [
    dict(Q=None), dict(Qo=None), dict(K=None), dict(Vo=None), dict(freqs=None), dict(freqs=0x1004), dict(pos=0x1004), dict(rows=0), dict(rows=-1),
    dict(Hq=0), dict(Hkv=-1), dict(Hkv=0), dict(D=0), dict(rot=0), dict(rot=63), dict(rot=130), dict(layout=2), dict(dtype=2), dict(amp=math.nan),
    dict(qr=511), dict(kor=255), dict(vr=-256), dict(Q=0x10000001), dict(Vo=0x60000001),
    dict(Qo=0x10000002), dict(Qo=0x10000000, qor=1024), dict(Ko=0x40000000), dict(Ko=0x10000000), dict(Vo=0x20000000),
    # a column of the neighbour's heads in one product's rows
    dict(Qo=0x40000000, qor=1024, Ko=0x40000000 + 2 * 511, kor=1024),
    dict(Qo=0x40000000, qor=1024, Ko=0x40000000 + 2 * (1024 + 800), kor=1024)])
def test_refused(bad):
    assert _status(**bad) == 1 and TW.fpdt_tw_last_error() != ""


@pytest.mark.parametrize("bad", [dict(D=8194, rot=2, qr=1 << 20, kr=1 << 20, vr=1 << 20, qor=1 << 20, kor=1 << 20, vor=1 << 20), dict(rows=1 << 31),
                                 dict(Hq=4097, qr=1 << 20, qor=1 << 20), dict(qr=(1 << 28) + 1)])
def test_unsupported(bad):
    assert _status(**bad) == 2


def test_binding_refuses_what_the_library_cannot_see():
    f = TW.fpdt_tw_rope_freqs(8, 100.0)
    x = torch.zeros(3, 2, 8)
    with pytest.raises(ValueError, match="current device"):
        TW.fpdt_tw_rope_fwd(x, None, None, x, None, None, f)


# ------------------------------------------------------------------ GPU parity
def _budget(x, ref, amplitude, dtype, rot, interleaved):
    """One rounding to the type (half a step), and in fp32: sine and cosine to 2^-23 each (polynomial, its argument, the
    amplitude), two products and a sum: 2^-21 of what the pair's channels hold, times the amplitude."""
    half = rot // 2
    pair = np.array(np.abs(x))
    a, b = (np.s_[..., 0:rot:2], np.s_[..., 1:rot:2]) if interleaved else (np.s_[..., :half], np.s_[..., half:rot])
    pair[a] = pair[b] = np.abs(x[a]) + np.abs(x[b])
    return 2.0 ** (-8 if dtype == "bf16" else -24) * np.abs(ref) + 2.0 ** -21 * amplitude * pair


def _check(name, got, ref, x, amplitude, dtype, rot, interleaved):
    err = np.abs(got.double().cpu().numpy() - ref) / (_budget(x, ref, amplitude, dtype, rot, interleaved) + 1e-300)
    assert err.max() <= 1.0, (name, err.max())


SHAPES = [  # rows, Hq, Hkv, D, rot: accesses of 8, 4, 2 and 1 elements, one head and many, part of the head, one token
    (1, 8, 2, 128, 128), (33, 8, 2, 128, 128), (257, 4, 4, 80, 80), (100, 4, 1, 80, 32), (7, 5, 5, 64, 2), (65, 3, 1, 20, 10), (9, 2, 2, 6, 6),
    (31, 1, 1, 7, 4), (1000, 32, 8, 64, 64), (33, 32, 8, 128, 34), (5000, 8, 2, 128, 30), (3, 200, 100, 16, 6), (50, 1, 1, 512, 6), (2100, 3, 3, 80, 20), (3, 2, 1, 1024, 600), (2, 1, 1, 2050, 2050), (70000, 1, 1, 8, 8)]


@pytest.mark.gpu
@pytest.mark.parametrize("rows,Hq,Hkv,D,rot", SHAPES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
def test_gpu_split_and_gather_match_the_oracle(rows, Hq, Hkv, D, rot, dtype, interleaved):
    print("[case] rope", rows, Hq, Hkv, D, rot, dtype, interleaved, flush=True)
    g = torch.Generator().manual_seed(rows + D)
    layout = TW.FPDT_TW_ROPE_INTERLEAVED if interleaved else TW.FPDT_TW_ROPE_HALF
    X = torch.randn(rows, (Hq + 2 * Hkv) * D, generator=g).to(DT[dtype])
    freqs = TW.fpdt_tw_rope_freqs(rot, 500000.0)
    start, amplitude = 2000000, 1.25
    Xd, fd = X.cuda(), freqs.cuda()
    q, k, v = Xd.view(rows, Hq + 2 * Hkv, D).split([Hq, Hkv, Hkv], 1)
    Qo, Ko, Vo = (torch.full((rows + 1, h, D), 7.0, dtype=DT[dtype], device="cuda") for h in (Hq, Hkv, Hkv))
    TW.fpdt_tw_rope_fwd(q, k, v, Qo[:rows], Ko[:rows], Vo[:rows], fd, position0=start, amplitude=amplitude, layout=layout)
    torch.cuda.synchronize()
    pos = np.arange(start, start + rows)
    x64 = X.double().numpy().reshape(rows, -1, D)
    for name, got, part in (("Q", Qo, np.s_[:, :Hq]), ("K", Ko, np.s_[:, Hq:Hq + Hkv])):
        ref = otw.rope(x64[part], pos, freqs.numpy(), amplitude, interleaved)
        _check(name, got[:rows], ref, x64[part], amplitude, dtype, rot, interleaved)
        assert torch.equal(got[:rows, :, rot:], Xd.view(rows, -1, D)[part][..., rot:])
    assert torch.equal(Vo[:rows], v)
    assert all((t[rows] == 7).all() for t in (Qo, Ko, Vo))
    # the way back, into rows that are longer than the product's; given positions; the columns behind it stay
    dX = torch.full((rows, (Hq + 2 * Hkv) * D + 5), 3.0, dtype=DT[dtype], device="cuda")
    dq, dk, dv = (dX[:, a * D:b * D].unflatten(1, (b - a, D)) for a, b in ((0, Hq), (Hq, Hq + Hkv), (Hq + Hkv, Hq + 2 * Hkv)))
    positions = torch.randint(0, 1 << 21, (rows,), generator=g)
    TW.fpdt_tw_rope_bwd(Qo[:rows], Ko[:rows], Vo[:rows], dq, dk, dv, fd, positions=positions.cuda(), amplitude=amplitude, layout=layout)
    torch.cuda.synchronize()
    for name, got, src in (("dQ", dq, Qo), ("dK", dk, Ko)):
        x = src[:rows].double().cpu().numpy()
        ref = otw.rope(x, positions.numpy(), freqs.numpy(), amplitude, interleaved, inverse=True)
        _check(name, got, ref, x, amplitude, dtype, rot, interleaved)
    assert torch.equal(dv, Vo[:rows]) and (dX[:, (Hq + 2 * Hkv) * D:] == 3).all()


HALVES = [  # a head's lanes: 3 (21 heads of a wave), 2, 6 (groups of heads across waves), 64 and 65 or 128, 12 of which 4 turn, 24 in fp32; heads that end inside a group
    (67, 7, 3, 24, 16), (300, 17, 5, 16, 16), (129, 40, 24, 48, 32), (40, 33, 9, 512, 512), (5, 4, 2, 520, 512), (19, 9, 4, 256, 256), (2100, 12, 12, 96, 32),
    (2, 64, 64, 64, 64), (1, 1, 1, 16, 16), (70, 2, 2, 128, 128), (70, 3, 2, 128, 128), (513, 1, 0, 80, 80), (66000, 2, 1, 24, 16)]


@pytest.mark.gpu
@pytest.mark.parametrize("rows,Hq,Hkv,D,rot", HALVES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gpu_halves_over_lanes(rows, Hq, Hkv, D, rot, dtype):
    """Q and K there with given positions, in place as out of place, each pair within the parity tests' budget; K behind Q in a product's rows
    (V is copied beside them); what lies between the heads' rows stays."""
    print("[case] halves", rows, Hq, Hkv, D, rot, dtype, flush=True)
    g = torch.Generator().manual_seed(rows + D)
    H, freqs = Hq + 2 * Hkv, TW.fpdt_tw_rope_freqs(rot, 10000.0)
    pos = torch.randint(-(1 << 20), 1 << 21, (rows,), generator=g)
    X = torch.randn(rows, H * D + 3, generator=g).to(DT[dtype])
    for sign, call in ((1, TW.fpdt_tw_rope_fwd), (-1, TW.fpdt_tw_rope_bwd)):
        Xd, fd, pd = X.cuda(), freqs.cuda(), pos.cuda()
        parts = lambda t: [t[:, a * D:b * D].unflatten(1, (b - a, D)) if b > a else None for a, b in ((0, Hq), (Hq, Hq + Hkv), (Hq + Hkv, H))]
        q, k, v = parts(Xd)
        outs = [None if t is None else torch.empty(t.shape, dtype=DT[dtype], device="cuda") for t in (q, k, v)]
        call(q, k, v, *outs, fd, positions=pd, amplitude=0.75)
        call(q, k, v, q, k, v, fd, positions=pd, amplitude=0.75)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, (q, k, v)) if a is not None)
        assert torch.equal(Xd[:, H * D:].cpu(), X[:, H * D:])
        for name, got, was in zip("QKV", outs, parts(X)):
            if was is None or name == "V":
                assert was is None or torch.equal(got.cpu(), was)
                continue
            x = was.double().numpy()
            _check(name, got, otw.rope(x, pos.numpy(), freqs.numpy(), 0.75, inverse=sign < 0), x, 0.75, dtype, rot, False)
            assert torch.equal(got[..., rot:].cpu(), was[..., rot:])


@pytest.mark.gpu
@pytest.mark.parametrize("off", [0, 1, 3])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gpu_in_place_at_any_alignment_q_alone(off, dtype):
    """Q alone, in its own place, `off` elements behind a 16-byte boundary; the same within a product's rows for Q and K."""
    g = torch.Generator(device="cuda").manual_seed(off)
    fd = TW.fpdt_tw_rope_freqs(64, 10000.0).cuda()
    buf = torch.randn(50 * 4 * 64 + 16, device="cuda", generator=g).to(DT[dtype])
    q = buf[off:off + 50 * 4 * 64].view(50, 4, 64)
    was, out = buf.clone(), torch.empty_like(q)
    TW.fpdt_tw_rope_fwd(q.clone(), None, None, out, None, None, fd)
    TW.fpdt_tw_rope_fwd(q, None, None, q, None, None, fd)
    torch.cuda.synchronize()
    assert torch.equal(q, out) and torch.equal(buf[:off], was[:off]) and torch.equal(buf[off + 50 * 4 * 64:], was[off + 50 * 4 * 64:])
    x = torch.randn(50, 8 * 64 + off, device="cuda", generator=g).to(DT[dtype])
    was = x.clone()
    part = lambda t, a, b: t[:, a * 64:b * 64].unflatten(1, (b - a, 64))
    Qo, Ko = torch.empty(50, 4, 64, dtype=DT[dtype], device="cuda"), torch.empty(50, 2, 64, dtype=DT[dtype], device="cuda")
    TW.fpdt_tw_rope_fwd(part(was, 0, 4), part(was, 4, 6), None, Qo, Ko, None, fd, position0=9)
    TW.fpdt_tw_rope_fwd(part(x, 0, 4), part(x, 4, 6), None, part(x, 0, 4), part(x, 4, 6), None, fd, position0=9)
    torch.cuda.synchronize()
    assert torch.equal(part(x, 0, 4), Qo) and torch.equal(part(x, 4, 6), Ko) and torch.equal(x[:, 6 * 64:], was[:, 6 * 64:])


@pytest.mark.gpu
def test_gpu_far_positions_keep_their_angle_and_negative_ones_turn_back():
    """Angles at 2^21 tokens and beyond: the pair (1, 0) becomes (cos t, sin t), to 2^-21 (budget of the parity tests) in
    fp32 wherever the 64-bit angle is right to that: 2^-52 of 2^40 radians and the product's rounding are 2^-11.  So to 2^31."""
    freqs = TW.fpdt_tw_rope_freqs(16, 10000.0)
    pos = torch.tensor([0, 1, 2 ** 21 - 1, 2 ** 21, 2 ** 28 + 1, 2 ** 31 - 1, -1, -2 ** 30, 5, 5])
    x = torch.zeros(len(pos), 1, 16)
    x[..., :8] = 1.0
    y = torch.empty(len(pos), 1, 16, device="cuda")
    TW.fpdt_tw_rope_fwd(x.cuda(), None, None, y, None, None, freqs.cuda(), positions=pos.cuda())
    torch.cuda.synchronize()
    t = pos.double()[:, None] * freqs
    ref = torch.cat([t.cos(), t.sin()], 1)
    # two roundings of the angle to 2^-53 each, in the reference and here: 2^31 * 2^-51
    assert (y.cpu().double()[:, 0] - ref).abs().max() <= 2.0 ** -21 + 2.0 ** -20
    assert torch.equal(y[8], y[9])
    # not finite: stays with its pair
    x[0, 0, 3], x[1, 0, 12] = math.inf, math.nan
    z = torch.empty_like(y)
    TW.fpdt_tw_rope_fwd(x.cuda(), None, None, z, None, None, freqs.cuda(), positions=pos.cuda())
    torch.cuda.synchronize()
    bad = ~torch.isfinite(z[:, 0])
    assert bad.nonzero().tolist() == [[0, 3], [0, 11], [1, 4], [1, 12]]
    assert torch.equal(z[~bad[:, None]], y[~bad[:, None]])


@pytest.mark.gpu
@pytest.mark.parametrize("rot,interleaved", [(64, False), (64, True), (6, False)])
def test_gpu_sines_and_cosines_to_their_last_steps(rot, interleaved):
    """The pair (1, 0) becomes (cos t, sin t), in fp32 without another rounding.  The angle is reduced in 64 bits (positions up to 2^21: 2^-51 of 2^21 radians at
    most, 1e-9) and rounded once to fp32: 2^-25 below pi / 4, times a slope of at most 0.88 where it is that much.  The result's own rounding is
    2^-25.  Before it: for the cosine z^2 / 2 <= 0.31 with z^2 rounded to 2^-24 of itself (1.9e-8) and a factor near 1/2 to 2^-26 (times z^2: 0.9e-8), where the slope is
    0.71 at most; for the sine z^3 / 6 <= 0.081 with three roundings of 2^-24 (1.5e-8).  The cosine: 2.1e-8 + 3.0e-8 + 1.9e-8 + 0.9e-8 + 0.1e-8 = 8.0e-8, the
    sine 7.2e-8."""
    rows, heads = 16384, 2
    freqs = TW.fpdt_tw_rope_freqs(rot, 10000.0)
    pos = torch.randint(0, 1 << 21, (rows,), generator=torch.Generator().manual_seed(rot))
    x = torch.zeros(rows, heads, 64, device="cuda")
    a, b = (np.s_[..., 0:rot:2], np.s_[..., 1:rot:2]) if interleaved else (np.s_[..., :rot // 2], np.s_[..., rot // 2:rot])
    x[a] = 1.0
    y = torch.empty_like(x)
    TW.fpdt_tw_rope_fwd(x, None, None, y, None, None, freqs.cuda(), positions=pos.cuda(), layout=TW.FPDT_TW_ROPE_INTERLEAVED if interleaved else TW.FPDT_TW_ROPE_HALF)
    torch.cuda.synchronize()
    t = (pos.double()[:, None] * freqs)[:, None]
    y = y.double().cpu()
    assert (y[a] - t.cos()).abs().max() <= 8.0e-8 and (y[b] - t.sin()).abs().max() <= 8.0e-8


@pytest.mark.gpu
@pytest.mark.parametrize("rot", [64, 30])
def test_gpu_tokens_far_apart(rot):
    """Rows whose distance in a tile does not fit the short offsets: 2^26 elements, the last ones behind 2^31 bytes."""
    rows, far = 20, (1 << 26) + 8
    if torch.cuda.mem_get_info()[0] < 8 << 30:
        pytest.skip("needs 8 GB")
    big = torch.zeros((rows - 1) * far + 2 * 64, dtype=torch.bfloat16, device="cuda")
    q = big.as_strided((rows, 2, 64), (far, 64, 1))
    x = torch.randn(rows, 2, 64, device="cuda").to(torch.bfloat16)
    q.copy_(x)
    fd = TW.fpdt_tw_rope_freqs(rot, 10000.0).cuda()
    near, out = torch.empty_like(x), torch.empty_like(x)
    TW.fpdt_tw_rope_fwd(x, None, None, near, None, None, fd, position0=3)
    TW.fpdt_tw_rope_fwd(q, None, None, out, None, None, fd, position0=3)
    TW.fpdt_tw_rope_fwd(x, None, None, q, None, None, fd, position0=3)
    torch.cuda.synchronize()
    # (other accesses, but the same operations on each pair)
    assert torch.equal(out, near) and torch.equal(q, near)
    assert int(torch.count_nonzero(big)) == int(torch.count_nonzero(near))


@pytest.mark.gpu
def test_gpu_captured_on_a_side_stream_with_eager_calls_between():
    rows, Hq, Hkv, D = 300, 4, 2, 64
    fd = TW.fpdt_tw_rope_freqs(D, 10000.0).cuda()
    X = torch.randn(rows, Hq + 2 * Hkv, D, device="cuda").to(torch.bfloat16)
    pos = torch.arange(rows, device="cuda")
    outs = [torch.empty(rows, h, D, dtype=torch.bfloat16, device="cuda") for h in (Hq, Hkv, Hkv)]
    eager = [torch.empty_like(t) for t in outs]
    call = lambda o: TW.fpdt_tw_rope_fwd(*X.split([Hq, Hkv, Hkv], 1), *o, fd, positions=pos)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        call(outs)
    for k in range(3):
        X.normal_()
        pos += 1000 * k
        graph.replay()
        call(eager)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, eager))
