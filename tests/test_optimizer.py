"""Gradient norm and AdamW over lists of tensors (fpdt_tw_grad_norm, fpdt_tw_adamw_*): oracle pins and refusals (no GPU), and
GPU parity against the oracle."""
import ctypes
import math
import weakref

import numpy as np
import pytest
import torch

import kernel_resources
from oracle import tokenwise as otw
from paper_2408_16978_amd import tokenwise as TW

HYPER = dict(lr=1e-2, beta1=0.9, beta2=0.95, eps=1e-8)


# ------------------------------------------------------------------ oracle pins (CPU)
def test_adamw_oracle_against_torch():
    r = np.random.default_rng(4)
    p = torch.tensor(r.standard_normal(50), requires_grad=True)
    opt = torch.optim.AdamW([p], lr=1e-2, betas=(0.9, 0.95), eps=1e-8, weight_decay=0.1)
    q, m, v = p.detach().numpy().copy(), np.zeros(50), np.zeros(50)
    for step in range(1, 6):
        g = r.standard_normal(50)
        p.grad = torch.tensor(g)
        opt.step()
        q, m, v = otw.adamw(q, g, m, v, weight_decay=0.1, step=step, **HYPER)
        np.testing.assert_allclose(q, p.detach().numpy(), rtol=1e-12)


@pytest.mark.parametrize("signed", [True, False])
def test_state_codes_of_the_oracle(signed):
    """Every code's value is its own rounding, whatever decides; a value between two codes goes up as often as it is far; the
    random numbers are spread evenly, and differ from step to step and tensor to tensor."""
    codes = np.arange(256 if not signed else 128)
    code = np.zeros(256, dtype=np.int64)
    code[:len(codes)] = codes
    exp = np.array([120, 120])
    value = otw.state_value(code, exp, signed)
    if signed:
        value[128:] = value[127]  # the same largest value in both blocks
    else:
        value[:128][-1] = value[255]
    for chance in (0.0, 0.5, 65535 / 65536):
        got, _, e = otw.state_rounded(value, np.full(256, chance), signed)
        assert np.array_equal(got, value) and (e == 120).all()
    x = np.full(128, 1.0 + 0.3 / 8)
    x[0] = 1.5
    a = otw.state_chances(65536, 3, 7, 0)[0 if signed else 1]
    ups = np.concatenate([otw.state_rounded(x, c, signed)[0][1:] > 1.1 for c in a.reshape(-1, 128)])
    assert abs(ups.mean() - 0.3) < 4 * math.sqrt(0.3 * 0.7 / ups.size)
    for other in ((3, 8, 0), (3, 7, 1), (4, 7, 0)):
        b = otw.state_chances(65536, *other)[0 if signed else 1]
        assert abs(np.corrcoef(a, b)[0, 1]) < 4 / 256 and abs(np.histogram(b, 16)[0] / 4096 - 1).max() < 5 / 64


def _chances(n, seed, step, k):
    """oracle.tokenwise.state_chances of many elements at once"""
    def mix(x):
        x = x ^ x >> np.uint64(15)
        x = x * np.uint64(0xB7E15163) & low
        x = x ^ x >> np.uint64(13)
        x = x * np.uint64(0x93C467E3) & low
        return x ^ x >> np.uint64(16)
    low = np.uint64(2 ** 32 - 1)
    key = otw._mix(otw._mix(otw._mix(seed ^ 0x243F6A88) ^ (step * 0x9E3779B1 % 2 ** 32)) ^ (k * 0x85A308D3 % 2 ** 32))
    r = mix((np.arange(n, dtype=np.uint64) * np.uint64(0x9E3779B1) & low) ^ np.uint64(key)).astype(np.int64)
    return (r % 65536) / 65536.0, (r // 65536) / 65536.0


def test_chances_of_many_elements_are_those_of_the_oracle():
    for args in ((3000, 11, 7, 2), (1, 2 ** 32 - 1, 1, 0)):
        assert all(np.array_equal(a, b) for a, b in zip(_chances(*args), otw.state_chances(*args)))


def test_state_bytes_of_huge_tiny_and_other_values():
    for signed in (True, False):
        x = np.zeros(384)
        x[0], x[128], x[129], x[256] = np.inf, 1e-35, 0.0, 1.9
        got, _, e = otw.state_rounded(x, np.full(384, 0.25), signed)
        assert e.tolist() == [255, 40, 128] and np.isnan(got[:128]).all()
        assert (got[129:256] == 0).all() and got[256] == 1.875


# ------------------------------------------------------------------ refusals (CPU)
def _list(**kw):
    t = (TW._Param * 2)()
    for i in range(2):
        base = 0x10000000 * (i + 1)
        d = dict(n=1000, g=base, p=base + 0x100000, w=base + 0x200000, m=base + 0x300000, v=base + 0x400000, m_exp=base + 0x500000, v_exp=base + 0x600000,
                 m_value=base + 0x700000, v_value=base + 0x800000, weight_decay=0.1)
        if i == 1:
            d.update(kw)
        for k, x in d.items():
            setattr(t[i], k, x)
    return t


def _norm(t, **kw):
    a = dict(t=t, count=2, grads=0, most=1.0, out=0x1000, ws=0x100000, wsb=1 << 20)
    a.update(kw)
    return TW.load().fpdt_tw_grad_norm(*[a[k] for k in ("t", "count", "grads", "most", "out", "ws", "wsb")], None)


def _step(t, **kw):
    a = dict(t=t, count=2, grads=0, bits=32, lr=1e-3, b1=0.9, b2=0.95, eps=1e-8, step=1, lr_dev=None, step_dev=None, scale=None, seed=0, flags=0)
    a.update(kw)
    return TW.load().fpdt_tw_adamw_step(*[a[k] for k in ("t", "count", "grads", "bits", "lr", "b1", "b2", "eps", "step", "lr_dev", "step_dev", "scale",
                                                         "seed", "flags")], None)


def test_norm_refused():
    assert _norm(None) == 1 and _norm(_list(), count=0) == 1 and _norm(_list(), grads=2) == 1
    assert _norm(_list(n=-1)) == 1 and _norm(_list(g=None)) == 1 and _norm(_list(g=0x20000002)) == 1 and _norm(_list(g=0x20000001), grads=1) == 1
    assert "tensor 1" in TW.fpdt_tw_last_error()
    for most in (0.0, -1.0, math.nan):
        assert _norm(_list(), most=most) == 1
    assert _norm(_list(), out=None) == 1 and _norm(_list(), out=0x1002) == 1
    assert _norm(_list(), ws=None) == 3 and _norm(_list(), ws=0x100010) == 3 and _norm(_list(), wsb=8191) == 3
    assert _norm(_list(n=1 << 40)) == 2
    size = TW.load().fpdt_tw_grad_norm_workspace_bytes
    assert size(0) == 0 and size(1) == size(192) == 8192 and size(193) == 16384


@pytest.mark.parametrize("status,tensor,call", [
    (1, {}, dict(count=0)), (1, {}, dict(grads=5)), (1, {}, dict(bits=16)), (1, {}, dict(lr=-1.0)), (1, {}, dict(lr=math.nan)), (1, {}, dict(b1=1.0)),
    (1, {}, dict(b2=-0.1)), (1, {}, dict(b2=math.nan)), (1, {}, dict(eps=-1e-8)), (1, {}, dict(step=0)), (1, {}, dict(flags=2)), (1, {}, dict(lr_dev=0x1002)),
    (1, {}, dict(step_dev=0x1004)), (1, {}, dict(scale=0x1002)), (1, dict(n=-5), {}), (1, dict(g=None), {}), (1, dict(p=None), {}), (1, dict(m=None), {}),
    (1, dict(v=None), {}), (1, dict(m_exp=None), dict(bits=8)), (1, dict(v_exp=None), dict(bits=8)), (1, dict(p=0x20100002), {}), (1, dict(w=0x20200001), {}),
    (1, dict(v=0x20400002), {}), (1, dict(weight_decay=math.inf), {}), (2, dict(n=1 << 36), {})])
def test_step_refused(status, tensor, call):
    assert _step(_list(**tensor), **call) == status and TW.fpdt_tw_last_error() != ""


def test_unpack_refused():
    f = TW.load().fpdt_tw_adamw_unpack
    assert f(None, 2, None) == 1 and f(_list(), 0, None) == 1
    for bad in (dict(m=None), dict(v_exp=None), dict(m_value=None), dict(v_value=0x20800001), dict(n=-1)):
        assert f(_list(**bad), 2, None) == 1, bad
    assert f(_list(n=1 << 36), 2, None) == 2


def test_lists_are_checked_where_they_are_made():
    z = lambda n, dt=torch.float32: torch.zeros(n, dtype=dt)
    ok = dict(g=[z(300)], p=[z(300)], m=[z(300)], v=[z(300)])
    assert TW.FpdtTwParams(**ok).state_bits == 32
    eight = dict(ok, m=[z(300, torch.uint8)], v=[z(300, torch.uint8)], m_exp=[z(3, torch.uint8)], v_exp=[z(3, torch.uint8)])
    assert TW.FpdtTwParams(**eight).state_bits == 8
    for bad, error in ((dict(p=[z(299)]), ValueError), (dict(p=[z(300, torch.bfloat16)]), TypeError), (dict(w=[z(300)]), TypeError), (dict(m=[]), ValueError), (dict(g=[]), ValueError),
                       (dict(p=[z(600)[::2]]), ValueError), (dict(m=ok["v"]), ValueError), (dict(g=[z(300, torch.float16)]), TypeError),
                       (dict(weight_decay=[0.1, 0.2]), ValueError), (dict(v=[z(300, torch.uint8)]), TypeError)):
        with pytest.raises(error):
            TW.FpdtTwParams(**dict(ok, **bad))
    with pytest.raises(ValueError, match="elements"):
        TW.FpdtTwParams(**dict(eight, m_exp=[z(2, torch.uint8)]))
    t = z(500)
    with pytest.raises(ValueError, match="overlap"):  # the same tensor twice, or a part of it
        TW.FpdtTwParams(g=[z(300), z(300)], p=[t[:300], t[200:]], m=[z(300), z(300)], v=[z(300), z(300)])
    with pytest.raises(ValueError, match="current device"):
        TW.fpdt_tw_adamw_unpack(TW.FpdtTwParams(**eight))
    assert ctypes.sizeof(TW._Param) == 88


def test_a_list_keeps_its_tensors_when_the_callers_lists_change():
    """The library has their addresses: neither an emptied or refilled list nor a parameter that is given other memory may free them."""
    z = lambda n, dt=torch.float32: torch.zeros(n, dtype=dt)
    lists = dict(g=[z(300), z(40)], p=[z(300), z(40)], w=[None, z(40, torch.bfloat16)], m=[z(300, torch.uint8), z(40, torch.uint8)],
                 v=[z(300, torch.uint8), z(40, torch.uint8)], m_exp=[z(3, torch.uint8), z(1, torch.uint8)], v_exp=[z(3, torch.uint8), z(1, torch.uint8)])
    held = TW.FpdtTwParams(**lists)
    refs = {(k, i): weakref.ref(t) for k, ts in lists.items() for i, t in enumerate(ts) if t is not None}
    for k, ts in lists.items():
        if k == "g":
            ts[0] = z(300)
        elif k != "p":
            ts.clear()
    p = lists["p"][1]
    p.data = z(40)
    assert p.data_ptr() != held.array[1].p
    freed = [k for k, r in refs.items() if r() is None]
    assert not freed, freed
    # the memory as well, also where the tensor has another by now: what is taken from the allocator next lies elsewhere
    taken = {t.data_ptr() for t in [z(40) for _ in range(64)]}
    assert held.array[1].p not in taken
    assert any(s.data_ptr() == held.array[1].p for _, s in held._keep)


@pytest.mark.parametrize("source", ["tw_optim.hip", "tw_rope.hip", "tw_norm.hip"])
def test_no_scratch_memory(source):
    """What a thread has under way stays in registers; but for layer norms' backward over fp32 rows of more than 8192 columns,
    whose rows do not fit those of 16 waves."""
    found = {n: v[2] for n, v in kernel_resources.kernels(source).items() if v[2]}
    assert all(n.startswith("norm_bwd_kernel<float, 0, 4, true") and b <= 64 for n, b in found.items()), found


# ------------------------------------------------------------------ GPU parity
class Model:
    """Tensors of `sizes` on the GPU, some `off` elements behind a boundary, each with 8 elements of its buffer before and
    behind it that must stay."""

    def __init__(self, sizes, bits=32, grads=torch.float32, copies=True, seed=1, off=0, fresh=False, decay=0.1):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.sizes, self.bits, self.buffers = sizes, bits, []
        n = lambda k, std: torch.randn(k, device="cuda", generator=gen) * std
        place = lambda k, x: self._place(k, x, off)
        self.g = [place("g", n(k, 1e-2).to(grads)) for k in sizes]
        self.p = [place("p", n(k, 0.5)) for k in sizes]
        self.w = [place("w", p.to(torch.bfloat16)) for p in self.p] if copies else None
        more = {}
        if bits == 32:
            self.m = [place("m", n(k, 0.0 if fresh else 1e-3)) for k in sizes]
            self.v = [place("v", n(k, 0.0 if fresh else 1e-2).square()) for k in sizes]
        else:
            code = lambda k: torch.randint(0, 256, (k,), device="cuda", generator=gen, dtype=torch.uint8) * (not fresh)
            exp = lambda k, e: (torch.randint(-3, 4, (-(-k // 128),), device="cuda", generator=gen) + e).to(torch.uint8) * (not fresh)
            self.m, self.v = [place("m", code(k)) for k in sizes], [place("v", code(k)) for k in sizes]
            self.me, self.ve = [place("me", exp(k, 118)) for k in sizes], [place("ve", exp(k, 113)) for k in sizes]
            self.mv, self.vv = ([place("value", torch.zeros(k, dtype=torch.bfloat16, device="cuda")) for k in sizes] for _ in range(2))
            more = dict(m_exp=self.me, v_exp=self.ve, m_value=self.mv, v_value=self.vv)
        self.decay = [decay * (k % 2) for k in range(len(sizes))]
        self.list = TW.FpdtTwParams(g=self.g, p=self.p, m=self.m, v=self.v, w=self.w, weight_decay=self.decay, **more)

    def _place(self, kind, x, off):
        b = torch.full((x.numel() + 16 + off,), 77, dtype=x.dtype, device="cuda")
        t = b[8 + off:8 + off + x.numel()]
        t.copy_(x)
        self.buffers.append((b, 8 + off, 8 + off + x.numel()))
        return t

    def state(self):
        f = lambda ts: [t.double().cpu().numpy() for t in ts]
        if self.bits == 32:
            return f(self.p), f(self.g), f(self.m), f(self.v)
        value = lambda c, e, s: [otw.state_value(a.cpu().numpy(), b.cpu().numpy(), s) for a, b in zip(c, e)]
        return f(self.p), f(self.g), value(self.m, self.me, True), value(self.v, self.ve, False)

    def bits_of_all(self):
        return [b.clone() for b, _, _ in self.buffers]

    def check_surroundings(self):
        for b, i, j in self.buffers:
            assert (b[:i] == 77).all() and (b[j:] == 77).all()


def _check_step(model, before, step, scale=1.0, seed=0, hyper=HYPER):
    """Against the oracle in 64 bits.  m, v: three roundings of 2^-24 of their terms.  The move: root, quotient, products and
    factors, eight of 2^-24, and half of v's, relative to it: 2^-20 with m's share; p: two more of p.  8-bit states: the code that the
    oracle's decision gives, or the one beside it where the decision is within 2^-18 of a step (their values before it are
    2^-22 of themselves apart, a step is an eighth to a sixteenth of them)."""
    P, G, M, V = before
    now = model.state()
    for k, n in enumerate(model.sizes):
        p, m, v = otw.adamw(P[k], G[k], M[k], V[k], weight_decay=model.decay[k], step=step, scale=scale, **hyper)
        m_terms = np.abs(hyper["beta1"] * M[k]) + np.abs((1 - hyper["beta1"]) * G[k] * scale)
        root = np.sqrt(v / (1 - hyper["beta2"] ** step)) + hyper["eps"]
        tol = 2.0 ** -22 * np.abs(P[k]) + hyper["lr"] * 2.0 ** -20 * m_terms / (1 - hyper["beta1"] ** step) / root
        assert (np.abs(now[0][k] - p) <= tol).all(), k
        if model.w is not None:
            assert torch.equal(model.w[k], model.p[k].to(torch.bfloat16))
        if model.bits == 32:
            assert (np.abs(now[2][k] - m) <= 2.0 ** -22 * m_terms).all() and (np.abs(now[3][k] - v) <= 2.0 ** -22 * v).all()
            continue
        chances = otw.state_chances(n, seed, step, k)
        for got, x, chance, exp, signed in ((now[2][k], m, chances[0], model.me[k], True), (now[3][k], v, chances[1], model.ve[k], False)):
            want, slack, e = otw.state_rounded(x, chance, signed)
            assert np.array_equal(exp.cpu().numpy(), e)
            off = ~((got == want) | (np.isnan(got) & np.isnan(want)))
            assert (slack[off] < 2.0 ** -18).all() and (np.abs(got - want)[off] <= np.abs(want[off]) / 8 + 1e-30).all(), (k, off.sum())


RAGGED = [1, 7, 128, 129, 4096, 4097, 5000, 0, 131, 20000, 2, 127]


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("grads", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("off,copies", [(0, True), (1, True), (3, False)])
def test_gpu_steps_match_the_oracle(bits, grads, off, copies):
    print("[case] adamw", bits, grads, off, copies, flush=True)
    model = Model(RAGGED, bits, grads, copies, off=off)
    for step in (1, 2, 1000):
        before = model.state()
        TW.fpdt_tw_adamw_step(model.list, step=step, seed=11, **HYPER)
        torch.cuda.synchronize()
        _check_step(model, before, step, seed=11)
    if bits == 8:
        TW.fpdt_tw_adamw_unpack(model.list)
        torch.cuda.synchronize()
        _, _, M, V = model.state()
        for k in range(len(RAGGED)):
            assert np.array_equal(model.mv[k].double().cpu().numpy(), M[k]) and np.array_equal(model.vv[k].double().cpu().numpy(), V[k])
    model.check_surroundings()


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("beta1,beta2,eps,lr", [(0.0, 0.0, 1e-3, 1e-2), (0.9, 0.999, 1e-8, 0.0), (0.0, 0.99, 1.0, 1e-1)])
def test_gpu_hyperparameters_at_their_ends(bits, beta1, beta2, eps, lr):
    hyper = dict(lr=lr, beta1=beta1, beta2=beta2, eps=eps)
    model = Model([300, 5000], bits, fresh=True)
    for step in (1, 2):
        before = model.state()
        TW.fpdt_tw_adamw_step(model.list, step=step, seed=2 ** 32 - 1, **hyper)
        torch.cuda.synchronize()
        _check_step(model, before, step, seed=2 ** 32 - 1, hyper=hyper)


@pytest.mark.gpu
@pytest.mark.parametrize("large", [False, True])
def test_gpu_a_first_step_from_zero_is_the_rate_to_the_bit(large):
    """Both betas 0, eps 0, a rate that is a power of two: v is g^2 rounded once, the root of which, rounded once, is |g|
    again (short of overflow and underflow, as with any correctly rounded root), m times the rate is exact, and the quotient is the rate.  p is its
    move then, and nothing else: root and quotient have to be right to half a step for this to hold for every g."""
    model = Model([70000, 1, 4097] + ([4096 * 1024] if large else []), decay=0.5, fresh=True, seed=12)
    for p, g in zip(model.p, model.g):
        p.zero_()
        g.mul_(torch.exp2(torch.randint(-20, 21, g.shape, device="cuda").float()))
    TW.fpdt_tw_adamw_step(model.list, lr=2.0 ** -7, beta1=0.0, beta2=0.0, eps=0.0, step=1)
    torch.cuda.synchronize()
    for p, g in zip(model.p, model.g):
        assert (g != 0).all() and torch.equal(p, -torch.sign(g) * 2.0 ** -7)


def _check_long(model, before, step, scale, seed):
    """_check_step for millions of elements, among which some m are the small difference of their terms, and for factors that are no power of two.  m: the
    gradient times its factor, 1 - beta1 as a float, their product and the sum are four roundings of 2^-24, 2^-22 of the terms' sizes; v: the first
    of them counts twice in the square, which is rounded itself, so 6 in all: 2^-21.  p: m's four, v's six halved, and root, quotient, products and factors: under 16,
    2^-20.  8-bit states: m is 2^-22 terms / |m| of itself off before it is rounded, and it is 8 to 16 steps: the decision may be the other one within
    2^-18 terms / |m| of a step (v, whose terms have one sign: 2^-17).  Below the smallest code a step is that code, and m less than one.  A block whose largest
    is as near to 1.875 of a power of two, where its exponent changes (bf16 gradients and codes have few bits, and meet it exactly), may have the other exponent:
    the codes stand for the same values, but for the smallest."""
    P, G, M, V = before
    now = model.state()
    for k, n in enumerate(model.sizes):
        p, m, v = otw.adamw(P[k], G[k], M[k], V[k], weight_decay=model.decay[k], step=step, scale=scale, **HYPER)
        m_terms = np.abs(HYPER["beta1"] * M[k]) + np.abs((1 - HYPER["beta1"]) * G[k] * scale)
        root = np.sqrt(v / (1 - HYPER["beta2"] ** step)) + HYPER["eps"]
        tol = 2.0 ** -22 * np.abs(P[k]) + HYPER["lr"] * 2.0 ** -20 * m_terms / (1 - HYPER["beta1"] ** step) / root
        assert (np.abs(now[0][k] - p) <= tol).all(), k
        assert torch.equal(model.w[k], model.p[k].to(torch.bfloat16))
        if model.bits == 32:
            assert (np.abs(now[2][k] - m) <= 2.0 ** -22 * m_terms).all() and (np.abs(now[3][k] - v) <= 2.0 ** -21 * v).all()
            continue
        chances = _chances(n, seed, step, k)
        for got, x, terms, chance, exp, signed in ((now[2][k], m, m_terms, chances[0], model.me[k], True), (now[3][k], v, 2 * v, chances[1], model.ve[k], False)):
            want, slack, e = otw.state_rounded(x, chance, signed)
            exp, blocks = exp.cpu().numpy().astype(np.int64), -(-n // 128)
            other = np.flatnonzero(exp != e)
            whole = lambda a: np.concatenate([np.abs(a), np.zeros(blocks * 128 - n)]).reshape(blocks, 128).max(axis=1)[other] if n else a
            border = 1.875 * 2.0 ** (np.minimum(exp, e)[other] - 127)
            assert (np.abs(exp - e)[other] == 1).all() and (np.abs(whole(x) - border) <= 2.0 ** -22 * whole(terms)).all(), (k, other)
            small = np.repeat(np.where(exp != e, 2.0 ** (np.maximum(exp, e) - 127 - (15 if signed else 31) + 1), 0.0), 128)[:n]
            off = (got != want) & (np.abs(x) >= small)
            near = slack[off] * np.abs(x[off]) <= 2.0 ** -18 * terms[off]
            assert near.all() and (np.abs(got - want)[off] <= np.abs(want[off]) / 8 + 1e-30).all(), (k, off.sum())


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("grads", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("off", [0, 1])
def test_gpu_lists_of_whole_large_units(bits, grads, off):
    """Lists of 1024 units of 4096 elements (8-bit states: 2048) or more take other kernels than short ones: units that are whole, units that are cut off, tensors
    of less than one, clipped, with cleared gradients, and passed over."""
    print("[case] large units", bits, grads, off, flush=True)
    unit = 4096 if bits == 32 else 2048
    model = Model([unit * 1024 + 5, 0, unit + 1, 1, 3 * unit, unit - 1, 130], bits, grads, off=off, seed=bits + off)
    scale = torch.tensor([math.nan], device="cuda")
    was = model.bits_of_all()
    step = lambda k, flags=0: TW.fpdt_tw_adamw_step(model.list, step=k, grad_scale=scale, seed=5, flags=flags, **HYPER)
    step(4)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(was, model.bits_of_all()))
    scale.fill_(0.5)
    for k, flags in ((4, 0), (5, TW.FPDT_TW_ADAMW_ZERO_GRAD)):
        before = model.state()
        step(k, flags)
        torch.cuda.synchronize()
        _check_long(model, before, k, 0.5, 5)
    assert all((g == 0).all() for g in model.g)
    for g in model.g:
        g.fill_(1.0)
    scale.fill_(math.inf)
    was = model.bits_of_all()
    step(6, TW.FPDT_TW_ADAMW_ZERO_GRAD)
    torch.cuda.synchronize()
    n = len(model.sizes)
    assert all((g == 0).all() for g in model.g) and all(torch.equal(a, b) for a, b in zip(was[n:], model.bits_of_all()[n:]))
    if bits == 8:
        TW.fpdt_tw_adamw_unpack(model.list)
        torch.cuda.synchronize()
        _, _, M, V = model.state()
        assert all(np.array_equal(a.double().cpu().numpy(), b, equal_nan=True) for a, b in zip(model.mv + model.vv, M + V))
    model.check_surroundings()


@pytest.mark.gpu
@pytest.mark.parametrize("most", [1e-3, 1e3, math.inf])
@pytest.mark.parametrize("grads", [torch.float32, torch.bfloat16])
def test_gpu_norm_and_factor_of_one_tensor(grads, most):
    """One tensor, clipped and not: norm and factor each rounded once to fp32 (sums and roots in 64 bits; 1% of that for those)."""
    g = [(torch.randn(37, device="cuda") * 0.01).to(grads)]
    out, ws = torch.zeros(2, device="cuda"), torch.empty(8192, dtype=torch.uint8, device="cuda")
    TW.fpdt_tw_grad_norm(TW.FpdtTwParams(g=g), most, out, ws)
    torch.cuda.synchronize()
    norm, factor = otw.grad_norm([g[0].double().cpu().numpy()], most)
    assert (factor < 1) == (most < 1)
    assert abs(out[0].item() - norm) <= 2.0 ** -24 * norm * 1.01
    assert abs(out[1].item() - factor) <= 2.0 ** -24 * factor * 1.01


@pytest.mark.gpu
def test_gpu_moments_at_the_ends_of_the_range():
    """g^2 beyond fp32 (v is infinite and the move none, as in fp32's own arithmetic), v that is no normal number, m so small that its move is none:
    p stays a number, and as it was; a v that is not a number makes p none."""
    model = Model([8], fresh=True, decay=0.0)
    p, g, m, v = model.p[0], model.g[0], model.m[0], model.v[0]
    g[:] = torch.tensor([1e30, -1e30, 0.0, 1e-30, 1e-22, 0.0, 0.0, 0.0], device="cuda")
    v[:] = torch.tensor([0.0, 1e38, 1e-40, 0.0, 0.0, math.inf, math.nan, 0.0], device="cuda")
    m[:] = torch.tensor([0.0, 0.0, 0.0, 0.0, 0.0, 3.0, 0.0, 0.0], device="cuda")
    was = p.clone()
    TW.fpdt_tw_adamw_step(model.list, step=1, **HYPER)
    torch.cuda.synchronize()
    assert torch.isnan(p).tolist() == [False] * 6 + [True, False]
    assert torch.equal(p[[0, 1, 2, 5, 7]], was[[0, 1, 2, 5, 7]])
    # (g^2 is lost, or all of it but its size; eps 1e-8 is what is left of the root: moves of 1e-24 and 1e-16 are none)
    assert torch.equal(p[3:5], was[3:5]) and torch.isinf(v[[0, 1, 5]]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("count", [1, 47, 49, 200])
def test_gpu_many_tensors_norm_clip_step_and_zeroed_gradients(bits, count):
    sizes = [(37 * k) % 700 for k in range(1, count + 1)]
    model = Model(sizes, bits, seed=count)
    out, ws = torch.zeros(2, device="cuda"), torch.empty(TW.fpdt_tw_grad_norm_workspace_bytes(model.list), dtype=torch.uint8, device="cuda")
    norm, factor = otw.grad_norm([g.double().cpu().numpy() for g in model.g], 0.05)
    TW.fpdt_tw_grad_norm(model.list, 0.05, out, ws)
    before = model.state()
    TW.fpdt_tw_adamw_step(model.list, step=3, grad_scale=out[1:], flags=TW.FPDT_TW_ADAMW_ZERO_GRAD, **HYPER)
    torch.cuda.synchronize()
    got = out.double().cpu().numpy()
    assert abs(got[0] - norm) <= 2.0 ** -24 * norm * 1.01 and abs(got[1] - factor) <= 2.0 ** -24 * factor * 1.01 and factor < 1 or count == 1
    _check_step(model, before, 3, scale=float(got[1]))
    assert all((g == 0).all() for g in model.g)
    model.check_surroundings()


@pytest.mark.gpu
@pytest.mark.parametrize("grads", [torch.float32, torch.bfloat16])
def test_gpu_norm_of_large_small_and_other_gradients(grads):
    """Squares that a float does not hold, several units a workgroup, none at all, no limit; and what is not finite."""
    out = torch.zeros(2, device="cuda")
    ws = torch.full((8192,), 255, dtype=torch.uint8, device="cuda")
    for sizes, std in (([1], 1.0), ([16384 * 1100 + 5, 3], 1e-3), ([5000, 1], 1e30), ([5000], 1e-30), ([0, 0], 1.0)):
        gen = torch.Generator(device="cuda").manual_seed(len(sizes))
        g = [(torch.randn(n, device="cuda", generator=gen) * std).to(grads) for n in sizes]
        for most in (1e-2, math.inf):
            TW.fpdt_tw_grad_norm(TW.FpdtTwParams(g=g), most, out, ws)
            torch.cuda.synchronize()
            norm, factor = otw.grad_norm([t.double().cpu().numpy() for t in g], most)
            assert abs(out[0].item() - norm) <= 2.0 ** -24 * norm * 1.01 + 2.0 ** -149, (sizes, std)
            assert abs(out[1].item() - factor) <= 2.0 ** -24 * factor * 1.01, (sizes, std, most)
    for bad in (math.inf, -math.inf, math.nan):
        g = [torch.ones(5000, device="cuda", dtype=grads) for _ in range(2)]
        g[1][4321] = bad
        TW.fpdt_tw_grad_norm(TW.FpdtTwParams(g=g), 1.0, out, ws)
        torch.cuda.synchronize()
        assert not math.isfinite(out[0].item()) and math.isnan(out[1].item())


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("scale", [math.nan, math.inf])
def test_gpu_a_step_whose_gradients_overflowed_is_passed_over(bits, scale):
    model = Model(RAGGED, bits)
    was = model.bits_of_all()
    s = torch.tensor([scale], device="cuda")
    TW.fpdt_tw_adamw_step(model.list, step=1, grad_scale=s, **HYPER)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(was, model.bits_of_all()))
    TW.fpdt_tw_adamw_step(model.list, step=1, grad_scale=s, flags=TW.FPDT_TW_ADAMW_ZERO_GRAD, **HYPER)
    torch.cuda.synchronize()
    n = len(RAGGED)
    assert all((g == 0).all() for g in model.g) and all(torch.equal(a, b) for a, b in zip(was[n:], model.bits_of_all()[n:]))
    model.check_surroundings()


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_gpu_copies_of_some_tensors_only(bits):
    """A tensor without a bf16 copy, and the same elements of it; lists that only the norm is taken of cannot be stepped."""
    a, b = Model([500, 300], bits, seed=6), Model([500, 300], bits, seed=6)
    more = {} if bits == 32 else dict(m_exp=b.me, v_exp=b.ve)
    some = TW.FpdtTwParams(g=b.g, p=b.p, m=b.m, v=b.v, w=[None, b.w[1]], weight_decay=b.decay, **more)
    was = b.w[0].clone()
    TW.fpdt_tw_adamw_step(a.list, step=1, **HYPER)
    TW.fpdt_tw_adamw_step(some, step=1, **HYPER)
    torch.cuda.synchronize()
    assert torch.equal(b.w[0], was) and torch.equal(a.w[1], b.w[1]) and all(torch.equal(x, y) for x, y in zip(a.p + a.m + a.v, b.p + b.m + b.v))
    with pytest.raises(TW.FpdtTwError) as e:
        TW.fpdt_tw_adamw_step(TW.FpdtTwParams(g=a.g), step=1, **HYPER)
    assert e.value.status == 1
    with pytest.raises(ValueError):
        TW.fpdt_tw_adamw_step(a.list, step=1, grad_scale=torch.ones(2, device="cuda"), **HYPER)


@pytest.mark.gpu
def test_gpu_8_bit_blocks_that_are_zero_huge_tiny_or_not_finite():
    """A gradient that is not finite makes its block NaN, and no other; zeros stay zeros; what is too small for a block goes to
    zero in m and not in v; signs are kept."""
    model = Model([640], 8, fresh=True, decay=0.0)
    g = model.g[0]
    g[:128] = 0
    g[128:256] = 1e-3
    g[200] = math.nan
    g[256:384] = 1.0
    g[300], g[301] = -1e-12, 0.0
    g[384:512] = 1e-18
    g[512:] *= -1
    before = model.state()
    TW.fpdt_tw_adamw_step(model.list, step=1, **HYPER)
    TW.fpdt_tw_adamw_unpack(model.list)
    torch.cuda.synchronize()
    m, v = model.mv[0].float(), model.vv[0].float()
    assert (m[:128] == 0).all() and (v[:128] == 0).all() and model.me[0][0] == 40
    assert torch.isnan(m[128:256]).all() and torch.isnan(v[128:256]).all() and model.me[0][1] == 255
    assert torch.isfinite(m[256:]).all() and torch.isfinite(v[256:]).all()
    assert m[300] == 0 and v[300] > 0 and v[301] == 0 and m[301] == 0
    assert (v[384:512] > 0).all() and (torch.sign(m[512:]) == torch.sign(g[512:]))[m[512:] != 0].all()
    # p: only the element whose gradient was not a number
    assert torch.isnan(model.p[0]).nonzero().flatten().tolist() == [200]
    after = model.state()
    keep = np.r_[256:640]
    part = lambda s: [[a[keep] for a in t] for t in s]
    ref = otw.adamw(*[t[0] for t in part(before)], weight_decay=0.0, step=1, **HYPER)[0]
    assert (np.abs(part(after)[0][0] - ref) <= 2.0 ** -21 * (np.abs(ref) + 1)).all()


@pytest.mark.gpu
def test_gpu_8_bit_moments_follow_slow_changes():
    """beta2 = 0.999: a step moves v by a thousandth of what is left, a sixtieth of half a code step: rounded to nearest it
    would not move.  With a constant gradient v has to reach (1 - 0.999^n) g^2 from zero, and to come down again.  Chance: a code
    step is at most v / 8, a step up or down is taken with probability f = 0.001 .. 1 and adds f (1 - f) (v / 8)^2 <= f v^2 / 64 of
    variance, of which 2 * 0.001 is lost a step: at most v^2 / 64 * max(f) / 0.002 -- where f is 0.008 to 0.016 (v near its end):
    0.13 v^2; earlier f is larger, but a step is then no part of 1 / 8 of the end's v.  So sigma <= 0.4 v for one element, and below 0.4 / 256
    = 0.16% for the mean of 65536; the random numbers have 16 bits, and cutting below them loses up to 2^-16 of a step each, 1000 * v / 8 *
    2^-16 = 0.2% of v at most.  2% is ten of the one and the other."""
    n = 65536
    model = Model([n], 8, fresh=True, decay=0.0, copies=False)
    hyper = dict(lr=0.0, beta1=0.9, beta2=0.999, eps=1e-8)
    g, want = 0.3, 0.0
    model.g[0].fill_(g)
    for step in range(1, 1201):
        if step == 801:
            g = 0.1
            model.g[0].fill_(g)
        TW.fpdt_tw_adamw_step(model.list, step=step, seed=5, **hyper)
        want = 0.999 * want + 0.001 * float(np.float32(g)) ** 2
        if step in (100, 800, 1200):
            TW.fpdt_tw_adamw_unpack(model.list)
            torch.cuda.synchronize()
            assert abs(model.vv[0].double().mean().item() / want - 1) < 0.02, step
    assert abs(model.mv[0].double().mean().item() / 0.1 - 1) < 0.02


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_gpu_captured_step_reads_step_and_rate_on_the_device(bits):
    """Norm and step captured once and replayed with eager steps of a twin between: the same bits, whatever step and lr
    are at each replay; on the host or the device they come to the same."""
    sizes = [300, 9000, 77]
    a, b = Model(sizes, bits, seed=3), Model(sizes, bits, seed=3)
    lr, step = torch.zeros(1, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
    outs, wss = [torch.zeros(2, device="cuda") for _ in range(2)], [torch.empty(8192, dtype=torch.uint8, device="cuda") for _ in range(2)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step.add_(1)
        TW.fpdt_tw_grad_norm(a.list, 0.3, outs[0], wss[0])
        TW.fpdt_tw_adamw_step(a.list, 0.0, 0.9, 0.95, 1e-8, 0, lr_dev=lr, step_dev=step, grad_scale=outs[0][1:], seed=9, flags=TW.FPDT_TW_ADAMW_ZERO_GRAD)
    for k in range(1, 5):
        g = torch.randn(9000, device="cuda")
        rate = float(np.float32(1e-2 / k))
        lr.fill_(rate)
        for m in (a, b):
            for t in m.g:
                t.copy_(g[:t.numel()])
        graph.replay()
        TW.fpdt_tw_grad_norm(b.list, 0.3, outs[1], wss[1])
        TW.fpdt_tw_adamw_step(b.list, rate, 0.9, 0.95, 1e-8, k, grad_scale=outs[1][1:], seed=9, flags=TW.FPDT_TW_ADAMW_ZERO_GRAD)
        torch.cuda.synchronize()
        assert step.item() == k and torch.equal(outs[0], outs[1])
        assert all(torch.equal(x, y) for x, y in zip(a.bits_of_all(), b.bits_of_all())), k


@pytest.mark.gpu
def test_gpu_elements_behind_2_to_32():
    """One tensor of 2^32 + 300 elements in 8 bits (38 GB): the last ones have offsets that pass 32 bits, and random numbers of a
    key of their own."""
    n = 2 ** 32 + 300
    tail = 1000
    if torch.cuda.mem_get_info()[0] < 64 << 30:
        pytest.skip("needs 64 GB")
    z = lambda dt, k=n: torch.zeros(k, dtype=dt, device="cuda")
    g, p, m, v, me, ve = z(torch.bfloat16), z(torch.float32), z(torch.uint8), z(torch.uint8), z(torch.uint8, -(-n // 128)), z(torch.uint8, -(-n // 128))
    gen = torch.Generator(device="cuda").manual_seed(8)
    for s in (slice(0, tail), slice(n - tail, n)):
        g[s] = torch.randn(tail, device="cuda", generator=gen).to(torch.bfloat16)
        p[s] = torch.randn(tail, device="cuda", generator=gen)
    params = TW.FpdtTwParams(g=[g], p=[p], m=[m], v=[v], m_exp=[me], v_exp=[ve])
    out, ws = torch.zeros(2, device="cuda"), torch.empty(8192, dtype=torch.uint8, device="cuda")
    TW.fpdt_tw_grad_norm(params, 1.0, out, ws)
    norm = otw.grad_norm([torch.cat([g[:tail], g[-tail:]]).double().cpu().numpy()], 1.0)[0]
    was = [torch.cat([t[:tail], t[-tail:]]).double().cpu().numpy() for t in (p, g)]
    TW.fpdt_tw_adamw_step(params, step=1, seed=1, **HYPER)
    torch.cuda.synchronize()
    assert abs(out[0].item() - norm) <= 2.0 ** -24 * norm * 1.01
    want = otw.adamw(was[0], was[1], 0 * was[0], 0 * was[0], weight_decay=0.0, step=1, **HYPER)
    got = torch.cat([p[:tail], p[-tail:]]).double().cpu().numpy()
    assert (np.abs(got - want[0]) <= 2.0 ** -22 * np.abs(was[0]) + HYPER["lr"] * 2.0 ** -20).all()
    # the states of the last whole blocks behind 2^32 (256 elements): key mix(key + 1)
    first = 2 ** 32
    key = otw._mix(otw._mix(otw._mix(1 ^ 0x243F6A88) ^ 0x9E3779B1) ^ 0)
    key = otw._mix((key + 1) % 2 ** 32)
    r = np.array([otw._mix((i * 0x9E3779B1 % 2 ** 32) ^ key) for i in range(256)])
    at = 2 * tail - 300
    for code, exp, x, chance, signed in ((m, me, want[1], (r % 65536) / 65536, True), (v, ve, want[2], (r // 65536) / 65536, False)):
        value = otw.state_value(code[first:first + 256].cpu().numpy(), exp[first // 128:first // 128 + 2].cpu().numpy(), signed)
        ref, slack, e = otw.state_rounded(x[at:at + 256], chance, signed)
        off = value != ref
        assert np.array_equal(exp[first // 128:first // 128 + 2].cpu().numpy(), e) and (slack[off] < 2.0 ** -18).all() and off.sum() <= 2
    assert (p[tail:2 ** 31] == 0).all()
