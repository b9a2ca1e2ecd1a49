"""The operators of a training step around the products and the attention, as timed cases.

A case is a dict of plain values.  `listed()` names the representative ones, `draw(rng)` gives
further ones over the ranges they stand for, `prepare(case, seed)` makes what a program holds
before the call, `run(state)` is one pass (the library's entry points where `own` is set,
elementary torch operations otherwise), `work(case)` the bytes and operations a pass cannot do
without, `exact(case, seed)` the pass in 64 bits from the definition.

Operators:
  rope       split of the fused QKV product into Q, K, V with rotary positions (forward), and the
             gradients' way back into the rows of the product (backward)
  norm       residual add and RMS / layer normalisation, forward or backward
  grad_norm  global norm of many gradients and the factor that clips it
  adamw      (clipped) AdamW step over many tensors, states in 32 or in 8 bits
"""
import math
import random

import torch

own = False

EPS_NORM = 1e-5
LR, BETA1, BETA2, EPS, STEP = 3e-4, 0.9, 0.95, 1e-8, 1000
BLOCK = 128  # elements of a block of 8-bit states


# ------------------------------------------------------------------------------------ cases
def _rope(direction, rows, Hq, Hkv, D, rot, layout, dtype="bf16", scaling="plain", given=False, start=0):
    return {"op": "rope", "direction": direction, "rows": rows, "Hq": Hq, "Hkv": Hkv, "D": D, "rot": rot, "layout": layout,
            "dtype": dtype, "scaling": scaling, "given": given, "start": start}


def _norm(direction, rows, hidden, kind="rms", dtype="bf16", residual=True):
    return {"op": "norm", "direction": direction, "rows": rows, "hidden": hidden, "kind": kind, "dtype": dtype, "residual": residual}


def _layers(op, layers, hidden, qkv, ffn, swiglu=True, **more):
    return dict({"op": op, "tensors": "layers", "layers": layers, "hidden": hidden, "qkv": qkv, "ffn": ffn, "swiglu": swiglu}, **more)


def _ragged(op, count, low, high, pick, **more):
    return dict({"op": op, "tensors": "ragged", "count": count, "low": low, "high": high, "pick": pick}, **more)


def listed():
    cases = {
        # 16 sequences decode a token each at Llama-8B's whole heads: every row its own far position; latency counts
        "rope_decode": _rope("fwd", 16, 32, 8, 128, 128, "half", given=True),
        # a 64K-token chunk of a 2M-token sequence at a Llama-8B head share, frequencies scaled by parts
        "rope_64k": _rope("fwd", 65536, 8, 2, 128, 128, "half", scaling="parts", start=1966080),
        # the way back at a GPT-2.7B head share (D = 80), interleaved pairs in part of each head, packed documents
        "rope_bwd_256k": _rope("bwd", 262144, 4, 4, 80, 32, "interleaved", given=True),
        # 16 rows of a decode step through the norm in front of a Llama-8B layer
        "norm_decode": _norm("fwd", 16, 4096),
        # a chunk of 64K tokens at Llama-8B width: residual add and norm
        "rms_64k": _norm("fwd", 65536, 4096),
        # the gradient of the same, the residual stream's gradient added
        "rms_bwd_64k": _norm("bwd", 65536, 4096),
        # GPT-2.7B's layer norm, backward over a ragged number of tokens, in fp32
        "layer_bwd_ragged": _norm("bwd", 30001, 2560, "layer", "f32"),
        # gradients of a small model: 150 ragged tensors, mostly latency
        "grad_norm_small": _ragged("grad_norm", 150, 64, 65536, 5, grads="f32"),
        # fp32 weight gradients of four Llama-8B layers
        "grad_norm_llama": _layers("grad_norm", 4, 4096, 6144, 14336, grads="f32"),
        # the small model's step
        "adamw_small": _ragged("adamw", 150, 64, 65536, 6, grads="f32", bits=32, clip=False),
        # one Llama-8B layer, clipped, states in 32 bits
        "adamw_llama": _layers("adamw", 1, 4096, 6144, 14336, grads="f32", bits=32, clip=True),
        # the same layer with states in 8 bits, looked at afterwards
        "adamw8_llama": _layers("adamw", 1, 4096, 6144, 14336, grads="f32", bits=8, clip=True),
    }
    return [dict(c, name=n) for n, c in cases.items()]


def _log(rng, lo, hi):
    return lo * (hi / lo) ** rng.random()


def draw(rng):
    op = rng.choice(["rope", "rope", "norm", "norm", "norm", "grad_norm", "adamw", "adamw"])
    if op == "rope":
        hq, hkv = rng.choice([(8, 2), (8, 1), (4, 4), (8, 8), (16, 2), (32, 8), (1, 1), (5, 5)])
        D = rng.choice([64, 80, 128, 128])
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        most = min(262144, 250_000_000 // ((hq + 2 * hkv) * D) // (2 if dtype == "f32" else 1))
        return _rope(rng.choice(["fwd", "bwd"]), int(_log(rng, 1, most)), hq, hkv, D, rng.choice([D, D, D // 2, 2 * rng.randint(1, D // 2)]),
                     rng.choice(["half", "interleaved"]), dtype, rng.choice(["plain", "parts"]), rng.random() < 0.5, rng.randint(0, 1 << 21))
    if op == "norm":
        hidden = rng.choice([1024, 2560, 4096, 4096, 5120, 8192, rng.randint(64, 12000), 8 * rng.randint(8, 1500)])
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        most = min(131072, 268_000_000 // hidden // (2 if dtype == "f32" else 1))
        return _norm(rng.choice(["fwd", "bwd"]), int(_log(rng, 1, most)), hidden, rng.choice(["rms", "rms", "layer"]), dtype, rng.random() < 0.8)
    count = int(_log(rng, 1, 200))
    high = int(_log(rng, 2000, max(4000, min(100_000_000, 400_000_000 // count))))
    more = {"grads": rng.choice(["f32", "f32", "bf16"])}
    if op == "adamw":
        more.update(bits=rng.choice([32, 8]), clip=rng.random() < 0.5)
    return _ragged(op, count, int(_log(rng, 1, 1000)), high, rng.randint(1, 9999), **more)


def _sizes(case):
    """Elements of each tensor."""
    if case["tensors"] == "layers":
        h, f = case["hidden"], case["ffn"]
        return [case["qkv"] * h, h * h, h * f, h * f, h, h] * case["layers"] if not case["swiglu"] else [case["qkv"] * h, h * h, h * f, h * f, h * f, h, h] * case["layers"]
    rng, most, sizes = random.Random(case["pick"]), 180_000_000, []
    for _ in range(case["count"]):
        sizes.append(max(1, min(int(_log(rng, case["low"], case["high"])), most - sum(sizes))))
    return sizes


# ------------------------------------------------------------------------------------ inputs
_TYPE = {"f32": torch.float32, "bf16": torch.bfloat16}


def _freqs(rot, scaling, device):
    """Radians per token of each pair: 500000^(-2i/rot); by parts: divided by 8 where a context of 8192
    tokens sees less than one turn, left where it sees more than four, and in between a mixture."""
    f = 500000.0 ** (-torch.arange(rot // 2, dtype=torch.float64, device=device) * 2 / rot)
    if scaling == "parts":
        keep = ((8192 * f / (2 * math.pi) - 1) / 3).clamp(0, 1)
        f = keep * f + (1 - keep) * f / 8
    return f


def _offsets(sizes):
    """Where each tensor begins in a buffer of them all (blocks do not cross tensors), and its length."""
    at, total = [], 0
    for n in sizes:
        at.append(total)
        total += (n + BLOCK - 1) // BLOCK * BLOCK
    return at, total


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *s, std=1.0: torch.randn(*s, device="cuda", generator=gen) * std  # noqa: E731
    if case["op"] == "rope":
        dt, rows, Hq, Hkv, D = _TYPE[case["dtype"]], case["rows"], case["Hq"], case["Hkv"], case["D"]
        s = {"case": case, "freqs": _freqs(case["rot"], case["scaling"], "cuda"), "positions": None, "amplitude": 1.0}
        if case["scaling"] == "parts":
            s["amplitude"] = 0.1 * math.log(8.0) + 1.0
        if case["given"]:
            s["positions"] = torch.randint(0, 1 << 21, (rows,), device="cuda", generator=gen)
        make = normal if case["direction"] == "fwd" else None
        s["qkv"] = normal(rows, (Hq + 2 * Hkv) * D).to(dt) if make else torch.empty(rows, (Hq + 2 * Hkv) * D, dtype=dt, device="cuda")
        for name, h in (("q", Hq), ("k", Hkv), ("v", Hkv)):
            s[name] = torch.empty(rows, h, D, dtype=dt, device="cuda") if make else normal(rows, h, D, std=1e-2).to(dt)
        return s
    if case["op"] == "norm":
        dt, rows, hidden = _TYPE[case["dtype"]], case["rows"], case["hidden"]
        layer = case["kind"] == "layer"
        s = {"case": case, "w": (1 + normal(hidden, std=0.1)).to(dt), "b": normal(hidden, std=0.1).to(dt) if layer else None}
        x = (normal(rows, hidden) + normal(hidden, std=0.5)).to(dt)
        y = normal(rows, hidden, std=0.1 if case["direction"] == "fwd" else 1e-2).to(dt)  # what a layer adds, or the gradient that reaches the norm
        if case["direction"] == "fwd":
            s.update(x=x, r=y if case["residual"] else None, sum=torch.empty_like(x) if case["residual"] else None, y=torch.empty_like(x),
                     stats=torch.empty((2, rows) if layer else (1, rows), device="cuda"))
            return s
        f = x.double()
        mean = f.mean(1) if layer else torch.zeros(rows, dtype=torch.float64, device="cuda")
        rstd = ((f - mean[:, None]).square().mean(1) + EPS_NORM).rsqrt()
        s.update(x=x, dy=y, dr=normal(rows, hidden, std=1e-2).to(dt) if case["residual"] else None, dx=torch.empty_like(x),
                 stats=torch.stack([mean, rstd] if layer else [rstd]).float(), dw=normal(hidden, std=1e-2), db=normal(hidden, std=1e-2) if layer else None)
        if own:
            from paper_2408_16978_amd import tokenwise as TW
            s["workspace"] = torch.empty(TW.fpdt_tw_norm_bwd_workspace_bytes(rows, hidden, TW.FPDT_TW_LAYERNORM if layer else TW.FPDT_TW_RMSNORM), dtype=torch.uint8, device="cuda")
        return s
    sizes = _sizes(case)
    at, total = _offsets(sizes)
    here = torch.zeros(total, dtype=torch.bool, device="cuda")  # what belongs to a tensor
    here.view(-1, BLOCK)[:] = True
    inside = torch.arange(total, device="cuda")
    ends = torch.tensor([a + n for a, n in zip(at, sizes)], device="cuda")
    tops = torch.tensor([(n + BLOCK - 1) // BLOCK * BLOCK for n in sizes], device="cuda")
    here &= inside < ends.repeat_interleave(tops, output_size=total)
    del inside
    flat = lambda std: normal(total, std=std).mul_(here)  # noqa: E731
    s = {"case": case, "at": torch.tensor(at, device="cuda"), "tops": tops, "total": total, "g": flat(1e-3).to(_TYPE[case["grads"]]),
         "out": torch.zeros(2, device="cuda"), "seed": seed & 0xffff}
    s["max_norm"] = 1e-3 * math.sqrt(sum(sizes)) / 2  # half of what the gradients have
    if case["op"] == "adamw":
        # matrices decay, vectors do not
        decay = [0.1 if n > 16384 else 0.0 for n in sizes]
        s["decay"] = torch.tensor(decay, dtype=torch.float64, device="cuda")
        s["p"] = flat(2e-2)
        s["w"] = s["p"].to(torch.bfloat16)
        m, v = flat(3e-4), flat(1e-3).square_()
        if case["bits"] == 32:
            s.update(m=m, v=v)
        else:
            half = torch.full((1, 1), 0x80008000, dtype=torch.int64, device="cuda")
            (s["m"], s["m_exp"]), (s["v"], s["v_exp"]) = _encode_m(m, half), _encode_v(v, half)
            s["m_value"], s["v_value"] = torch.zeros_like(s["w"]), torch.zeros_like(s["w"])
    if own:
        from paper_2408_16978_amd import tokenwise as TW
        part = lambda name, by=1: [s[name][a // by:a // by + -(-n // by)] for a, n in zip(at, sizes)] if name in s else None  # noqa: E731
        s["params"] = TW.FpdtTwParams(g=part("g"), p=part("p"), m=part("m"), v=part("v"), w=part("w"), m_exp=part("m_exp", BLOCK), v_exp=part("v_exp", BLOCK),
                                      m_value=part("m_value"), v_value=part("v_value"), weight_decay=decay if case["op"] == "adamw" else 0.0)
        s["workspace"] = torch.empty(TW.fpdt_tw_grad_norm_workspace_bytes(s["params"]), dtype=torch.uint8, device="cuda")
    return s


# ------------------------------------------------------------------------------------ plain forms
def _turned(x, cos, sin, rot, layout):
    x = x.float()
    if layout == "half":
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        y = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    else:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    return torch.cat([y, x[..., rot:]], -1)


def _plain_rope(s):
    c = s["case"]
    rows, Hq, Hkv, D, rot, layout = c["rows"], c["Hq"], c["Hkv"], c["D"], c["rot"], c["layout"]
    pos = s["positions"] if s["positions"] is not None else torch.arange(c["start"], c["start"] + rows, device="cuda")
    angle = pos.double()[:, None] * s["freqs"]
    cos, sin = (angle.cos() * s["amplitude"]).float()[:, None], (angle.sin() * s["amplitude"]).float()[:, None]
    dt = s["qkv"].dtype
    if c["direction"] == "bwd":
        q, k = (_turned(t, cos, -sin, rot, layout).to(dt).flatten(1) for t in (s["q"], s["k"]))
        return torch.cat([q, k, s["v"].flatten(1)], 1)
    q, k, v = s["qkv"].view(rows, Hq + 2 * Hkv, D).split([Hq, Hkv, Hkv], 1)
    return _turned(q, cos, sin, rot, layout).to(dt), _turned(k, cos, sin, rot, layout).to(dt), v.contiguous()


def _plain_norm(s):
    c = s["case"]
    layer = c["kind"] == "layer"
    w = s["w"].float()
    if c["direction"] == "fwd":
        total = s["x"] if s["r"] is None else (s["x"].float() + s["r"].float()).to(s["x"].dtype)
        f = total.float()
        mean = f.mean(1, keepdim=True) if layer else None
        d = f - mean if layer else f
        rstd = ((d * d).mean(1, keepdim=True) + EPS_NORM).rsqrt()
        y = d * rstd * w
        if layer:
            y = y + s["b"].float()
        stats = torch.cat([mean, rstd] if layer else [rstd], 1).t().contiguous()
        return {"sum": None if s["r"] is None else total, "y": y.to(total.dtype), "stats": stats}
    rstd = s["stats"][-1][:, None]
    unit = s["x"].float()
    if layer:
        unit = unit - s["stats"][0][:, None]
    unit = unit * rstd
    dy = s["dy"].float()
    h = dy * w
    dx = h - unit * (h * unit).mean(1, keepdim=True)
    if layer:
        dx = dx - h.mean(1, keepdim=True)
    dx = dx * rstd
    if s["dr"] is not None:
        dx = dx + s["dr"].float()
    s["dw"] += (dy * unit).sum(0)
    if layer:
        s["db"] += dy.sum(0)
    return {"dx": dx.to(s["x"].dtype), "dw": s["dw"], "db": s["db"]}


def _plain_grad_norm(s):
    norm = s["g"].float().square().view(-1, BLOCK).sum(1).double().sum().sqrt()
    s["out"].copy_(torch.stack([norm, (s["max_norm"] / (norm + 1e-6)).clamp(max=1.0)]))
    return s["out"]


_LOW = 0xffffffff


def _mix(x):
    """32 bits out of 32 bits, held in 64."""
    x = x ^ (x >> 15)
    x = (x * 0xB7E15163) & _LOW
    x = x ^ (x >> 13)
    x = (x * 0x93C467E3) & _LOW
    return x ^ (x >> 16)


def _spread(s, each):
    """What each tensor has, for each of its blocks: [blocks, 1]."""
    return each.repeat_interleave(s["tops"] // BLOCK, output_size=s["total"] // BLOCK)[:, None]


def _random(s):
    """The 32 random bits of every element of this step: [blocks, BLOCK]."""
    key = _mix(torch.tensor(s["seed"] ^ 0x243F6A88, device="cuda"))
    key = _mix(key ^ (STEP * 0x9E3779B1 & _LOW))
    key = _mix(key ^ (torch.arange(len(s["tops"]), device="cuda") * 0x85A308D3 & _LOW))
    at = torch.arange(s["total"], device="cuda").view(-1, BLOCK) - _spread(s, s["at"])
    return _mix((at * 0x9E3779B1 & _LOW) ^ _spread(s, key))


def _bits(x):
    return x.view(torch.int32).to(torch.int64)


def _exponent(size):
    """The exponent of each block of sizes: that of its largest rounded up to three fraction bits."""
    top = (_bits(size.amax(1, keepdim=True)) + 0xfffff) >> 23
    return torch.where(top >= 255, 255, top.clamp(min=40))


def _encode(size, low16, exp, steps):
    """Codes of sizes: three fraction bits, 2^steps exponents up to the block's, rounded up with the probability
    of what is cut off; code 0 is zero.  Sizes below code 1 get `low`."""
    base = exp - (2 ** steps - 1) << 3
    least = ((base + 1) << 20).to(torch.int32).view(torch.float32)
    low = low16.float() * 2.0 ** -16 * least < size if steps == 4 else size > 0  # a step divides by v: never down to zero
    code = torch.where(size >= least, ((_bits(size) + (low16 << 4)) >> 20) - base, low.to(torch.int64))
    return torch.where(exp == 255, 0, code)


def _encode_m(x, random32):
    size = x.view(-1, BLOCK).abs()
    exp = _exponent(size)
    code = _encode(size, random32 & 0xffff, exp, 4) | torch.where((x.view(-1, BLOCK) < 0) & (exp < 255), 128, 0)
    return code.to(torch.uint8).flatten(), exp.to(torch.uint8).flatten()


def _encode_v(x, random32):
    size = x.view(-1, BLOCK)
    exp = _exponent(size)
    return _encode(size, random32 >> 16, exp, 5).to(torch.uint8).flatten(), exp.to(torch.uint8).flatten()


def _decode(code, exp, steps):
    code, exp = code.view(-1, BLOCK).to(torch.int32), exp.to(torch.int32)[:, None]
    mag = code & 127 if steps == 4 else code
    x = torch.where(mag == 0, 0, (exp - (2 ** steps - 1) << 23) + (mag << 20)).view(torch.float32)
    x = torch.where(exp == 255, math.nan, x)
    return (torch.where(code > 127, -x, x) if steps == 4 else x).flatten()


def _plain_adamw(s):
    c = s["case"]
    g = s["g"].float()
    if c["clip"]:
        g = g * _plain_grad_norm(s)[1]
    if c["bits"] == 32:
        m, v = s["m"], s["v"]
    else:
        m, v = _decode(s["m"], s["m_exp"], 4), _decode(s["v"], s["v_exp"], 5)
    m.mul_(BETA1).add_(g * (1 - BETA1))
    v.mul_(BETA2).add_(g * g * (1 - BETA2))
    s["p"].view(-1, BLOCK).mul_(_spread(s, (1 - LR * s["decay"]).float()))
    s["p"].sub_(m * (LR / (1 - BETA1 ** STEP)) / (v.sqrt() * (1 - BETA2 ** STEP) ** -0.5 + EPS))
    s["w"].copy_(s["p"])
    if c["bits"] == 8:
        random32 = _random(s)
        (s["m"], s["m_exp"]), (s["v"], s["v_exp"]) = _encode_m(m, random32), _encode_v(v, random32)
        s["m_value"].copy_(_decode(s["m"], s["m_exp"], 4))  # four significant bits: bfloat16 holds them
        s["v_value"].copy_(_decode(s["v"], s["v_exp"], 5))
    return _adamw_outputs(s)


def _adamw_outputs(s):
    states = {"m": s["m"], "v": s["v"]} if s["case"]["bits"] == 32 else {"m": s["m_value"], "v": s["v_value"]}
    return dict(states, p=s["p"], w=s["w"], norm=s["out"])


# ------------------------------------------------------------------------------------ a pass
def _own(s):
    from paper_2408_16978_amd import tokenwise as TW
    c = s["case"]
    if c["op"] == "rope":
        rows, Hq, Hkv, D = c["rows"], c["Hq"], c["Hkv"], c["D"]
        q, k, v = s["qkv"].view(rows, Hq + 2 * Hkv, D).split([Hq, Hkv, Hkv], 1)
        more = dict(positions=s["positions"], position0=c["start"], amplitude=s["amplitude"],
                    layout=TW.FPDT_TW_ROPE_HALF if c["layout"] == "half" else TW.FPDT_TW_ROPE_INTERLEAVED)
        if c["direction"] == "fwd":
            TW.fpdt_tw_rope_fwd(q, k, v, s["q"], s["k"], s["v"], s["freqs"], **more)
            return s["q"], s["k"], s["v"]
        TW.fpdt_tw_rope_bwd(s["q"], s["k"], s["v"], q, k, v, s["freqs"], **more)
        return s["qkv"]
    if c["op"] == "norm":
        kind = TW.FPDT_TW_LAYERNORM if c["kind"] == "layer" else TW.FPDT_TW_RMSNORM
        if c["direction"] == "fwd":
            TW.fpdt_tw_norm_fwd(s["x"], s["r"], s["w"], s["b"], s["sum"], s["y"], s["stats"], EPS_NORM, kind)
            return {"sum": s["sum"], "y": s["y"], "stats": s["stats"]}
        TW.fpdt_tw_norm_bwd(s["x"], s["w"], s["stats"], s["dy"], s["dr"], s["dx"], s["dw"], s["db"], kind, s["workspace"])
        return {"dx": s["dx"], "dw": s["dw"], "db": s["db"]}
    if c["op"] == "grad_norm":
        TW.fpdt_tw_grad_norm(s["params"], s["max_norm"], s["out"], s["workspace"])
        return s["out"]
    if c["clip"]:
        TW.fpdt_tw_grad_norm(s["params"], s["max_norm"], s["out"], s["workspace"])
    TW.fpdt_tw_adamw_step(s["params"], LR, BETA1, BETA2, EPS, STEP, grad_scale=s["out"][1:] if c["clip"] else None, seed=s["seed"])
    if c["bits"] == 8:
        TW.fpdt_tw_adamw_unpack(s["params"])
    return _adamw_outputs(s)


def run(state):
    if own:
        return _own(state)
    return {"rope": _plain_rope, "norm": _plain_norm, "grad_norm": _plain_grad_norm, "adamw": _plain_adamw}[state["case"]["op"]](state)


def work(case):
    if case["op"] == "rope":
        n = case["rows"] * (case["Hq"] + 2 * case["Hkv"]) * case["D"]
        return {"bytes": 2 * n * (4 if case["dtype"] == "f32" else 2) + case["rows"] * 8 * case["given"] + case["rot"] * 4,
                "flops": 3 * case["rows"] * (case["Hq"] + case["Hkv"]) * case["rot"]}
    if case["op"] == "norm":
        n, e = case["rows"] * case["hidden"], 4 if case["dtype"] == "f32" else 2
        res, layer = case["residual"], case["kind"] == "layer"
        if case["direction"] == "fwd":
            return {"bytes": n * e * (4 if res else 2) + case["hidden"] * e * (1 + layer) + 4 * case["rows"] * (1 + layer), "flops": n * 6}
        return {"bytes": n * e * (4 if res else 3) + case["hidden"] * (e + 8 * (1 + layer)) + 4 * case["rows"] * (1 + layer), "flops": n * 10}
    n, grad = sum(_sizes(case)), 2 if case["grads"] == "bf16" else 4
    if case["op"] == "grad_norm":
        return {"bytes": n * grad, "flops": 2 * n}
    # p, m, v in and out, w out, the gradient once; in 8 bits what the states stand for goes out too
    each = grad + 8 + 2 + (16 if case["bits"] == 32 else 4 + 4) + (grad if case["clip"] else 0)
    return {"bytes": n * each, "flops": 16 * n}


# ------------------------------------------------------------------------------------ in 64 bits
def _exact_rope(s):
    c = s["case"]
    rows, Hq, Hkv, D, rot = c["rows"], c["Hq"], c["Hkv"], c["D"], c["rot"]
    pos = torch.arange(rows, device="cuda") + c["start"] if s["positions"] is None else s["positions"]
    back = c["direction"] == "bwd"
    angle = torch.outer(pos.double(), s["freqs"]) * (-1 if back else 1)
    unit = torch.polar(torch.full_like(angle, s["amplitude"]), angle)[:, None]
    if not back:
        every = s["qkv"].view(rows, Hq + 2 * Hkv, D).double()
    else:
        every = torch.cat([s["q"], s["k"], s["v"]], 1).double()
    head = every[:, :Hq + Hkv, :rot]
    if c["layout"] == "half":
        z = torch.complex(*head.unflatten(-1, (2, rot // 2)).unbind(-2)) * unit
        every[:, :Hq + Hkv, :rot] = torch.cat([z.real, z.imag], -1)
    else:
        z = torch.view_as_complex(head.unflatten(-1, (rot // 2, 2)).contiguous()) * unit
        every[:, :Hq + Hkv, :rot] = torch.view_as_real(z).flatten(-2)
    return every.flatten(1) if back else (every[:, :Hq], every[:, Hq:Hq + Hkv], every[:, Hq + Hkv:])


def _exact_norm(s):
    c = s["case"]
    layer = c["kind"] == "layer"
    x, w = s["x"].double(), s["w"].double()
    if c["direction"] == "fwd":
        total = None
        if s["r"] is not None:
            total = x + s["r"].double()
            x = total.to(s["x"].dtype).double()  # the statistics are those of the stored sum
        var, mean = torch.var_mean(x, 1, correction=0)
        rstd = (var + EPS_NORM) ** -0.5 if layer else (var + mean * mean + EPS_NORM) ** -0.5
        y = (x - mean[:, None] if layer else x) * torch.outer(rstd, w)
        if layer:
            y += s["b"].double()
        return {"sum": total, "y": y, "stats": torch.stack([mean, rstd] if layer else [rstd])}
    rstd, dy = s["stats"][-1].double(), s["dy"].double()
    unit = (x - s["stats"][0].double()[:, None] if layer else x) * rstd[:, None]
    n, h = c["hidden"], dy * w
    along = (h * unit).sum(1) / n
    dx = rstd[:, None] * (h - along[:, None] * unit - ((h.sum(1) / n)[:, None] if layer else 0.0))
    if s["dr"] is not None:
        dx += s["dr"].double()
    return {"dx": dx, "dw": s["dw"].double() + (dy * unit).sum(0), "db": s["db"].double() + dy.sum(0) if layer else None}


def _exact_norm_of(s):
    norm = math.sqrt(float(torch.sum(s["g"].double() ** 2)))
    return torch.tensor([norm, min(1.0, s["max_norm"] / (norm + 1e-6))], dtype=torch.float64, device="cuda")


def _exact_values(code, exp, steps):
    """What 8-bit codes stand for: (8 + fraction) / 8 times two to the exponent."""
    code, exp = code.double(), exp.double().repeat_interleave(BLOCK)
    sign = torch.where(code > 127, -1.0, 1.0) if steps == 4 else torch.ones_like(code)
    mag = torch.where(code > 127, code - 128, code) if steps == 4 else code
    value = (1 + (mag % 8) / 8) * torch.exp2(exp - 127 - (2 ** steps - 1) + torch.floor(mag / 8))
    return sign * torch.where(mag > 0, value, 0.0)


def _exact_rounded(x, chance, steps):
    """x rounded to a code of its block with `chance` in [0, 1) deciding, as a value."""
    size = x.abs()
    top = size.view(-1, BLOCK).amax(1)
    e = torch.floor(torch.log2(top.clamp(min=1e-300)))
    e = torch.where(top > 1.875 * torch.exp2(e), e + 1, e).clamp(min=40 - 127).repeat_interleave(BLOCK)
    least = 1.125 * torch.exp2(e - (2 ** steps - 1))
    grid = torch.exp2(torch.floor(torch.log2(size.clamp(min=1e-300))) - 3)
    value = torch.floor(size / grid + chance) * grid
    low = torch.where(size > 0, least, 0.0) if steps == 5 else torch.where(chance * least < size, least, 0.0)
    return torch.where(size >= least, value, low) * torch.sign(x)


def _exact_chances(s):
    """The random bits of every element as two numbers in [0, 1), tensor by tensor."""
    def mix(x):
        x = x ^ x.bitwise_right_shift(15)
        x = torch.remainder(x * 0xB7E15163, 1 << 32)
        x = x ^ x.bitwise_right_shift(13)
        x = torch.remainder(x * 0x93C467E3, 1 << 32)
        return x ^ x.bitwise_right_shift(16)

    start = mix(mix(torch.tensor(s["seed"] ^ 0x243F6A88)) ^ (STEP * 0x9E3779B1 % (1 << 32)))
    every = []
    for k, n in enumerate(s["tops"].tolist()):
        key = int(mix(start ^ (k * 0x85A308D3 % (1 << 32))))
        every.append(mix(torch.remainder(torch.arange(n, device="cuda") * 0x9E3779B1, 1 << 32) ^ key))
    every = torch.cat(every)
    return (every % 65536).double() / 65536, (every // 65536).double() / 65536


def _exact_adamw(s):
    c = s["case"]
    norm = _exact_norm_of(s) if c["clip"] else s["out"].double()
    g = s["g"].double() * (float(norm[1]) if c["clip"] else 1.0)
    wide = c["bits"] == 32
    m = s["m"].double() if wide else _exact_values(s["m"], s["m_exp"], 4)
    v = s["v"].double() if wide else _exact_values(s["v"], s["v_exp"], 5)
    m = BETA1 * m + (1 - BETA1) * g
    v = BETA2 * v + (1 - BETA2) * g ** 2
    decay = torch.cat([d.expand(n) for d, n in zip(s["decay"], s["tops"].tolist())])
    p = s["p"].double()
    p = p - LR * (m / (1 - BETA1 ** STEP) / (torch.sqrt(v / (1 - BETA2 ** STEP)) + EPS) + decay * p)
    if not wide:
        for_m, for_v = _exact_chances(s)
        m, v = _exact_rounded(m, for_m, 4), _exact_rounded(v, for_v, 5)
    return {"m": m, "v": v, "p": p, "w": p, "norm": norm}


def exact(case, seed):
    global own
    was, own = own, False
    s = prepare(case, seed)
    own = was
    return {"rope": _exact_rope, "norm": _exact_norm, "grad_norm": _exact_norm_of, "adamw": _exact_adamw}[case["op"]](s)
