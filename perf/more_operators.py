"""The feed-forward part of a layer as it is trained, dense or with experts, as timed cases.

A case is a dict of plain values.  `listed()` names the representative ones, `draw(rng)` gives
further ones over the ranges they stand for, `prepare(case, seed)` makes what a program holds
before the call, `run(state)` is one pass (the library's entry points where `own` is set,
elementary torch operations otherwise), `work(case)` the bytes and operations a pass cannot do
without, `exact(case, seed)` the pass in 64 bits from the definition.

Operators:
  affine   product with bias, activation and residual (or gate) behind it; the gradient of what is
           behind it, with the bias's sums, of one or of many experts' rows
  dropout  with the residual add, from a counter-based generator: no mask is stored
  route    tokens sorted by expert and copied to their places, weighted sums on the way back, and
           the gradients of both
  experts  the affine product of every expert's rows with its own weights; the products of its backward
"""
import math

import torch

own = False

STEP = 1000


# ------------------------------------------------------------------------------------ cases
def _affine(direction, rows, n_in, n_out, act, join, bias, experts=0):
    return {"op": "affine", "direction": direction, "rows": rows, "n_in": n_in, "n_out": n_out, "act": act, "join": join, "bias": bias, "experts": experts}


def _dropout(direction, rows, hidden, p, residual, dtype="bf16", start=0):
    return {"op": "dropout", "direction": direction, "rows": rows, "hidden": hidden, "p": p, "residual": residual, "dtype": dtype, "start": start}


def _route(direction, rows, top, experts, hidden, residual=False, dtype="bf16", lost=0.0):
    return {"op": "route", "direction": direction, "rows": rows, "top": top, "experts": experts, "hidden": hidden, "residual": residual, "dtype": dtype,
            "lost": lost}


def _experts(direction, rows, experts, n_in, n_out, act="none", join="none", bias=False, lost=0.0):
    return {"op": "experts", "direction": direction, "rows": rows, "experts": experts, "n_in": n_in, "n_out": n_out, "act": act, "join": join, "bias": bias,
            "lost": lost}


def listed():
    cases = {
        # 16 sequences decode a token each: the attention's output projection and the residual add, all about reading the weight
        "affine_decode": _affine("fwd", 16, 4096, 4096, "none", "add", False),
        # GPT-2.7B's first feed-forward product in training: bias, GELU, the pre-activation kept for the backward
        "affine_gelu_16k": _affine("fwd", 16384, 2560, 10240, "gelu", "none", True),
        # Llama-8B's gated half of the block over a ragged number of tokens
        "affine_gate_ragged": _affine("fwd", 16001, 4096, 14336, "silu", "times", False),
        # the way back through GELU and bias
        "affine_bwd_gelu": _affine("bwd", 16384, 2560, 10240, "gelu", "none", True),
        # dropout of a short sequence's hidden states: latency counts
        "dropout_small": _dropout("fwd", 64, 2560, 0.1, True),
        # a chunk of 64K tokens, second half of a long sequence: element numbers beyond 2^32
        "dropout_64k": _dropout("fwd", 65536, 2560, 0.1, True, start=1966080 * 2560),
        # a decode step's tokens to two of eight experts each
        "dispatch_decode": _route("dispatch", 16, 2, 8, 4096),
        # a 32K-token chunk to two of eight experts each
        "dispatch_32k": _route("dispatch", 32768, 2, 8, 4096),
        # the gradient of the weighted sums: many small experts, a ragged number of tokens, some of them padding without an expert
        "combine_bwd_ragged": _route("combine_bwd", 10007, 8, 64, 2560, lost=0.05),
        # the decode step's rows through the experts' gated product: all about reading the weights
        "experts_decode": _experts("fwd", 32, 8, 4096, 14336, "silu", "times"),
        # 8192 tokens in two of eight experts
        "experts_fwd_16k": _experts("fwd", 16384, 8, 4096, 14336, "silu", "times"),
        # the products of the backward: 64 small experts, one idle, some rows without an expert
        "experts_bwd_64": _experts("bwd", 30000, 64, 2048, 1536, lost=0.05),
    }
    return [dict(c, name=n) for n, c in cases.items()]


def _log(rng, lo, hi):
    return lo * (hi / lo) ** rng.random()


def draw(rng):
    op = rng.choice(["affine", "affine", "affine", "dropout", "route", "route", "experts", "experts"])
    act, join = rng.choice(["none", "gelu", "silu"]), rng.choice(["none", "add", "times"])
    width = lambda: rng.choice([1024, 2048, 2560, 4096, 5120, 8192, 10240, 14336, 8 * rng.randint(16, 1600)])  # noqa: E731
    if op == "affine":
        n_in, n_out = width(), width()
        if rng.random() < 0.2:
            n_in, n_out = n_in + rng.randint(0, 7), n_out + rng.randint(0, 7)
        if rng.random() < 0.6:
            return _affine("fwd", int(_log(rng, 1, min(32768, 9e11 // (n_in * n_out)))), n_in, n_out, act, join, rng.random() < 0.5)
        experts = rng.choice([0, 0, 8, 60])
        return _affine("bwd", int(_log(rng, 1, min(32768, 1.6e8 // n_out))), n_in, n_out, act, join, act == join == "none" or rng.random() < 0.5, experts)
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if op == "dropout":
        hidden = rng.choice([1024, 2560, 4096, 5120, rng.randint(64, 9000)])
        most = min(131072, 160_000_000 // hidden // (2 if dtype == "f32" else 1))
        return _dropout(rng.choice(["fwd", "bwd"]), int(_log(rng, 1, most)), hidden, rng.choice([0.1, 0.1, 0.5, rng.random()]), rng.random() < 0.6, dtype,
                        rng.randint(0, 1 << 33))
    if op == "route":
        experts = rng.choice([4, 8, 16, 64, 128, 256, rng.randint(2, 300)])
        top = min(experts, rng.choice([1, 2, 2, 4, 6, 8]))
        hidden = rng.choice([1024, 2048, 2560, 4096, 4096, 5120, 7168, rng.randint(64, 9000)])
        most = min(65536, 260_000_000 // hidden // top // (2 if dtype == "f32" else 1))
        return _route(rng.choice(["dispatch", "gather_bwd", "combine", "combine_bwd"]), int(_log(rng, 1, most)), top, experts, hidden, rng.random() < 0.5, dtype,
                      rng.choice([0.0, 0.05, 0.3]))
    n_in, n_out = rng.choice([1024, 1536, 2048, 2560, 4096, 8 * rng.randint(16, 600)]), rng.choice([768, 1024, 1536, 2048, 4096, 8 * rng.randint(16, 600)])
    most, direction = min(32768, 4e11 // (n_in * n_out)), rng.choice(["fwd", "fwd", "bwd"])
    experts = rng.choice([n for n in (4, 8, 8, 16, 32, 64) if n * n_in * n_out < (2e8 if direction == "bwd" else 4.7e8)])
    return _experts(direction, int(_log(rng, 1, most)), experts, n_in, n_out, act, join, rng.random() < 0.5, rng.choice([0.0, 0.05, 0.3]))


# ------------------------------------------------------------------------------------ inputs
_TYPE = {"f32": torch.float32, "bf16": torch.bfloat16}


def _chosen(case, gen, rows, top):
    """[rows, top] experts, different ones of a token, some of them chosen more often; the last expert idle where there are 16 and
    more; a share of the tokens without any (-1)."""
    E = case["experts"]
    liking = torch.randn(E, device="cuda", generator=gen) * 0.4
    if E >= 16:
        liking[-1] = -1e9
    noise = torch.rand(rows, E, device="cuda", generator=gen).clamp_(1e-6, 1 - 1e-6)
    expert = (liking - (-noise.log()).log()).topk(min(top, E), 1).indices.to(torch.int32)
    return torch.where(torch.rand(rows, 1, device="cuda", generator=gen) < case.get("lost", 0.0), -1, expert).contiguous()


def _offsets(expert, experts):
    """Where the rows of each expert begin, and all of them end: [experts + 1]."""
    counts = (expert.flatten()[:, None] == torch.arange(experts, device="cuda")).sum(0)
    return torch.cat([counts.new_zeros(1), counts.cumsum(0)]).to(torch.int32)


def _places(expert, experts):
    """The place of each assignment in the order of experts, then tokens; -1 without an expert."""
    flat = expert.flatten()
    there = (flat >= 0) & (flat < experts)
    order = torch.where(there, flat, experts).sort(stable=True).indices
    place = torch.empty_like(flat)
    place[order] = torch.arange(flat.numel(), dtype=torch.int32, device="cuda")
    return torch.where(there, place, -1).view_as(expert)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *s, std=1.0: torch.randn(*s, device="cuda", generator=gen) * std  # noqa: E731
    half = lambda *s, std=1.0: normal(*s, std=std).to(torch.bfloat16)  # noqa: E731
    rows = case["rows"]
    s = {"case": case}
    if case["op"] == "dropout":
        dt, hidden = _TYPE[case["dtype"]], case["hidden"]
        s.update(x=normal(rows, hidden).to(dt), r=normal(rows, hidden).to(dt) if case["residual"] else None, y=torch.empty(rows, hidden, dtype=dt, device="cuda"),
                 seed=(seed * 0x9E3779B97F4A7C15 + 12345) % (1 << 63))
        return s
    if case["op"] == "route":
        dt, hidden, top = _TYPE[case["dtype"]], case["hidden"], case["top"]
        wide, narrow = rows * top, rows
        s["expert"] = _chosen(case, gen, rows, top)
        if case["direction"] == "dispatch":
            s.update(x=normal(rows, hidden).to(dt), xs=torch.zeros(wide, hidden, dtype=dt, device="cuda"),
                     offsets=torch.zeros(case["experts"] + 1, dtype=torch.int32, device="cuda"), place=torch.zeros(rows, top, dtype=torch.int32, device="cuda"))
            if own:
                from paper_2408_16978_amd import tokenwise as TW
                s["workspace"] = torch.empty(TW.fpdt_tw_experts_sort_workspace_bytes(wide, case["experts"]), dtype=torch.uint8, device="cuda")
            return s
        s["place"] = _places(s["expert"], case["experts"])
        s.update(ys=normal(wide, hidden).to(dt), r=normal(rows, hidden).to(dt) if case["residual"] and case["direction"] != "combine_bwd" else None)
        if case["direction"] != "gather_bwd":
            s["weight"] = normal(rows, top).softmax(1)
        if case["direction"] == "combine_bwd":
            s.update(dy=normal(narrow, hidden, std=1e-2).to(dt), dys=torch.zeros(wide, hidden, dtype=dt, device="cuda"),
                     dweight=torch.zeros(rows, top, device="cuda"))
        else:
            s["y"] = torch.empty(narrow, hidden, dtype=dt, device="cuda")
        return s
    n_in, n_out, E = case["n_in"], case["n_out"], case["experts"]
    if E:
        s["offsets"] = _offsets(_chosen(case, gen, rows, 1), E)
        s["counts"] = s["offsets"].diff().tolist()
    each = (E,) if case["op"] == "experts" else ()
    if case["direction"] == "fwd":
        s.update(x=half(rows, n_in), w=torch.empty(*each, n_out, n_in, dtype=torch.bfloat16, device="cuda"),
                 b=half(*each, n_out, std=0.3) if case["bias"] else None, r=half(rows, n_out) if case["join"] != "none" else None,
                 y=torch.zeros(rows, n_out, dtype=torch.bfloat16, device="cuda"), z=torch.zeros(rows, n_out, dtype=torch.bfloat16, device="cuda") if case["act"] != "none" else None)
        s["w"].normal_(std=n_in ** -0.5, generator=gen)
    elif case["op"] == "experts":
        s.update(x=half(rows, n_in), w=torch.empty(E, n_out, n_in, dtype=torch.bfloat16, device="cuda"), dy=half(rows, n_out, std=1e-2),
                 dx=torch.zeros(rows, n_in, dtype=torch.bfloat16, device="cuda"), dw=torch.zeros(E, n_out, n_in, device="cuda"))
        s["w"].normal_(std=n_in ** -0.5, generator=gen)
    else:
        behind, gate = case["act"] != "none" or case["join"] == "times", case["join"] == "times"
        s.update(z=half(rows, n_out) if behind else None, r=half(rows, n_out) if gate else None, dy=half(rows, n_out, std=1e-2),
                 dz=torch.zeros(rows, n_out, dtype=torch.bfloat16, device="cuda") if behind else None,
                 dr=torch.zeros(rows, n_out, dtype=torch.bfloat16, device="cuda") if gate else None,
                 db=normal(max(E, 1), n_out, std=1e-2) if case["bias"] else None)
    if own:
        from paper_2408_16978_amd import tokenwise as TW
        if case["op"] == "affine":
            need = TW.fpdt_tw_affine_workspace_bytes(rows, n_in, n_out) if case["direction"] == "fwd" else TW.fpdt_tw_affine_bwd_workspace_bytes(rows, n_out, max(E, 1))
            s["workspace"] = torch.empty(need, dtype=torch.uint8, device="cuda")
    return s


# ------------------------------------------------------------------------------------ plain forms
def _act(z, act):
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if act == "silu":
        return z / (1 + torch.exp(-z))
    return z


def _slope(z, act):
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (2 * math.pi) ** -0.5
    if act == "silu":
        keep = 1 / (1 + torch.exp(-z))
        return keep * (1 + z * (1 - keep))
    return torch.ones_like(z)


def _behind(s, z):
    """(activation and what joins it, pre-activation) from the product with its bias."""
    c = s["case"]
    y = _act(z, c["act"])
    if c["join"] == "add":
        y = y + s["r"].float()
    if c["join"] == "times":
        y = y * s["r"].float()
    return y.to(torch.bfloat16), z.to(torch.bfloat16)


def _of_row(s):
    """(expert, row within it) of each row, and how many rows have one."""
    used = sum(s["counts"])
    expert = torch.searchsorted(s["offsets"][1:], torch.arange(used, dtype=torch.int32, device="cuda"), right=True)
    return expert, torch.arange(used, device="cuda") - s["offsets"][expert], used


def _padded(s, x, expert, at, used):
    """Rows of `x` by expert, as many of each as the largest has: [experts, most, columns], zeros behind."""
    p = torch.zeros(s["case"]["experts"], max(s["counts"]), x.shape[1], device="cuda")
    p[expert, at] = x[:used].float()
    return p


def _plain_affine(s):
    c = s["case"]
    if c["direction"] == "fwd":
        z = s["x"].float() @ s["w"].float().t()
        if c["bias"]:
            z = z + s["b"].float()
        y, z = _behind(s, z)
        return {"y": y, "z": z if s["z"] is not None else None}
    dy = s["dy"].float()
    used = c["rows"]
    if c["experts"]:
        expert, _, used = _of_row(s)
    dz = dy
    if s["z"] is not None:
        z = s["z"].float()
        dz = dy * _slope(z, c["act"])
        if c["join"] == "times":
            dz = dz * s["r"].float()
            s["dr"][:used] = (dy * _act(z, c["act"])).to(torch.bfloat16)[:used]
        s["dz"][:used] = dz.to(torch.bfloat16)[:used]
    if c["bias"]:
        if c["experts"]:
            s["db"].index_put_((expert,), dz[:used], accumulate=True)
        else:
            s["db"] += dz.sum(0)
    return {"dz": s["dz"], "dr": s["dr"], "db": s["db"]}


def _mul(a, b):
    """(high, low) 32 bits of the product of 32 bits and a constant of 32 bits."""
    p = a * b  # mod 2^64
    return (p >> 32) & 0xffffffff, p & 0xffffffff


def _kept(s, n):
    """Which of n elements from case["start"] on are kept: sixteen random bits each, Philox4x32-10 of the number of its block of
    eight and of the step, with the seed for a key."""
    start = s["case"]["start"]
    block = torch.arange(start // 8, (start + n + 7) // 8, device="cuda")
    x = [block & 0xffffffff, block >> 32, torch.full_like(block, STEP & 0xffffffff), torch.full_like(block, STEP >> 32)]
    k = [s["seed"] & 0xffffffff, s["seed"] >> 32]
    for _ in range(10):
        (h0, l0), (h1, l1) = _mul(x[0], 0xD2511F53), _mul(x[2], 0xCD9E8D57)
        x = [h1 ^ x[1] ^ k[0], l1, h0 ^ x[3] ^ k[1], l0]
        k = [(k[0] + 0x9E3779B9) & 0xffffffff, (k[1] + 0xBB67AE85) & 0xffffffff]
    bits = torch.stack([h for w in x for h in (w & 0xffff, w >> 16)], 1).flatten()
    return bits[start % 8:start % 8 + n] >= round(s["case"]["p"] * 65536)


def _plain_dropout(s):
    c = s["case"]
    x = s["x"].float().flatten()
    dropped = round(c["p"] * 65536)
    y = torch.where(_kept(s, x.numel()), x * (65536 / (65536 - dropped) if dropped < 65536 else 0.0), 0.0).view_as(s["x"])
    if s["r"] is not None and c["direction"] == "fwd":
        y = y + s["r"].float()
    return y.to(s["x"].dtype)


def _plain_route(s):
    c = s["case"]
    rows, top, hidden = c["rows"], c["top"], c["hidden"]
    if c["direction"] == "dispatch":
        place = _places(s["expert"], c["experts"])
        flat = place.flatten()
        there = flat >= 0
        s["xs"][flat[there]] = s["x"].repeat_interleave(top, 0)[there]
        return {"offsets": _offsets(s["expert"], c["experts"]), "place": place, "xs": s["xs"]}
    there = s["place"] >= 0
    if c["direction"] == "combine_bwd":
        dy, flat, here = s["dy"].float(), s["place"].flatten(), there.flatten()
        dot = (s["ys"][s["place"].clamp(min=0)].float() * dy[:, None]).sum(2)
        s["dys"][flat[here]] = (dy[:, None] * s["weight"][..., None]).to(s["dys"].dtype).view(-1, hidden)[here]
        return {"dys": s["dys"], "dweight": torch.where(there, dot, 0.0)}
    y = torch.where(there[..., None], s["ys"][s["place"].clamp(min=0)].float(), 0.0)
    if c["direction"] == "combine":
        y = y * s["weight"][..., None]
    y = y.sum(1)
    if s["r"] is not None:
        y = y + s["r"].float()
    return y.to(s["ys"].dtype)


def _plain_experts(s):
    c = s["case"]
    expert, at, used = _of_row(s)
    if used == 0:
        return {"dx": s["dx"], "dw": s["dw"]} if c["direction"] == "bwd" else {"y": s["y"], "z": s["z"]}
    x, w = _padded(s, s["x"], expert, at, used), s["w"].float()
    if c["direction"] == "bwd":
        dy = _padded(s, s["dy"], expert, at, used)
        s["dx"][:used] = torch.bmm(dy, w)[expert, at].to(torch.bfloat16)
        s["dw"] += torch.bmm(dy.transpose(1, 2), x)
        return {"dx": s["dx"], "dw": s["dw"]}
    z = torch.bmm(x, w.transpose(1, 2))[expert, at]
    if c["bias"]:
        z = z + s["b"].float()[expert]
    y, z = _behind({"case": c, "r": None if s["r"] is None else s["r"][:used]}, z)
    s["y"][:used] = y
    if s["z"] is not None:
        s["z"][:used] = z
    return {"y": s["y"], "z": s["z"]}


# ------------------------------------------------------------------------------------ a pass
def _own(s):
    from paper_2408_16978_amd import tokenwise as TW
    c = s["case"]
    if c["op"] == "dropout":
        more = dict(p=c["p"], seed=s["seed"], step=STEP, first=c["start"])
        if c["direction"] == "fwd":
            TW.fpdt_tw_dropout_fwd(s["x"], s["r"], s["y"], **more)
        else:
            TW.fpdt_tw_dropout_bwd(s["x"], s["y"], **more)
        return s["y"]
    if c["op"] == "route":
        if c["direction"] == "dispatch":
            TW.fpdt_tw_experts_sort(s["expert"], s["offsets"], s["place"], s["workspace"])
            TW.fpdt_tw_experts_gather_fwd(s["x"], s["place"], s["xs"])
            return {"offsets": s["offsets"], "place": s["place"], "xs": s["xs"]}
        if c["direction"] == "gather_bwd":
            TW.fpdt_tw_experts_gather_bwd(s["ys"], s["place"], s["r"], s["y"])
            return s["y"]
        if c["direction"] == "combine":
            TW.fpdt_tw_experts_combine_fwd(s["ys"], s["weight"], s["place"], s["r"], s["y"])
            return s["y"]
        TW.fpdt_tw_experts_combine_bwd(s["ys"], s["weight"], s["place"], s["dy"], s["dys"], s["dweight"])
        return {"dys": s["dys"], "dweight": s["dweight"]}
    act = {"none": TW.FPDT_TW_ACT_NONE, "gelu": TW.FPDT_TW_ACT_GELU, "silu": TW.FPDT_TW_ACT_SILU}[c["act"]]
    join = TW.FPDT_TW_JOIN_TIMES if c["join"] == "times" else TW.FPDT_TW_JOIN_ADD
    if c["op"] == "experts":
        if c["direction"] == "fwd":
            TW.fpdt_tw_experts_affine_fwd(s["x"], s["w"], s["b"], s["r"], s["z"], s["y"], s["offsets"], act, join)
            return {"y": s["y"], "z": s["z"]}
        TW.fpdt_tw_experts_linear_bwd(s["x"], s["w"], s["dy"], s["dx"], s["dw"], s["offsets"])
        return {"dx": s["dx"], "dw": s["dw"]}
    if c["direction"] == "fwd":
        TW.fpdt_tw_affine_fwd(s["x"], s["w"], s["b"], s["r"], s["z"], s["y"], act, join, s["workspace"])
        return {"y": s["y"], "z": s["z"]}
    if s["dz"] is not None or s["db"] is not None:  # (a residual alone: its gradient and the product's are dy itself, and no call is made)
        TW.fpdt_tw_affine_bwd(s["z"], s["r"], s["dy"], s["dz"], s["dr"], s["db"], act, join, s["offsets"] if c["experts"] else None, s["workspace"])
    return {"dz": s["dz"], "dr": s["dr"], "db": s["db"]}


def run(state):
    if own:
        return _own(state)
    return {"affine": _plain_affine, "dropout": _plain_dropout, "route": _plain_route, "experts": _plain_experts}[state["case"]["op"]](state)


def work(case):
    rows = case["rows"]
    if case["op"] == "dropout":
        n = rows * case["hidden"]
        fwd = case["direction"] == "fwd"
        return {"bytes": n * (4 if case["dtype"] == "f32" else 2) * (3 if fwd and case["residual"] else 2), "flops": 2 * n}
    kept = 1 - case.get("lost", 0.0)
    if case["op"] == "route":
        top, e = case["top"], 4 if case["dtype"] == "f32" else 2
        one, many = rows * case["hidden"] * e, int(kept * rows * top * case["hidden"]) * e
        index = rows * top * 4
        if case["direction"] == "dispatch":
            return {"bytes": one + many + 2 * index + 4 * case["experts"], "flops": 0}
        if case["direction"] == "combine_bwd":
            return {"bytes": one + 2 * many + 3 * index, "flops": 3 * many // e}
        return {"bytes": one * (1 + case["residual"]) + many + index * (2 if case["direction"] == "combine" else 1), "flops": 2 * many // e}
    n_in, n_out, E = case["n_in"], case["n_out"], case["experts"]
    gate, behind = case["join"] != "none", case["act"] != "none"
    rows = int(kept * rows)
    if case["op"] == "affine" and case["direction"] == "bwd":
        times = case["join"] == "times"
        n = rows * n_out * 2
        return {"bytes": n * (1 + 2 * (behind or times) + 2 * times) + 8 * n_out * max(E, 1) * case["bias"], "flops": 10 * rows * n_out}
    weights = n_in * n_out * min(max(E, 1), max(rows, 1))
    if case["direction"] == "bwd":
        return {"bytes": 4 * rows * n_in + 2 * rows * n_out + 10 * weights, "flops": 4 * rows * n_in * n_out}
    return {"bytes": 2 * rows * n_in + 2 * weights + 2 * rows * n_out * (1 + gate + behind), "flops": 2 * rows * n_in * n_out}


# ------------------------------------------------------------------------------------ in 64 bits
def _exact_act(z, act):
    """The activation and its derivative."""
    if act == "gelu":
        upper = torch.special.erfc(-z / math.sqrt(2)) / 2  # the normal distribution's share below z
        return z * upper, upper + z * torch.exp(-z.square() / 2) / math.sqrt(2 * math.pi)
    if act == "silu":
        share = torch.sigmoid(z)
        return z * share, share + z * share * torch.sigmoid(-z)
    return z, torch.ones_like(z)


def _exact_rows(c, x, w, b, r):
    z = torch.mm(x.double(), w.double().T)
    if b is not None:
        z += b.double()
    y = _exact_act(z, c["act"])[0]
    if c["join"] != "none":
        y = y + r.double() if c["join"] == "add" else y * r.double()
    return y, z


def _exact_affine(s):
    c = s["case"]
    if c["direction"] == "fwd":
        y, z = _exact_rows(c, s["x"], s["w"], s["b"], s["r"])
        return {"y": y, "z": z if s["z"] is not None else None}
    out = {"dz": None, "dr": None, "db": None}
    grad = s["dy"].double()
    limits = s["offsets"].tolist() if c["experts"] else [0, c["rows"]]
    if s["z"] is not None:
        y, slope = _exact_act(s["z"].double(), c["act"])
        if c["join"] == "times":
            out["dr"] = grad * y
            out["dr"][limits[-1]:] = 0
            grad = grad * s["r"].double()
        grad = grad * slope
        out["dz"] = grad.clone()
        out["dz"][limits[-1]:] = 0
    if c["bias"]:
        out["db"] = s["db"].double() + torch.stack([grad[a:b].sum(0) for a, b in zip(limits, limits[1:])])
    return out


def _exact_dropout(s):
    """Philox in halves of 16 bits, eight elements of a counter side by side."""
    c = s["case"]
    n, start = s["x"].numel(), c["start"]
    number = torch.arange(start, start + n, device="cuda")
    at = torch.div(number, 8, rounding_mode="floor")
    x0, x1 = torch.remainder(at, 1 << 32), torch.div(at, 1 << 32, rounding_mode="floor")
    x2, x3 = torch.full_like(at, STEP % (1 << 32)), torch.full_like(at, STEP // (1 << 32))
    k0, k1 = s["seed"] % (1 << 32), s["seed"] // (1 << 32)

    def product(x, m):
        low, high = torch.remainder(x, 65536) * m, torch.div(x, 65536, rounding_mode="floor") * m + torch.div(torch.remainder(x, 65536) * m, 65536, rounding_mode="floor")
        return torch.div(high, 65536, rounding_mode="floor"), torch.remainder(high, 65536) * 65536 + torch.remainder(low, 65536)

    for _ in range(10):
        a, b = product(x0, 0xD2511F53), product(x2, 0xCD9E8D57)
        x0, x1, x2, x3 = b[0].bitwise_xor(x1).bitwise_xor(k0), b[1], a[0].bitwise_xor(x3).bitwise_xor(k1), a[1]
        k0, k1 = (k0 + 0x9E3779B9) % (1 << 32), (k1 + 0xBB67AE85) % (1 << 32)
    lane = torch.remainder(number, 8)
    word = torch.where(lane < 2, x0, torch.where(lane < 4, x1, torch.where(lane < 6, x2, x3)))
    bits = torch.where(lane % 2 == 1, torch.div(word, 65536, rounding_mode="floor"), torch.remainder(word, 65536))
    drop = round(c["p"] * 65536)
    y = s["x"].double().flatten() * (bits >= drop) / max(1 - drop / 65536, 1e-300)
    y = y.view(s["x"].shape)
    return y + s["r"].double() if s["r"] is not None and c["direction"] == "fwd" else y


def _exact_sorted(c, expert):
    """Places and offsets by counting, expert after expert."""
    flat = expert.flatten()
    place, offsets = torch.full_like(flat, -1), [0]
    for e in range(c["experts"]):
        mine = (flat == e).nonzero().flatten()
        place[mine] = torch.arange(offsets[-1], offsets[-1] + mine.numel(), dtype=torch.int32, device="cuda")
        offsets.append(offsets[-1] + mine.numel())
    return place.view_as(expert), torch.tensor(offsets, dtype=torch.int32, device="cuda")


def _exact_route(s):
    c = s["case"]
    place, offsets = _exact_sorted(c, s["expert"])
    wide = c["rows"] * c["top"]
    source = torch.full((wide + 1,), -1, dtype=torch.int64, device="cuda")  # the assignment that sits at each place
    flat = place.flatten().long()
    source[torch.where(flat < 0, wide, flat)] = torch.arange(wide, device="cuda")
    source = source[:int(offsets[-1])]
    token = torch.div(source, c["top"], rounding_mode="floor")
    sent = token.numel()
    if c["direction"] == "dispatch":
        xs = torch.zeros(wide, c["hidden"], dtype=torch.float64, device="cuda")
        xs[:sent] = s["x"].double()[token]
        return {"offsets": offsets, "place": place, "xs": xs}
    if c["direction"] == "combine_bwd":
        dys, dweight = torch.zeros(wide, c["hidden"], dtype=torch.float64, device="cuda"), torch.zeros(wide, dtype=torch.float64, device="cuda")
        dys[:sent] = s["dy"].double()[token] * s["weight"].double().flatten()[source, None]
        dweight[source] = (s["dy"].double()[token] * s["ys"][:sent].double()).sum(1)
        return {"dys": dys, "dweight": dweight.view_as(s["weight"])}
    part = s["ys"][:sent].double()
    if c["direction"] == "combine":
        part = part * s["weight"].double().flatten()[source, None]
    y = torch.zeros(c["rows"], c["hidden"], dtype=torch.float64, device="cuda") if s["r"] is None else s["r"].double()
    return y.index_add_(0, token, part)


def _exact_experts(s):
    c, limits = s["case"], s["offsets"].tolist()
    spans = list(zip(range(c["experts"]), limits, limits[1:]))
    if c["direction"] == "bwd":
        dx, dw = torch.zeros(s["dx"].shape, dtype=torch.float64, device="cuda"), s["dw"].double()
        for e, a, b in spans:
            dx[a:b] = s["dy"][a:b].double() @ s["w"][e].double()
            dw[e] += s["dy"][a:b].double().T @ s["x"][a:b].double()
        return {"dx": dx, "dw": dw}
    y, z = (torch.zeros(s["y"].shape, dtype=torch.float64, device="cuda") for _ in range(2))
    for e, a, b in spans:
        y[a:b], z[a:b] = _exact_rows(c, s["x"][a:b], s["w"][e], None if s["b"] is None else s["b"][e], None if s["r"] is None else s["r"][a:b])
    return {"y": y, "z": z if s["z"] is not None else None}


def exact(case, seed):
    global own
    was, own = own, False
    s = prepare(case, seed)
    own = was
    return {"affine": _exact_affine, "dropout": _exact_dropout, "route": _exact_route, "experts": _exact_experts}[case["op"]](s)
