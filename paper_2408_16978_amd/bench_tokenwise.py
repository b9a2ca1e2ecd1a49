"""Throughput and workspace of the token-wise chunked operations (include/fpdt_tokenwise.h) as a
function of the chunk count, at Llama-8B layer shapes, and of the operations around them that are
not chunked (rotary positions with the QKV split, normalisation, gradient norm, AdamW) in bytes a
second; with --feed-forward also of products with something behind them, dropout, tokens to experts
and back and the experts' products.  Prints one JSON line per (operation, chunk count).  `python -m paper_2408_16978_amd.bench_tokenwise [--rows 65536] [--chunks 1,4,16,64]`.
"""
import argparse
import json

import torch

from . import tokenwise as TW


def _time(fn, iters):
    fn()
    torch.cuda.synchronize()
    a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    a.record()
    for _ in range(iters):
        fn()
    b.record()
    torch.cuda.synchronize()
    return a.elapsed_time(b) / iters


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--rows", type=int, default=65536, help="tokens on this GPU")
    ap.add_argument("--n-model", type=int, default=4096)
    ap.add_argument("--n-ffn", type=int, default=14336)
    ap.add_argument("--n-qkv", type=int, default=6144, help="(Hq + 2 Hkv) * D")
    ap.add_argument("--head-dim", type=int, default=128)
    ap.add_argument("--vocab", type=int, default=128256)
    ap.add_argument("--chunks", default="1,2,4,8,16,64")
    ap.add_argument("--iters", type=int, default=3)
    ap.add_argument("--feed-forward", action="store_true", help="time the parts of a feed-forward block, dense and with experts, too")
    ap.add_argument("--max-workspace-gib", type=float, default=64.0)
    a = ap.parse_args()
    if not torch.cuda.is_available():
        raise SystemExit("needs a GPU")
    TW.load()
    dev = "cuda"
    g = torch.Generator(device=dev).manual_seed(7)
    rows, nm, nf, nq, nv = a.rows, a.n_model, a.n_ffn, a.n_qkv, a.vocab
    bf = lambda *s, std=1.0: (torch.randn(*s, device=dev, generator=g) * std).to(torch.bfloat16)
    X, dY = bf(rows, nm), bf(rows, nm)
    W1, W3, W2 = bf(nf, nm, std=nm ** -0.5), bf(nf, nm, std=nm ** -0.5), bf(nm, nf, std=nf ** -0.5)
    Wq, Wv = bf(nq, nm, std=nm ** -0.5), bf(nv, nm, std=nm ** -0.5)
    tgt = torch.randint(0, nv, (rows,), device=dev, generator=g, dtype=torch.int32)
    Y, dX = torch.empty_like(X), torch.empty_like(X)
    Yq = torch.empty(rows, nq, dtype=torch.bfloat16, device=dev)
    dW1, dW3, dW2 = (torch.zeros_like(w, dtype=torch.float32) for w in (W1, W3, W2))
    dWq, dWv = torch.zeros_like(Wq, dtype=torch.float32), torch.zeros_like(Wv, dtype=torch.float32)
    loss, lse = torch.empty(rows, device=dev), torch.empty(rows, device=dev)
    cap = int(a.max_workspace_gib * 2 ** 30)
    for n in [int(c) for c in a.chunks.split(",")]:
        ops = []
        wf = TW.fpdt_tw_ffn_workspace_bytes(rows, nm, nf, TW.FPDT_TW_SWIGLU, n, False)
        wb = TW.fpdt_tw_ffn_workspace_bytes(rows, nm, nf, TW.FPDT_TW_SWIGLU, n, True)
        wl = TW.fpdt_tw_loss_workspace_bytes(rows, nm, nv, n)
        ops.append(("linear_fwd", 0, 2.0 * rows * nm * nq, lambda ws: TW.fpdt_tw_linear_fwd(X, Wq, Yq, n)))
        ops.append(("linear_bwd", 0, 4.0 * rows * nm * nq, lambda ws: TW.fpdt_tw_linear_bwd(X, Wq, Yq, dX, dWq, n)))
        ops.append(("ffn_swiglu_fwd", wf, 6.0 * rows * nm * nf,
                    lambda ws: TW.fpdt_tw_ffn_fwd(X, W1, W3, W2, Y, TW.FPDT_TW_SWIGLU, n, ws)))
        # backward = 2 recomputed GEMMs + dHh + dW2 + 2 dX + dW1 + dW3 = 8 GEMMs of 2 rows nm nf
        ops.append(("ffn_swiglu_bwd", wb, 16.0 * rows * nm * nf,
                    lambda ws: TW.fpdt_tw_ffn_bwd(X, W1, W3, W2, dY, dX, dW1, dW3, dW2, TW.FPDT_TW_SWIGLU, n, ws)))
        ops.append(("loss_fwd_bwd", wl, 6.0 * rows * nm * nv,
                    lambda ws: TW.fpdt_tw_loss_fwd_bwd(X, Wv, tgt, 1.0 / rows, loss, lse, dX, dWv, n, ws)))
        for name, wbytes, flops, fn in ops:
            rec = {"op": name, "rows": rows, "n_chunks": n, "workspace_gib": round(wbytes / 2 ** 30, 3)}
            if wbytes > cap:
                rec["skipped"] = "workspace above --max-workspace-gib"
            else:
                ws = torch.empty(max(wbytes, 256), dtype=torch.uint8, device=dev)
                ms = _time(lambda: fn(ws), a.iters)
                del ws
                rec.update(ms=round(ms, 3), tflops=round(flops / ms * 1e-9, 1))
            print(json.dumps(rec), flush=True)
    del dW1, dW3, dW2, dWq, dWv, W1, W3, W2, Wq, Wv, X, dY, Y, dX, Yq, loss, lse
    unchunked(rows, nm, nf, nq, a.head_dim, a.iters, bf)
    if a.feed_forward:
        feed_forward(rows, nm, nf, a.iters, bf)


def split_of(nm, nq, D):
    """Heads (Hq, Hkv) of a product of nq columns, or None where these are no whole heads of all three, or none that can be turned whole
    (an odd D) or at all (D beyond 8192, more than 4096 of them)."""
    Hq = nm // D if D > 0 else 0
    Hkv = (nq // D - Hq) // 2 if Hq else 0
    return (Hq, Hkv) if Hkv > 0 and (Hq + 2 * Hkv) * D == nq and D % 2 == 0 and D <= 8192 and max(Hq, Hkv) <= 4096 else None


def unchunked(rows, nm, nf, nq, D, iters, bf):
    """What a step does around the products: every array read or written once (bytes as in the headline of each line).  Widths that
    an operation does not take are left out."""
    dev, heads, ops = "cuda", split_of(nm, nq, D), []
    room = TW.fpdt_tw_norm_bwd_workspace_bytes(rows, nm)  # (0: too wide)
    if room:
        X, R, W, S, Y = bf(rows, nm), bf(rows, nm), bf(nm), bf(rows, nm), bf(rows, nm)
        rstd, dW = torch.empty(rows, device=dev), torch.zeros(nm, device=dev)
        ws = torch.empty(room, dtype=torch.uint8, device=dev)
        tensor = 2 * rows * nm
        ops += [("rms_norm_fwd", 4 * tensor, lambda: TW.fpdt_tw_norm_fwd(X, R, W, None, S, Y, rstd, 1e-5)),
                ("rms_norm_bwd", 4 * tensor, lambda: TW.fpdt_tw_norm_bwd(S, W, rstd, X, R, Y, dW, None, workspace=ws))]
    if heads:
        Hq, Hkv = heads
        qkv = bf(rows, nq)
        parts = qkv.view(rows, Hq + 2 * Hkv, D).split([Hq, Hkv, Hkv], 1)
        out = [torch.empty(rows, h, D, dtype=torch.bfloat16, device=dev) for h in (Hq, Hkv, Hkv)]
        freqs = TW.fpdt_tw_rope_freqs(D, 500000.0).to(dev)
        ops += [("rope_split_fwd", 4 * rows * nq, lambda: TW.fpdt_tw_rope_fwd(*parts, *out, freqs)),
                ("rope_gather_bwd", 4 * rows * nq, lambda: TW.fpdt_tw_rope_bwd(*out, *parts, freqs))]
    sizes = [nq * nm, nm * nm, nf * nm, nf * nm, nf * nm, nm, nm]  # a layer's weights
    n = sum(sizes)
    f = lambda dt=torch.float32, by=1: [torch.zeros(-(-k // by), dtype=dt, device=dev) for k in sizes]
    lists = {32: TW.FpdtTwParams(g=f(), p=f(), m=f(), v=f(), w=f(torch.bfloat16)),
             8: TW.FpdtTwParams(g=f(), p=f(), m=f(torch.uint8), v=f(torch.uint8), w=f(torch.bfloat16), m_exp=f(torch.uint8, TW.FPDT_TW_STATE_BLOCK),
                                v_exp=f(torch.uint8, TW.FPDT_TW_STATE_BLOCK))}
    norm, nws = torch.zeros(2, device=dev), torch.empty(TW.fpdt_tw_grad_norm_workspace_bytes(lists[32]), dtype=torch.uint8, device=dev)
    ops += [("grad_norm_layer", 4 * n, lambda: TW.fpdt_tw_grad_norm(lists[32], 1.0, norm, nws)),
            ("adamw_layer_32bit", 30 * n, lambda: TW.fpdt_tw_adamw_step(lists[32], 1e-4, 0.9, 0.95, 1e-8, 1)),
            ("adamw_layer_8bit", 18 * n, lambda: TW.fpdt_tw_adamw_step(lists[8], 1e-4, 0.9, 0.95, 1e-8, 1))]
    for name, nbytes, fn in ops:
        ms = _time(fn, max(iters, 10))
        print(json.dumps({"op": name, "rows": rows, "n_chunks": None, "ms": round(ms, 4), "tbytes_per_s": round(nbytes / ms * 1e-9, 2)}), flush=True)


def feed_forward(rows, nm, nf, iters, bf, E=8, top=2):
    """The feed-forward block's first product with bias and GELU, with a gate, and their gradient; dropout with the residual; `rows` tokens' assignments to `top` of E
    experts (rows / top tokens) and the experts' products, of weights half as wide.  Widths that experts do not take are left out."""
    dev, e32 = "cuda", lambda *s: torch.zeros(*s, device="cuda")
    X, W, B = bf(rows, nm), bf(nf, nm, std=nm ** -0.5), bf(nf)
    Y, Z, R = (torch.empty(rows, nf, dtype=torch.bfloat16, device=dev) for _ in range(3))
    R.normal_()
    dB, S = e32(nf), bf(rows, nm)
    out = torch.empty_like(X)
    ws = torch.empty(TW.fpdt_tw_affine_workspace_bytes(rows, nm, nf), dtype=torch.uint8, device=dev)
    wb = torch.empty(TW.fpdt_tw_affine_bwd_workspace_bytes(rows, nf), dtype=torch.uint8, device=dev)
    product, wide = 2.0 * rows * nm * nf, 2 * rows * nf
    gelu, silu, times = TW.FPDT_TW_ACT_GELU, TW.FPDT_TW_ACT_SILU, TW.FPDT_TW_JOIN_TIMES
    ops = [("affine_gelu_fwd", "tflops", product, lambda: TW.fpdt_tw_affine_fwd(X, W, B, None, Z, Y, gelu, workspace=ws)),
           ("affine_gate_fwd", "tflops", product, lambda: TW.fpdt_tw_affine_fwd(X, W, None, R, Z, Y, silu, times, ws)),
           ("affine_gelu_bwd", "tbytes_per_s", 3 * wide, lambda: TW.fpdt_tw_affine_bwd(Z, None, Y, Y, None, dB, gelu, workspace=wb)),
           ("dropout_residual_fwd", "tbytes_per_s", 6 * rows * nm, lambda: TW.fpdt_tw_dropout_fwd(X, S, out, 0.1, 1))]
    tokens, half = rows // top, nf // 2
    if tokens and nm % 8 == 0 and half % 8 == 0 and half:
        sent = tokens * top
        expert = torch.rand(tokens, E, device=dev).topk(top, 1).indices.to(torch.int32).contiguous()
        offsets, place, weight = (torch.zeros(E + 1, dtype=torch.int32, device=dev), torch.zeros_like(expert), torch.rand(tokens, top, device=dev))
        wsort = torch.empty(TW.fpdt_tw_experts_sort_workspace_bytes(sent, E), dtype=torch.uint8, device=dev)
        We, dWe, Xs, H, dys, dweight = bf(E, half, nm, std=nm ** -0.5), e32(E, half, nm), bf(sent, nm), bf(sent, half), bf(sent, nm), e32(tokens, top)
        one, many = 2 * tokens * nm, 2 * sent * nm

        def dispatch():
            TW.fpdt_tw_experts_sort(expert, offsets, place, wsort)
            TW.fpdt_tw_experts_gather_fwd(X[:tokens], place, Xs)

        ops += [("experts_sort_gather", "tbytes_per_s", one + many, dispatch),
                ("experts_combine_fwd", "tbytes_per_s", one + many, lambda: TW.fpdt_tw_experts_combine_fwd(Xs, weight, place, None, out[:tokens])),
                ("experts_combine_bwd", "tbytes_per_s", one + 2 * many, lambda: TW.fpdt_tw_experts_combine_bwd(Xs, weight, place, X[:tokens], dys, dweight)),
                ("experts_affine_fwd", "tflops", 2.0 * sent * nm * half, lambda: TW.fpdt_tw_experts_affine_fwd(Xs, We, None, None, None, H, offsets, silu)),
                ("experts_linear_bwd", "tflops", 4.0 * sent * nm * half, lambda: TW.fpdt_tw_experts_linear_bwd(Xs, We, H, dys, dWe, offsets))]
    for name, unit, amount, fn in ops:
        ms = _time(fn, iters)
        print(json.dumps({"op": name, "rows": rows, "n_chunks": None, "ms": round(ms, 4), unit: round(amount / ms * 1e-9, 2 if unit[1] == "b" else 1)}), flush=True)


if __name__ == "__main__":
    main()
