"""The library's operators together, as a training step uses them: a Llama-like layer and its loss forward and backward, the
clipping of its gradients and two AdamW steps, against the same in 64 bits with autograd."""
import math

import numpy as np
import pytest
import torch

import test_optimizer
from oracle import tokenwise as otw
from paper_2408_16978_amd import runner
from paper_2408_16978_amd import tokenwise as TW

S, HIDDEN, HQ, HKV, D, FFN, VOCAB = 512, 256, 4, 2, 64, 640, 768
EPS, MAX_NORM, CHUNKS = 1e-5, 0.5, 2
HYPER = dict(lr=1e-2, beta1=0.9, beta2=0.95, eps=1e-8)
NAMES = ["n1", "qkv", "out", "n2", "w1", "w3", "w2", "n3", "head"]
SHAPES = {"n1": (HIDDEN,), "qkv": ((HQ + 2 * HKV) * D, HIDDEN), "out": (HIDDEN, HQ * D), "n2": (HIDDEN,), "w1": (FFN, HIDDEN), "w3": (FFN, HIDDEN),
          "w2": (HIDDEN, FFN), "n3": (HIDDEN,), "head": (VOCAB, HIDDEN)}


def _reference(w, x, target, freqs, pos):
    """loss of the layer in the precision of its arguments"""
    rms = lambda t, g: t * (t.square().mean(1, keepdim=True) + EPS).rsqrt() * g
    def turn(t):
        a, b = t[..., :D // 2], t[..., D // 2:]
        ang = (pos[:, None] * freqs)[:, None]
        return torch.cat([a * ang.cos() - b * ang.sin(), b * ang.cos() + a * ang.sin()], -1)
    q, k, v = (rms(x, w["n1"]) @ w["qkv"].T).view(S, HQ + 2 * HKV, D).split([HQ, HKV, HKV], 1)
    q, k = turn(q), turn(k).repeat_interleave(HQ // HKV, 1)
    s = torch.stack([q[:, h] @ k[:, h].T for h in range(HQ)]) / math.sqrt(D)
    s = s.masked_fill(torch.ones(S, S, dtype=torch.bool).triu(1), -math.inf).softmax(-1)
    o = torch.stack([s[h] @ v[:, h // (HQ // HKV)] for h in range(HQ)], 1).flatten(1)
    x = x + o @ w["out"].T
    h = rms(x, w["n2"])
    x = x + (torch.nn.functional.silu(h @ w["w1"].T) * (h @ w["w3"].T)) @ w["w2"].T
    return torch.nn.functional.cross_entropy(rms(x, w["n3"]) @ w["head"].T, target)


class Layer:
    def __init__(self, weights, bits):
        n = lambda *s, dt=torch.bfloat16: torch.empty(*s, dtype=dt, device="cuda")
        self.p = {k: t.float().cuda() for k, t in weights.items()}
        self.w = {k: t.to(torch.bfloat16) for k, t in self.p.items()}
        self.g = {k: torch.zeros_like(t) for k, t in self.p.items()}
        state = torch.uint8 if bits == 8 else torch.float32
        lists = {k: [torch.zeros(t.shape, dtype=state, device="cuda") for t in self.p.values()] for k in ("m", "v")}
        if bits == 8:
            lists.update({k: [torch.zeros(-(-t.numel() // 128), dtype=state, device="cuda") for t in self.p.values()] for k in ("m_exp", "v_exp")})
        self.params = TW.FpdtTwParams(g=list(self.g.values()), p=list(self.p.values()), w=list(self.w.values()),
                                      weight_decay=[0.1 if t.dim() == 2 else 0.0 for t in self.p.values()], **lists)
        self.x1, self.x2, self.h1, self.h2, self.h3, self.a, self.f, self.dh, self.dx = (n(S, HIDDEN) for _ in range(9))
        self.rstd = [n(S, dt=torch.float32) for _ in range(3)]
        self.qkv, self.dqkv = n(S, (HQ + 2 * HKV) * D), n(S, (HQ + 2 * HKV) * D)
        q, k, v, do = n(S, HQ, D), n(S, HKV, D), n(S, HKV, D), n(S, HQ, D)
        self.attn = runner.make_buffers(q, k, v, do, S // CHUNKS, D ** -0.5, 0)
        self.loss, self.lse = n(S, dt=torch.float32), n(S, dt=torch.float32)
        u8 = lambda k: n(max(k, 256), dt=torch.uint8)
        self.ws = u8(max(TW.fpdt_tw_ffn_workspace_bytes(S, HIDDEN, FFN, TW.FPDT_TW_SWIGLU, CHUNKS, True),
                         TW.fpdt_tw_loss_workspace_bytes(S, HIDDEN, VOCAB, CHUNKS), TW.fpdt_tw_norm_bwd_workspace_bytes(S, HIDDEN),
                         TW.fpdt_tw_grad_norm_workspace_bytes(self.params)))
        self.out = n(2, dt=torch.float32)

    def gradients(self, x, target, freqs, position0):
        w, g, b, ws = self.w, self.g, self.attn, self.ws
        heads = lambda t: t.view(S, HQ + 2 * HKV, D).split([HQ, HKV, HKV], 1)
        TW.fpdt_tw_norm_fwd(x, None, w["n1"], None, None, self.h1, self.rstd[0], EPS)
        TW.fpdt_tw_linear_fwd(self.h1, w["qkv"], self.qkv, CHUNKS)
        TW.fpdt_tw_rope_fwd(*heads(self.qkv), b.Q, b.K, b.V, freqs, position0=position0)
        runner.forward(b)
        TW.fpdt_tw_linear_fwd(b.O.view(S, HQ * D), w["out"], self.a, CHUNKS)
        TW.fpdt_tw_norm_fwd(self.a, x, w["n2"], None, self.x1, self.h2, self.rstd[1], EPS)
        TW.fpdt_tw_ffn_fwd(self.h2, w["w1"], w["w3"], w["w2"], self.f, TW.FPDT_TW_SWIGLU, CHUNKS, ws)
        TW.fpdt_tw_norm_fwd(self.f, self.x1, w["n3"], None, self.x2, self.h3, self.rstd[2], EPS)
        TW.fpdt_tw_loss_fwd_bwd(self.h3, w["head"], target, 1.0 / S, self.loss, self.lse, self.dh, g["head"], CHUNKS, ws)
        TW.fpdt_tw_norm_bwd(self.x2, w["n3"], self.rstd[2], self.dh, None, self.dx, g["n3"], None, workspace=ws)
        TW.fpdt_tw_ffn_bwd(self.h2, w["w1"], w["w3"], w["w2"], self.dx, self.dh, g["w1"], g["w3"], g["w2"], TW.FPDT_TW_SWIGLU, CHUNKS, ws)
        TW.fpdt_tw_norm_bwd(self.x1, w["n2"], self.rstd[1], self.dh, self.dx, self.dx, g["n2"], None, workspace=ws)
        TW.fpdt_tw_linear_bwd(b.O.view(S, HQ * D), w["out"], self.dx, b.dO.view(S, HQ * D), g["out"], CHUNKS)
        runner.backward(b)
        TW.fpdt_tw_rope_bwd(b.dQ, b.dK, b.dV, *heads(self.dqkv), freqs, position0=position0)
        TW.fpdt_tw_linear_bwd(self.h1, w["qkv"], self.dqkv, self.dh, g["qkv"], CHUNKS)
        TW.fpdt_tw_norm_bwd(x, w["n1"], self.rstd[0], self.dh, self.dx, self.dx, g["n1"], None, workspace=ws)

    def step(self, k):
        TW.fpdt_tw_grad_norm(self.params, MAX_NORM, self.out, self.ws)
        TW.fpdt_tw_adamw_step(self.params, step=k, grad_scale=self.out[1:], flags=TW.FPDT_TW_ADAMW_ZERO_GRAD, **HYPER)


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_gpu_layer_loss_gradients_clip_and_steps(bits):
    gen = torch.Generator().manual_seed(21)
    weights = {k: (1 + 0.1 * torch.randn(s, generator=gen)) if len(s) == 1 else torch.randn(s, generator=gen) * s[1] ** -0.5 for k, s in SHAPES.items()}
    weights = {k: t.to(torch.bfloat16) for k, t in weights.items()}
    x = torch.randn(S, HIDDEN, generator=gen).to(torch.bfloat16)
    target = torch.randint(0, VOCAB, (S,), generator=gen)
    freqs, position0 = TW.fpdt_tw_rope_freqs(D, 10000.0), 1900000
    pos = torch.arange(position0, position0 + S, dtype=torch.float64)
    layer, xd, td, fd = Layer(weights, bits), x.cuda(), target.int().cuda(), freqs.cuda()
    ref = {k: t.double().requires_grad_() for k, t in weights.items()}
    x64 = x.double().requires_grad_()
    opt = torch.optim.AdamW([{"params": [t for t in ref.values() if t.dim() == 2], "weight_decay": 0.1},
                             {"params": [t for t in ref.values() if t.dim() == 1], "weight_decay": 0.0}], lr=HYPER["lr"], betas=(0.9, 0.95), eps=1e-8)
    # About 25 roundings to bf16 lie between the tokens and a gradient (weights are the same), each at most 2^-9 of a tensor's
    # norm on average; all in one direction they come to 5% of it.
    limit = 0.05
    far = lambda a, b: float((a.double().cpu() - b.detach()).norm() / b.detach().norm())
    for k in (1, 2):
        loss = _reference(ref, x64, target, freqs, pos)
        x64.grad = None
        opt.zero_grad()
        loss.backward()
        layer.gradients(xd, td, fd, position0)
        torch.cuda.synchronize()
        assert abs(float(layer.loss.double().mean()) - float(loss.detach())) < 0.02 * float(loss.detach())
        for name in NAMES:
            assert far(layer.g[name], ref[name].grad) < limit, (k, name)
        assert far(layer.dx, x64.grad) < limit
        norm = torch.nn.utils.clip_grad_norm_(list(ref.values()), MAX_NORM)
        before = {n: t.clone() for n, t in layer.p.items()}
        was = {n: t.detach().clone() for n, t in ref.items()}
        layer.step(k)
        opt.step()
        torch.cuda.synchronize()
        assert abs(float(layer.out[0]) / float(norm) - 1) < limit and float(layer.out[1]) < 1
        for name in NAMES:
            assert torch.equal(layer.w[name], layer.p[name].to(torch.bfloat16)) and (layer.g[name] == 0).all()
            # a first step moves every weight by lr in the direction of its gradient's sign: where the two differ, the
            # gradient is smaller than its error, so compare where it is larger than that (5% of the root mean square, times 4).
            # The second's length depends on both gradients, each then off by a quarter at most, and in 8 bits on moments a code step
            # (1 / 8 of m, 1 / 16 of v's root) off: 0.25 + 0.19.
            gr = ref[name].grad
            sure = gr.abs() > 4 * limit * gr.square().mean().sqrt()
            moved, want = (layer.p[name] - before[name]).double().cpu()[sure], (ref[name].detach() - was[name])[sure]
            assert float((moved - want).norm() / want.norm()) < (0.05 if k == 1 else 0.5), (k, name)
            # from here on the reference has this layer's weights
            ref[name].data.copy_(layer.w[name].double().cpu())
            layer.p[name].copy_(layer.w[name].float())


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_gpu_each_step_is_that_of_its_own_gradients(bits):
    """Three steps of the layer, each held to the oracle's step from the gradients, weights, moments and factor that it found: to the optimizer tests' tolerances,
    which are roundings of fp32, where the comparison with another model's gradients (above) can only be as close as those are."""
    gen = torch.Generator().manual_seed(5)
    weights = {k: (1 + 0.1 * torch.randn(s, generator=gen)) if len(s) == 1 else torch.randn(s, generator=gen) * s[1] ** -0.5 for k, s in SHAPES.items()}
    layer = Layer({k: t.to(torch.bfloat16) for k, t in weights.items()}, bits)
    x = torch.randn(S, HIDDEN, generator=gen).to(torch.bfloat16).cuda()
    target, freqs = torch.randint(0, VOCAB, (S,), generator=gen).int().cuda(), TW.fpdt_tw_rope_freqs(D, 10000.0).cuda()
    # the same tensors as the optimizer tests hold them, with moments of their own
    model = test_optimizer.Model.__new__(test_optimizer.Model)
    model.bits, model.g, model.p, model.w = bits, *([t.view(-1) for t in d.values()] for d in (layer.g, layer.p, layer.w))
    model.sizes, model.decay = [t.numel() for t in model.p], [0.1 if t.dim() == 2 else 0.0 for t in layer.p.values()]
    zeros = lambda by, dt: [torch.zeros(-(-n // by), dtype=dt, device="cuda") for n in model.sizes]
    state, more = (torch.float32, {}) if bits == 32 else (torch.uint8, dict(m_exp=zeros(128, torch.uint8), v_exp=zeros(128, torch.uint8)))
    model.m, model.v, model.me, model.ve = zeros(1, state), zeros(1, state), more.get("m_exp"), more.get("v_exp")
    layer.params = TW.FpdtTwParams(g=model.g, p=model.p, w=model.w, m=model.m, v=model.v, weight_decay=model.decay, **more)
    assert HYPER == test_optimizer.HYPER
    for k in (1, 2, 3):
        layer.gradients(x, target, freqs, 0)
        before = model.state()
        assert all(np.abs(g).max() > 0 for g in before[1])
        layer.step(k)
        torch.cuda.synchronize()
        # (each rounded once, as in the norm's own tests)
        for got, want in zip(layer.out.tolist(), otw.grad_norm(before[1], MAX_NORM)):
            assert abs(got - want) <= 2.0 ** -24 * want * 1.01, k
        test_optimizer._check_long(model, before, k, layer.out[1].item(), 0)
        assert all((g == 0).all() for g in model.g)
