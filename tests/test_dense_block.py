"""A dense feed-forward block as it is trained, made of the library's calls: product with bias and activation (or gate), product with bias, dropout with the residual, and the way
back through the library's own products.  Against autograd in 64 bits, captured, and beside calls on another stream."""
import pytest
import torch

from oracle import tokenwise as otw
from paper_2408_16978_amd import tokenwise as TW

GELU, SILU, TIMES = TW.FPDT_TW_ACT_GELU, TW.FPDT_TW_ACT_SILU, TW.FPDT_TW_JOIN_TIMES


class Dense:
    """y = x + dropout(h W2^T + b2),  h = gelu(x W1^T + b1)  or  silu(x W1^T + b1) * (x W3^T)."""

    def __init__(self, rows, n, f, gate, seed=3):
        g = torch.Generator(device="cuda").manual_seed(seed)
        bf = lambda *s, std=1.0: (torch.randn(*s, device="cuda", generator=g) * std).to(torch.bfloat16)
        e = lambda *s, dt=torch.bfloat16: torch.zeros(*s, dtype=dt, device="cuda")
        self.rows, self.gate = rows, gate
        self.W1, self.W2, self.W3 = bf(f, n, std=n ** -0.5), bf(n, f, std=f ** -0.5), bf(f, n, std=n ** -0.5) if gate else None
        self.b1, self.b2, self.x, self.dy, self.step = bf(f, std=0.3), bf(n, std=0.3), bf(rows, n), bf(rows, n), e(1, dt=torch.int64)
        self.u, self.z, self.h, self.sum, self.y = e(rows, f) if gate else None, e(rows, f), e(rows, f), e(rows, n), e(rows, n)
        self.dsum, self.dh, self.dz, self.du, self.dx1, self.dx3, self.dx = e(rows, n), e(rows, f), e(rows, f), e(rows, f) if gate else None, e(rows, n), e(rows, n), e(rows, n)
        self.dW1, self.dW2 = (torch.zeros_like(w, dtype=torch.float32) for w in (self.W1, self.W2))
        self.dW3 = torch.zeros_like(self.W3, dtype=torch.float32) if gate else None
        self.db1, self.db2 = e(f, dt=torch.float32), e(n, dt=torch.float32)
        room = lambda n_in, n_out: e(TW.fpdt_tw_affine_workspace_bytes(rows, n_in, n_out), dt=torch.uint8)
        back = lambda n_out: e(TW.fpdt_tw_affine_bwd_workspace_bytes(rows, n_out), dt=torch.uint8)
        self.ws1, self.ws2, self.wb1, self.wb2 = room(n, f), room(f, n), back(f), back(n)
        self.OUT = ("y", "dx", "dW1", "dW2", "db1", "db2") + (("dW3",) if gate else ())

    def forward(self, stream=None):
        more = dict(stream=stream)
        act, join = (SILU, TIMES) if self.gate else (GELU, TW.FPDT_TW_JOIN_ADD)
        if self.gate:
            TW.fpdt_tw_affine_fwd(self.x, self.W3, None, None, None, self.u, workspace=self.ws1, **more)
        TW.fpdt_tw_affine_fwd(self.x, self.W1, self.b1, self.u, self.z, self.h, act, join, self.ws1, **more)
        TW.fpdt_tw_affine_fwd(self.h, self.W2, self.b2, None, None, self.sum, workspace=self.ws2, **more)
        TW.fpdt_tw_dropout_fwd(self.sum, self.x, self.y, 0.1, 21, step_dev=self.step, **more)

    def backward(self):
        act, join = (SILU, TIMES) if self.gate else (GELU, TW.FPDT_TW_JOIN_ADD)
        TW.fpdt_tw_dropout_bwd(self.dy, self.dsum, 0.1, 21, step_dev=self.step)
        TW.fpdt_tw_affine_bwd(None, None, self.dsum, None, None, self.db2, workspace=self.wb2)
        TW.fpdt_tw_linear_bwd(self.h, self.W2, self.dsum, self.dh, self.dW2, 1)
        TW.fpdt_tw_affine_bwd(self.z, self.u, self.dh, self.dz, self.du, self.db1, act, join, workspace=self.wb1)
        TW.fpdt_tw_linear_bwd(self.x, self.W1, self.dz, self.dx1, self.dW1, 1)
        if self.gate:
            TW.fpdt_tw_linear_bwd(self.x, self.W3, self.du, self.dx3, self.dW3, 1)
            TW.fpdt_tw_dropout_fwd(self.dx1, self.dx3, self.dx1, 0.0, 0)  # (a sum: nothing is dropped)
        TW.fpdt_tw_dropout_fwd(self.dx1, self.dy, self.dx, 0.0, 0)

    def run(self):
        self.forward()
        self.backward()

    def clear(self):
        for k in self.OUT[2:]:
            getattr(self, k).zero_()

    def reference(self):
        leaves = {k: getattr(self, k).double().requires_grad_() for k in ("x", "W1", "W2", "b1", "b2") + (("W3",) if self.gate else ())}
        x, W1, W2, b1, b2 = (leaves[k] for k in ("x", "W1", "W2", "b1", "b2"))
        z = x @ W1.t() + b1
        h = torch.nn.functional.silu(z) * (x @ leaves["W3"].t()) if self.gate else torch.nn.functional.gelu(z)
        kept, scale = otw.dropout_kept(x.numel(), 0, 0.1, 21, int(self.step))
        y = x + (h @ W2.t() + b2) * torch.tensor(kept.reshape(x.shape) * scale, device="cuda")
        y.backward(self.dy.double())
        return dict({"d" + k: t.grad for k, t in leaves.items()}, y=y.detach())


@pytest.mark.gpu
@pytest.mark.parametrize("rows,n,f", [(300, 256, 512), (1, 64, 64), (77, 136, 72), (65, 100, 301), (2000, 512, 1024)])
@pytest.mark.parametrize("gate", [False, True])
def test_gpu_block_against_autograd(rows, n, f, gate):
    """Eight tensors on the way at most are rounded to bf16 (2^-8 at most, 2^-9.8 of the values in the root mean square): 2^-8.3 of an output's norm for those that
    reach it and for its own; twice that is allowed."""
    b = Dense(rows, n, f, gate)
    b.step.fill_(4)
    print("[case] dense block", rows, n, f, gate, flush=True)
    b.run()
    torch.cuda.synchronize()
    for k, want in b.reference().items():
        got = getattr(b, k).double()
        assert float((got - want).norm()) <= 2 * 2.0 ** -8.3 * float(want.norm()) + 1e-30, k


@pytest.mark.gpu
@pytest.mark.parametrize("rows,n,f", [(200, 128, 192), (65, 100, 301)])
@pytest.mark.parametrize("gate", [False, True])
def test_gpu_block_captured(rows, n, f, gate):
    """Captured once; replayed with other inputs and steps of dropout, with eager work between: the bits of the eager call."""
    a, b = Dense(rows, n, f, gate), Dense(rows, n, f, gate)
    a.run()  # (the library's products take their scratch in a call before)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.run()
    for k in range(4):
        for t in (a, b):
            g = torch.Generator(device="cuda").manual_seed(k)
            t.x.normal_(generator=g)
            t.dy.normal_(generator=g)
            t.step.fill_(k)
            t.clear()
        graph.replay()
        b.run()
        torch.cuda.synchronize()
        for name in a.OUT:
            assert torch.equal(getattr(a, name), getattr(b, name)), (k, name)


@pytest.mark.gpu
@pytest.mark.parametrize("gate", [False, True])
def test_gpu_forwards_on_two_streams(gate):
    """Forwards overlap (their workspaces are the caller's), another's way back on the current stream among them: the bits of each alone.  (fpdt_tw_linear_bwd of two streams would share the
    library's scratch.)"""
    made = [[Dense(400, 264, 1000, gate, s) for s in (1, 2, 3)] for _ in range(2)]
    for b in made[0] + made[1]:
        b.forward()
    made[0][2].backward()
    made[0][2].clear()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for b, s in zip(made[0], streams):
        b.y.fill_(float("nan"))
        b.z.zero_()
    torch.cuda.synchronize()
    for b, s in zip(made[0], streams):
        b.forward(s)
    made[0][2].backward()
    torch.cuda.synchronize()
    made[1][2].backward()
    torch.cuda.synchronize()
    for k, (a, b) in enumerate(zip(*made)):
        for name in a.OUT if k == 2 else ("y", "z", "h"):
            assert torch.equal(getattr(a, name), getattr(b, name)), (k, name)
