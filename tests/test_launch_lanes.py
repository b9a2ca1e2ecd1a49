"""Sizes for which one workgroup a piece of the work would be 2^32 lanes and more: of such a launch the runtime runs the remainder, without an error."""
import pytest
import torch

from paper_2408_16978_amd import binding as B
from paper_2408_16978_amd import inputs, runner
from paper_2408_16978_amd import tokenwise as TW


def _room(gib):
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < gib << 30:
        pytest.skip("needs %d GB" % gib)


@pytest.mark.gpu
def test_gpu_merge():
    """2^28 rows of heads and a few, of 8 elements: bit for bit what pieces of the rows give."""
    _room(40)
    rows, Hq, D, piece = (1 << 25) + 37, 8, 8, 1 << 22
    g = torch.Generator(device="cuda").manual_seed(1)
    Oa, Ob = (torch.randn(rows, Hq, D, device="cuda", generator=g, dtype=torch.bfloat16) for _ in range(2))
    La, Lb = (torch.randn(Hq, rows, device="cuda", generator=g) for _ in range(2))
    La[:, ::3] = float("-inf")
    O, L = torch.full_like(Oa, 9.0), torch.full_like(La, 9.0)
    print("[case] merge", rows, Hq, D, flush=True)
    B.fpdt_attn_merge(Oa, La, Ob, Lb, O, L)
    torch.cuda.synchronize()
    for r in range(0, rows, piece):
        at = slice(r, min(r + piece, rows))
        la, lb = La[:, at].contiguous(), Lb[:, at].contiguous()
        o, l = torch.empty_like(Oa[at]), torch.empty_like(la)
        B.fpdt_attn_merge(Oa[at], la, Ob[at], lb, o, l)
        assert torch.equal(O[at], o) and torch.equal(L[:, at], l), r


@pytest.mark.gpu
def test_gpu_backward_pair_by_pair():
    """65600 query heads of 4096 tokens, 2^28 rows of heads and a few: 64 heads, each of them 1025 times in its group, so that every repetition's dQ has the bits of the first, and that the value
    that the 64 heads alone give (the tolerance of the bf16 gradients)."""
    _room(215)
    S, few, times, D = 4096, 64, 1025, 64
    scale = D ** -0.5
    small = runner.make_buffers(*inputs.make_qkvdo(S, few, few, D, "bf16", 52, device="cuda"), 256, scale, B.FPDT_PAIRWISE)
    runner.forward(small)
    runner.backward(small)
    torch.cuda.synchronize()
    wide = lambda t: t.repeat_interleave(times, 1)
    Q, dO, O = wide(small.Q), wide(small.dO), wide(small.O)
    LSE = small.LSE.repeat_interleave(times, 0)
    dQ, dK, dV = torch.full_like(Q, float("nan")), torch.empty_like(small.K), torch.empty_like(small.V)
    ws = B.alloc_workspace(S, 256, few * times, few, D, B.FPDT_DTYPE_BF16, B.FPDT_PAIRWISE, True)
    ws.fill_(255)
    print("[case] backward pair by pair", S, few * times, D, flush=True)
    B.fpdt_attn_bwd(Q, small.K, small.V, O, LSE, dO, dQ, dK, dV, 256, scale, B.FPDT_PAIRWISE, ws)
    torch.cuda.synchronize()
    got = dQ.view(S, few, times, D)
    for r in range(0, S, 256):
        assert torch.equal(got[r:r + 256], got[r:r + 256, :, :1].expand(-1, -1, times, -1)), r
    want = small.dQ.double()
    rms = want.pow(2).mean().sqrt()
    assert float((got[:, :, 0].double() - want).abs().max() / rms) <= 2e-2 * max(1.0, float(want.abs().max() / rms))


@pytest.mark.gpu
@pytest.mark.parametrize("grads", [False, True])
def test_gpu_loss_of_the_longest_chunk(grads):
    """2^24 rows in one chunk, of eight logits, which repeat: every repetition has the bits of the first, and that those of a call of its own."""
    _room(20)
    rows, hidden, vocab, period = 1 << 24, 8, 8, 1 << 14
    g = torch.Generator(device="cuda").manual_seed(2)
    few = torch.randn(period, hidden, device="cuda", generator=g).to(torch.bfloat16)
    W = torch.randn(vocab, hidden, device="cuda", generator=g).to(torch.bfloat16)
    some = torch.randint(0, vocab, (period,), device="cuda", generator=g, dtype=torch.int32)

    def run(H, target):
        n = len(H)
        ws = torch.empty(TW.fpdt_tw_loss_workspace_bytes(n, hidden, vocab, 1), dtype=torch.uint8, device="cuda")
        ws.fill_(255)
        loss, lse = (torch.full((n,), float("nan"), device="cuda") for _ in range(2))
        dH = torch.full_like(H, float("nan")) if grads else None
        TW.fpdt_tw_loss_fwd_bwd(H, W, target, 2.0 ** -14, loss, lse, dH, None, 1, ws)
        torch.cuda.synchronize()
        return loss, lse, dH

    print("[case] loss of 2^24 rows", grads, flush=True)
    for got, want in zip(run(few.repeat(rows // period, 1), some.repeat(rows // period)), run(few, some)):
        assert want is None or (bool(torch.isfinite(want).all()) and torch.equal(got.view(-1, *want.shape), want.expand(rows // period, *want.shape)))
