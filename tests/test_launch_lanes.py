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
