"""More rows than a launch has workgroups for: the kernels that walk them take a second turn, at offsets beyond 2^31 bytes or 2^32 bytes.  Every call is
compared with calls over pieces of its rows, each of one turn, bit for bit (the operations of a token or a row do not depend on the others); the pieces' own
values are those of the parity tests."""
import pytest
import torch

from paper_2408_16978_amd import tokenwise as TW

TILES = 1 << 20  # of the rotary kernels; twice as many of the normalisation's forward
BF16 = torch.bfloat16


def _room(gib):
    if torch.cuda.mem_get_info()[0] < gib << 30:
        pytest.skip("needs %d GB" % gib)


def _noise(rows, cols, dtype):
    """Rows that differ: 2^20 + 7 random ones over and over, each time a little larger."""
    period = (1 << 20) + 7
    some = torch.randn(min(rows, period), cols, device="cuda", generator=torch.Generator(device="cuda").manual_seed(cols))
    out = torch.empty(rows, cols, dtype=dtype, device="cuda")
    for k, r in enumerate(range(0, rows, period)):
        n = min(period, rows - r)
        out[r:r + n] = some[:n] * (1 + k / 8)
    return out


# Tokens of a workgroup at a time: `per`.  Heads of 258 channels are 129 pairs, a token for each workgroup, in either layout; heads of 8 channels with one pair go
# through the kernel whose sines are in LDS, 16 tokens a workgroup; heads of 512 with 16 turning over all lanes of a wave, 4 tokens a workgroup.
@pytest.mark.gpu
@pytest.mark.parametrize("per,D,rot,interleaved", [(1, 258, 258, False), (1, 258, 258, True), (16, 8, 2, False), (16, 8, 2, True), (4, 512, 16, False)])
def test_gpu_rotary_positions(per, D, rot, interleaved):
    print("[case] rope, many rows", per, D, rot, interleaved, flush=True)
    _room(32)
    rows, layout = TILES * per + 21, TW.FPDT_TW_ROPE_INTERLEAVED if interleaved else TW.FPDT_TW_ROPE_HALF
    x = _noise(rows, D, BF16).view(rows, 1, D)
    fd = TW.fpdt_tw_rope_freqs(rot, 10000.0).cuda()
    got, piece = torch.full_like(x, 7.0), torch.empty_like(x[:TILES * per // 2])
    for call, start in ((TW.fpdt_tw_rope_fwd, 5), (TW.fpdt_tw_rope_bwd, -9)):
        call(x, None, None, got, None, None, fd, position0=start, layout=layout)
        for r in range(0, rows, len(piece)):
            n = min(len(piece), rows - r)
            call(x[r:r + n], None, None, piece[:n], None, None, fd, position0=start + r, layout=layout)
            assert torch.equal(got[r:r + n], piece[:n]), r
    # given positions, in place
    pos = torch.randint(0, 1 << 21, (rows,), device="cuda")
    TW.fpdt_tw_rope_fwd(x, None, None, got, None, None, fd, positions=pos, layout=layout)
    last = rows - 1000
    TW.fpdt_tw_rope_fwd(x[last:], None, None, piece[:1000], None, None, fd, positions=pos[last:], layout=layout)
    assert torch.equal(got[last:], piece[:1000])
    TW.fpdt_tw_rope_fwd(x, None, None, x, None, None, fd, positions=pos, layout=layout)
    torch.cuda.synchronize()
    assert torch.equal(x, got)


# Rows of a workgroup: 16, 8 or 4 of 16, 32 or 64 lanes, or one of several waves.  (136 and 264 columns: more than 2^32 bytes a
# tensor.)
@pytest.mark.gpu
@pytest.mark.parametrize("per,hidden", [(16, 8), (16, 5), (8, 136), (4, 264), (1, 520)])
@pytest.mark.parametrize("layer", [False, True])
def test_gpu_normalisation_forward_and_backward(per, hidden, layer):
    print("[case] norm, many rows", per, hidden, layer, flush=True)
    _room(48)
    rows, kind = 2 * TILES * per + 9, TW.FPDT_TW_LAYERNORM if layer else TW.FPDT_TW_RMSNORM
    x, w = _noise(rows, hidden, BF16), torch.randn(hidden, device="cuda").to(BF16)
    r = x.flip(1).contiguous()
    b = torch.randn(hidden, device="cuda").to(BF16) if layer else None
    y, stats = torch.full_like(x, 7.0), torch.empty(2 if layer else 1, rows, device="cuda")
    TW.fpdt_tw_norm_fwd(x, r, w, b, r, y, stats, 1e-5, kind)  # (the sum in r's place)
    step = TILES * per
    piece, total, ps = torch.empty_like(x[:step]), torch.empty_like(x[:step]), torch.empty(len(stats), step, device="cuda")
    for i in range(0, rows, step):
        n = min(step, rows - i)
        of = torch.empty(len(stats), n, device="cuda") if n < step else ps
        TW.fpdt_tw_norm_fwd(x[i:i + n], x[i:i + n].flip(1).contiguous(), w, b, total[:n], piece[:n], of, 1e-5, kind)
        assert torch.equal(y[i:i + n], piece[:n]) and torch.equal(r[i:i + n], total[:n]) and torch.equal(stats[:, i:i + n], of), i
    # backward of the sums: y is the gradient that comes, x the other way's
    dx = torch.full_like(x, 7.0)
    TW.fpdt_tw_norm_bwd(r, w, stats, y, x, dx, None, None, kind)
    for i in range(0, rows, step):
        n = min(step, rows - i)
        TW.fpdt_tw_norm_bwd(r[i:i + n], w, stats[:, i:i + n].contiguous(), y[i:i + n], x[i:i + n], piece[:n], None, None, kind)
        assert torch.equal(dx[i:i + n], piece[:n]), i
