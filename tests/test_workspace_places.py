"""Workspaces that the binding refuses: elsewhere than the tensors, or not one piece of memory (the library sees an address and a number of
bytes only)."""
import pytest
import torch

from paper_2408_16978_amd import tokenwise as TW


class _Reached(Exception):
    """The library was called."""


@pytest.fixture
def calls(monkeypatch):
    """{name: call(workspace)}: the two calls that take one, with tensors of the CPU that pass for device 0 and a library that only says that it was reached."""
    class Library:
        def __getattr__(self, name):
            def reached(*args):
                raise _Reached(name)
            return reached
    monkeypatch.setattr(TW, "load", lambda: Library())
    monkeypatch.setattr(TW, "_current", lambda t: 0)
    monkeypatch.setattr(TW, "_expect", lambda name, t, *rest: t.data_ptr())
    monkeypatch.setattr(TW, "_stats", lambda stats, *rest: stats.data_ptr())
    monkeypatch.setattr(TW, "_raw_stream", lambda stream, device: 0)
    monkeypatch.setattr(TW.FpdtTwParams, "_args", lambda self: (self.address, self.count))
    x, w, st, dw = torch.zeros(4, 8), torch.zeros(8), torch.zeros(4), torch.zeros(8)
    params = TW.FpdtTwParams(g=[torch.zeros(300)])
    params.device = torch.device("cuda", 0)
    return {"norm_bwd": lambda ws: TW.fpdt_tw_norm_bwd(x, w, st, x, None, x, dw, None, workspace=ws),
            "grad_norm": lambda ws: TW.fpdt_tw_grad_norm(params, 1.0, torch.zeros(2), ws)}


class _On0(torch.Tensor):
    """A tensor of the CPU that says that it is on device 0."""

    def get_device(self):
        return 0


@pytest.mark.parametrize("name", ["norm_bwd", "grad_norm"])
def test_refused(calls, name):
    with pytest.raises(TypeError, match="workspace must be on device 0"):
        calls[name](torch.zeros(1 << 16, dtype=torch.uint8))
    whole = torch.zeros(1 << 17, dtype=torch.uint8).as_subclass(_On0)
    for ws in (whole[::2], whole.view(256, 512)[:, :256], whole.view(256, 512).t()):
        with pytest.raises(ValueError, match="workspace must be contiguous"):
            calls[name](ws)
    for ws in (whole, whole[512:], None):  # (none: the library refuses it where it needs one)
        with pytest.raises(_Reached):
            calls[name](ws)


@pytest.mark.gpu
def test_gpu_refused_and_nothing_written():
    x, w, st = torch.randn(40, 64, device="cuda"), torch.ones(64, device="cuda"), torch.ones(40, device="cuda")
    dx, dw, out = torch.full_like(x, 3.0), torch.full_like(w, 5.0), torch.full((2,), 7.0, device="cuda")
    params = TW.FpdtTwParams(g=[torch.ones(300, device="cuda")])
    whole = torch.full((1 << 17,), 9, dtype=torch.uint8, device="cuda")
    for ws, error in ((torch.zeros(1 << 17, dtype=torch.uint8), TypeError), (whole[::2], ValueError), (whole[:1024], TW.FpdtTwError)):
        with pytest.raises(error):
            TW.fpdt_tw_norm_bwd(x, w, st, x, None, dx, dw, None, workspace=ws)
        with pytest.raises(error):
            TW.fpdt_tw_grad_norm(params, 1.0, out, ws)
    torch.cuda.synchronize()
    assert (dx == 3).all() and (dw == 5).all() and (out == 7).all() and (whole == 9).all()
    # fp32 words serve as well as bytes
    TW.fpdt_tw_norm_bwd(x, w, st, x, None, dx, dw, None, workspace=torch.empty(40 * 64, device="cuda"))
    TW.fpdt_tw_grad_norm(params, 1.0, out, torch.empty(1024, dtype=torch.float64, device="cuda"))
    torch.cuda.synchronize()
    assert abs(out[0].item() - 300 ** 0.5) < 1e-5
