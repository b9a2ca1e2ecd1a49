"""Sizes of 2^32 and a little more, of which the library would see the little: refused in the binding, as the library refuses what it sees to be too large."""
import pytest
import torch

from paper_2408_16978_amd import tokenwise as TW

FAR = 2 ** 32


@pytest.fixture
def seen(monkeypatch):
    """What reaches the library.  Tensors are without memory (their addresses are 0), and pass for device 0."""
    calls = []

    class Library:
        def __getattr__(self, name):
            return lambda *args: calls.append((name, args)) or 0
    monkeypatch.setattr(TW, "load", lambda: Library())
    monkeypatch.setattr(TW, "_current", lambda t: t.get_device())
    monkeypatch.setattr(TW, "_raw_stream", lambda stream, device: 0)
    return calls


def _meta(*shape, dtype=torch.bfloat16):
    return torch.empty(*shape, dtype=dtype, device="meta")


def test_refused(seen):
    x, w = _meta(1, FAR + 64), _meta(FAR + 64)
    for call in (lambda: TW.fpdt_tw_norm_fwd(x, None, w, None, None, x, None, 1e-5),
                 lambda: TW.fpdt_tw_norm_bwd(x, w, _meta(1, dtype=torch.float32), x, None, x, None, None)):
        with pytest.raises(TW.FpdtTwError) as e:
            call()
        assert e.value.status == 2
    f = _meta(4, dtype=torch.float64)
    heads, few, wide, long = _meta(1, FAR + 2, 8), _meta(1, 2, 8), _meta(1, 1, FAR + 8), _meta(FAR // 2 + 4, dtype=torch.float64)
    for q, k, freqs in ((heads, None, f), (few, heads, f), (wide, None, f), (few, None, long)):
        for call in (TW.fpdt_tw_rope_fwd, TW.fpdt_tw_rope_bwd):
            with pytest.raises(TW.FpdtTwError) as e:
                call(q, k, None, q, k, None, freqs)
            assert e.value.status == 2
    assert not seen


def test_queries():
    assert TW.fpdt_tw_norm_bwd_workspace_bytes(8, FAR + 64) == 0
    with pytest.raises(TW.FpdtTwError) as e:
        TW.fpdt_tw_rope_freqs(FAR + 8, 100.0)
    assert e.value.status == 1


def test_what_is_not_too_large_reaches_the_library(seen):
    x, w, f = _meta(3, 64), _meta(64), _meta(4, dtype=torch.float64)
    TW.fpdt_tw_norm_fwd(x, None, w, None, None, x, None, 1e-5)
    TW.fpdt_tw_rope_fwd(_meta(3, 2, 8), None, None, _meta(3, 2, 8), None, None, f)
    assert [n for n, _ in seen] == ["fpdt_tw_norm_fwd", "fpdt_tw_rope_fwd"]
