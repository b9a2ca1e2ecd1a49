"""The token-wise benchmark at widths that some of the operations it times do not take: it times the others."""
import json
import sys

import pytest

from paper_2408_16978_amd import bench_tokenwise as bench


@pytest.mark.parametrize("nm,nq,D,heads", [
    (4096, 6144, 128, (32, 8)), (2560, 7680, 80, (32, 32)), (2560, 7680, 128, (20, 20)), (64, 256, 128, None), (256, 256, 128, None), (4096, 6145, 128, None),
    (4096, 6272, 128, None), (270, 450, 45, None), (4096, 6144, 0, None), (8194 * 2, 8194 * 4, 8194, None), (8194, 12292, 2, None)])
def test_heads_of_a_product(nm, nq, D, heads):
    assert bench.split_of(nm, nq, D) == heads


@pytest.mark.gpu
@pytest.mark.parametrize("nm,nq,left_out", [(256, 768, ()), (64, 256, ("rope_split_fwd", "rope_gather_bwd")), (16512, 16768, ("rms_norm_fwd", "rms_norm_bwd"))])
def test_gpu_runs_to_its_end(monkeypatch, capsys, nm, nq, left_out):
    """Too few columns for a head of 128, and more than a normalised row may have."""
    monkeypatch.setattr(sys, "argv", ["bench"] + ("--rows 64 --n-model %d --n-ffn 256 --n-qkv %d --vocab 512 --chunks 1,2 --iters 1" % (nm, nq)).split())
    bench.main()
    lines = [json.loads(l) for l in capsys.readouterr().out.splitlines()]
    assert len(lines) == 2 * 5 + 7 - len(left_out) and all(l["ms"] > 0 for l in lines)
    assert {"rms_norm_fwd", "rms_norm_bwd", "rope_split_fwd", "rope_gather_bwd"} - {l["op"] for l in lines} == set(left_out)
