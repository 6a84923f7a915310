"""Cluster barriers of the adapters' kernel where warps and CTAs have little to do in front of them: token tiles without
tokens, CTAs without a share of K or of the channels, tiles whose copies differ from lane to lane.  The barriers are for whole
warps, so each stands behind a __syncwarp()."""
import os
import re

import pytest

from conftest import ROOT
from test_gpu_lora import _equal, _integers, _reference, gpu         # noqa: F401


def test_every_cluster_barrier_has_whole_warps():
    with open(os.path.join(ROOT, "paper_2508_06753_b200", "csrc", "w2a8_lora.cu")) as f:
        lines = f.read().splitlines()
    barrier = re.compile(r"barrier\.cluster|(?<!lora_)\bcluster_(sync|wait|arrive\w*)\(")
    found = [i for i, line in enumerate(lines) if barrier.search(line)]
    assert len(found) >= 3
    for i in found:
        assert lines[i - 1].strip() == "__syncwarp();", lines[i]


@pytest.mark.gpu
@pytest.mark.parametrize("rank_max", [16, 64, 128])
@pytest.mark.parametrize("tile", [16, 64])
@pytest.mark.parametrize("C", [2, 5, 8])
def test_warps_and_ctas_without_work(gpu, monkeypatch, C, tile, rank_max):           # noqa: F811
    torch, b = gpu
    monkeypatch.setenv("W2A8_LORA_TILE", str(tile))
    monkeypatch.setenv("W2A8_LORA_C", str(C))
    for M, Ns, K, L in [(1, (16,), 64, 1), (3, (48, 16), 64, 2), (18, (16, 16, 32, 16), 192, 5), (77, (80,), 128, 40)]:
        p = _integers(torch, M, Ns, K, L, rank_max, seed=M + C)
        lora = b.LoraGroup(p["A"], p["B"], rank=p["rank"], scale=p["scale"])
        want = _reference(torch, p["x"], p["adapter"], p["A"], p["B"], p["rank"], p["scale"], p["base"])
        for _ in range(5):
            _equal(torch, b.w2a8_lora_grouped(p["x"], p["adapter"], lora, base=p["base"]), want)
