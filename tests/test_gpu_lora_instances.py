"""Every instance of the adapters' kernel (tiles of 16 and 64 tokens, ranks of up to 16, 32, 64 and 128, fp32 and bf16
results) on shapes that end inside its stages, exact on integers (see test_gpu_lora.py), with the tile size forced."""
import pytest

from test_gpu_lora import _equal, _integers, _reference, gpu       # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("rank_max", [8, 16, 24, 32, 40, 64, 72, 128])
@pytest.mark.parametrize("tile", [16, 64])
def test_instances(gpu, monkeypatch, tile, rank_max, bf16):           # noqa: F811
    torch, b = gpu
    monkeypatch.setenv("W2A8_LORA_TILE", str(tile))
    for M, Ns, K, L in [(1, (16,), 64, 1), (15, (272, 48), 704, 2), (33, (144,), 1088, 1), (70, (528, 16), 192, 3), (129, (64,), 2112, 2)]:
        p = _integers(torch, M, Ns, K, L, rank_max, seed=M + rank_max, bf16=bf16)
        lora = b.LoraGroup(p["A"], p["B"], rank=p["rank"], scale=p["scale"])
        y = b.w2a8_lora_grouped(p["x"], p["adapter"], lora, base=p["base"])
        _equal(torch, y, _reference(torch, p["x"], p["adapter"], p["A"], p["B"], p["rank"], p["scale"], p["base"]))


@pytest.mark.parametrize("tile", [16, 64])
@pytest.mark.parametrize("C", [1, 4, 8])
def test_many_chunks_and_shares(gpu, monkeypatch, tile, C):          # noqa: F811
    """More tokens than are sorted at a time, more tiles than clusters, several shares of the channels, and adapters
    whose tokens fill tiles exactly, by one less and by one more."""
    torch, b = gpu
    monkeypatch.setenv("W2A8_LORA_TILE", str(tile))
    monkeypatch.setenv("W2A8_LORA_C", str(C))
    L, sizes = 6, [64, 63, 65, 128, 0, 1]
    owner = torch.cat([torch.full((n,), a) for a, n in enumerate(sizes)] + [torch.full((4100 - sum(sizes),), -1)])
    for shuffle in (False, True):
        p = _integers(torch, 4100, (1024, 32), 128, L, 16, seed=C)
        order = torch.randperm(4100, generator=torch.Generator().manual_seed(C)) if shuffle else torch.arange(4100)
        p["adapter"] = owner[order].to(torch.int32).cuda()
        lora = b.LoraGroup(p["A"], p["B"], rank=p["rank"], scale=p["scale"])
        y = b.w2a8_lora_grouped(p["x"], p["adapter"], lora, base=p["base"])
        _equal(torch, y, _reference(torch, p["x"], p["adapter"], p["A"], p["B"], p["rank"], p["scale"], p["base"]))
        b.w2a8_lora_grouped(p["x"], p["adapter"], lora, base=p["base"], y=p["base"])
        assert all(torch.equal(u, v) for u, v in zip(p["base"], y))


def test_replayed_with_other_owners(gpu):                            # noqa: F811
    """One captured launch, replayed with other owners of the tokens (one tile, many tiles, no adapter at all), other
    ranks and other adapters: everything is read anew."""
    torch, b = gpu
    M, Ns, K, L, r = 48, (256, 64), 512, 8, 32
    p = _integers(torch, M, Ns, K, L, r, seed=3)
    for t in p["A"] + p["B"]:
        t.nan_to_num_(nan=1.0)
    lora = b.LoraGroup(p["A"], p["B"], rank=p["rank"], scale=p["scale"])
    y = [torch.empty_like(t) for t in p["base"]]
    b.w2a8_lora_grouped(p["x"], p["adapter"], lora, base=p["base"], y=y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.w2a8_lora_grouped(p["x"], p["adapter"], lora, base=p["base"], y=y)
    g = torch.Generator(device="cuda").manual_seed(1)
    for k in range(4):
        p["adapter"].copy_([torch.zeros(M), torch.arange(M) % L, torch.full((M,), -1.0), torch.arange(M) // 7][k].to(torch.int32).cuda())
        p["rank"].copy_(torch.randint(0, r + 1, (L,), generator=g, device="cuda", dtype=torch.int32))
        for t in p["A"]:
            t.copy_(t.flip(0))
        graph.replay()
        torch.cuda.synchronize()
        _equal(torch, y, _reference(torch, p["x"], p["adapter"], p["A"], p["B"], p["rank"], p["scale"], p["base"]))


@pytest.mark.parametrize("rank_max", [16, 32, 64, 128])
@pytest.mark.parametrize("tile", [16, 64])
def test_low_ranks_beside_bits_of_nan(gpu, monkeypatch, tile, rank_max):   # noqa: F811
    """Ranks far below what the storage is laid out for, while what else passes through the kernel's stages holds the bit
    patterns of bf16 NaNs: the fp32 base values have them in their lower halves.  Nothing of it may meet the products."""
    torch, b = gpu
    monkeypatch.setenv("W2A8_LORA_TILE", str(tile))
    M, Ns, K, L = 150, (1040, 272), 576, 5
    p = _integers(torch, M, Ns, K, L, rank_max, seed=rank_max, ranks=[1, 3, 8, rank_max // 2 + 1, rank_max - 3])
    for t in p["base"]:
        bits = t.view(torch.int32)
        bits.copy_((bits & -65536) | 0x7FC0)
        assert bool(t.isfinite().all())
    lora = b.LoraGroup(p["A"], p["B"], rank=p["rank"], scale=p["scale"])
    for _ in range(2):
        y = b.w2a8_lora_grouped(p["x"], p["adapter"], lora, base=p["base"])
        _equal(torch, y, _reference(torch, p["x"], p["adapter"], p["A"], p["B"], p["rank"], p["scale"], p["base"]))
