"""Pools of hundreds of adapters with all of them in use (the tokens' sort lays its counts out by the size of the pool), in tiles
of both sizes; exact on integers, see test_gpu_lora.py."""
import pytest

from test_gpu_lora import _equal, _integers, gpu                     # noqa: F401

pytestmark = pytest.mark.gpu


def _reference(torch, p):
    """As in test_gpu_lora.py, with all adapters of a token's list at once."""
    out = []
    owner = p["adapter"].long()
    with_one = owner >= 0
    a = owner.clamp(min=0)
    for A, B, base in zip(p["A"], p["B"], p["base"]):
        ranks = torch.arange(A.shape[1], device="cuda")
        live = ranks[None] < p["rank"][:, None]                      # [adapters][rank_max]
        A0 = torch.where(live[:, :, None], A.double(), 0.0)
        B0 = torch.where(live[:, None, :], B.double(), 0.0)
        y = base.double().clone()
        for first in range(0, len(a), 1024):
            at = slice(first, first + 1024)
            h = torch.einsum("mk,mrk->mr", p["x"][at].double(), A0[a[at]]) * p["scale"].double()[a[at]][:, None]
            y[at] += torch.einsum("mr,mnr->mn", h, B0[a[at]]) * with_one[at][:, None]
        out.append(y)
    return out


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("tile", [None, 16, 64])
@pytest.mark.parametrize("M,L,rank_max", [(9000, 1024, 16), (5000, 1024, 8), (4097, 600, 24), (3000, 257, 64), (2000, 256, 16),
                                          (1500, 255, 40), (1100, 1023, 128)])
def test_all_in_use(gpu, monkeypatch, M, L, rank_max, tile, bf16):   # noqa: F811
    torch, b = gpu
    if tile:
        monkeypatch.setenv("W2A8_LORA_TILE", str(tile))
    p = _integers(torch, M, (48, 16), 128, L, rank_max, seed=M + L, bf16=bf16, none=0.1)
    if M >= L:                               # each of them at least once, in no order
        order = torch.randperm(M, generator=torch.Generator().manual_seed(L))[:L].cuda()
        p["adapter"][order] = torch.arange(L, dtype=torch.int32, device="cuda")
    lora = b.LoraGroup(p["A"], p["B"], rank=p["rank"], scale=p["scale"])
    want = _reference(torch, p)
    _equal(torch, b.w2a8_lora_grouped(p["x"], p["adapter"], lora, base=p["base"]), want)
    b.w2a8_lora_grouped(p["x"], p["adapter"], lora, base=p["base"], y=p["base"])
    _equal(torch, p["base"], want)
