"""Sizes that the library's ints do not hold are refused by the binding (ctypes would hand on their lower 32 bits, a small
and wrong size), without a GPU and without the memory."""
import pytest

BIG = 1 << 32


@pytest.fixture(scope="module")
def b():
    from paper_2508_06753_b200 import build, binding
    build.build()
    binding.lib()
    return binding


def test_adapters(b):
    import torch
    bf = lambda *shape: torch.empty(shape, dtype=torch.bfloat16, device="meta")
    b.LoraGroup([bf(2, 8, 64)], [bf(2, 16, 8)])
    for A, B in [((2, 8, BIG + 64), (2, 16, 8)), ((2, 8, 64), (2, BIG + 16, 8)), ((2, BIG + 8, 64), (2, 16, BIG + 8)),
                 ((BIG + 2, 8, 64), (BIG + 2, 16, 8))]:
        with pytest.raises(ValueError, match="32 bits"):
            b.LoraGroup([bf(*A)], [bf(*B)])
    with pytest.raises(ValueError, match="32 bits"):
        b.LoraGroup([bf(2, 8, 64)] * 2, [bf(2, 16, 8), bf(2, BIG + 16, 8)])


def test_heads(b):
    import torch
    x = torch.zeros((1, 1, 2))
    for shape in [(BIG + 3, 1, 2), (1, BIG + 3, 2)]:
        with pytest.raises(ValueError, match="32 bits"):
            b.Heads([x.expand(shape)], [x.expand(shape)])
    wide = torch.empty((1, 1, BIG + 64), device="meta")
    with pytest.raises(ValueError, match="32 bits"):
        b.Heads([wide])


def test_frequencies(b):
    good = b.w2a8_rope_frequencies(64, 1e4, "llama3", factor=2.0, high=4.0, original_length=8192, device="cpu")
    assert len(good[0]) == 32
    with pytest.raises(ValueError, match="32 bits"):
        b.w2a8_rope_frequencies(64, 1e4, "llama3", factor=2.0, high=4.0, original_length=BIG + 8192, device="cpu")
    with pytest.raises(ValueError, match="32 bits"):
        b.w2a8_rope_frequencies(BIG + 64, 1e4, device="cpu")


def test_rotation_without_positions(b, monkeypatch):
    import torch
    monkeypatch.setattr(b, "_launch_stream", lambda *a: 0)              # the checks behind the one for a device
    heads, freq = b.Heads([torch.zeros((3, 2, 64))]), torch.zeros(32, dtype=torch.float64)
    with pytest.raises(ValueError, match="positions"):
        b.w2a8_qk_norm_rope(heads, 1e-6, inv_freq=freq)
    with pytest.raises(ValueError, match="positions"):
        b.w2a8_rope(heads, None, freq)
