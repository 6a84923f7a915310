"""Angles of far positions against whole numbers: a frequency of 2 pi / 2^n turns a position by (position mod 2^n) / 2^n of a
turn, which integers give exactly.  Bound: ROTATION of test_gpu_rope.py, and four half steps of the angle in 64 bits (2 pi 2^-n
as it is stored, its quotient by 2 pi with the rounded constant, their product, the product with the position)."""
import math

import pytest

from test_gpu_rope import ROTATION, gpu                              # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("interleaved", [False, True])
def test_turns_of_integers(gpu, interleaved):                        # noqa: F811
    torch, b = gpu
    D = 64
    n = torch.arange(D // 2)                                         # pair p turns once in 2^p positions
    at = [0, 1, -1, 3, 12345, -98765, 131071, 2 ** 20 + 1, 2 ** 24 + 3, 2 ** 30 + 7, 2 ** 31 - 1, -(2 ** 31), -(2 ** 31) + 1]
    inv_freq = (2 * math.pi * 0.5 ** n.double()).cuda()
    pos = torch.tensor(at, dtype=torch.int32, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(9)
    x = torch.randn((len(at), 3, D), generator=g, device="cuda")
    y, = b.w2a8_rope(b.Heads([x]), pos, inv_freq, interleaved=interleaved)
    turns = torch.tensor([[(t % 2 ** int(k)) / 2 ** int(k) for k in n] for t in at], dtype=torch.float64, device="cuda")
    c, s = torch.cos(2 * math.pi * turns)[:, None], torch.sin(2 * math.pi * turns)[:, None]
    i, j = (slice(0, D, 2), slice(1, D, 2)) if interleaved else (slice(0, D // 2), slice(D // 2, D))
    u, v = x[..., i].double(), x[..., j].double()
    angle = pos.double().abs()[:, None, None] * inv_freq
    tol = (u.abs() + v.abs()) * (ROTATION + 4 * 2.0 ** -53 * angle)
    assert bool(((y[..., i].double() - (u * c - v * s)).abs() <= tol).all())
    assert bool(((y[..., j].double() - (v * c + u * s)).abs() <= tol).all())
