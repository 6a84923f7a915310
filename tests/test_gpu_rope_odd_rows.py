"""Rotary positions and head norms on column ranges of wider rows whose heads, rotated parts or strides are no multiple of 8
(single values, see test_gpu_rope.py for the bounds), from one token to as many as make a CTA take several."""
import pytest

from test_gpu_rope import _reference, gpu                            # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("src,dst", [("float32", "bfloat16"), ("bfloat16", "bfloat16"), ("bfloat16", "float32"), ("float32", "float32")])
@pytest.mark.parametrize("M,H,Hk,D,rot,spare", [(1, 3, 1, 30, 30, 0), (5, 3, 1, 30, 14, 1), (4001, 12, 5, 80, 60, 0), (4001, 5, 3, 80, 20, 3),
                                                (3003, 9, 2, 42, 42, 5), (2600, 7, 1, 128, 36, 0), (9001, 2, 1, 10, 6, 1), (1200, 3, 2, 510, 254, 0)])
def test_packed_rows(gpu, M, H, Hk, D, rot, spare, src, dst, interleaved, norm):     # noqa: F811
    """q and k of one q|k|v result, into results of their own and, of one type, in place; `spare` values behind each row."""
    torch, b = gpu
    src, dst = getattr(torch, src), getattr(torch, dst)
    g = torch.Generator(device="cuda").manual_seed(M + D + rot)
    wide = (H + 2 * Hk) * D + spare
    rows = torch.randn((M, wide), generator=g, device="cuda").to(src)
    start = rows.clone()
    cut = lambda t, h0, h: t[:, h0 * D:(h0 + h) * D].unflatten(1, (h, D))
    x = [cut(rows, 0, H), cut(rows, H, Hk)]
    pos = torch.randint(-1000, 200000, (M,), generator=g, device="cuda", dtype=torch.int32)
    inv_freq, amp = b.w2a8_rope_frequencies(rot, 10000.0, "linear", factor=2.0)
    weight = [1 + 0.3 * torch.randn(D, generator=g, device="cuda") for _ in x]
    run = (lambda hd: b.w2a8_qk_norm_rope(hd, 1e-5, pos, inv_freq, amp, interleaved=interleaved)) if norm else \
        (lambda hd: b.w2a8_rope(hd, pos, inv_freq, amp, interleaved=interleaved))
    to = torch.full((M, wide), 5.0, dtype=dst, device="cuda")
    out = [cut(to, 0, H), cut(to, H, Hk)]
    got = run(b.Heads(x, out, weight=weight))
    assert torch.equal(rows, start)
    for y, t, w in zip(got, x, weight):
        want, tol = _reference(torch, t, w if norm else None, 1e-5 if norm else None, pos, inv_freq, amp, interleaved, dst == torch.bfloat16)
        err = (y.double() - want).abs()
        assert bool((err <= tol).all()), float((err - tol).max())
        if not norm:
            assert torch.equal(y[..., rot:], t[..., rot:].to(dst))
    assert bool((to[:, (H + Hk) * D:] == 5.0).all())
    if src == dst:
        run(b.Heads(x, x, weight=weight))
        assert torch.equal(rows[:, :(H + Hk) * D], to[:, :(H + Hk) * D])
        assert torch.equal(rows[:, (H + Hk) * D:], start[:, (H + Hk) * D:])
