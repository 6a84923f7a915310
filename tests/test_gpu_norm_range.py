"""Norms of rows whose squares pass the range of fp32: above it, and below it with an eps of next to nothing.  Bound: as in
test_gpu_rope.py (the scaling is by a power of two), and 2^-140 for what becomes subnormal on the way: a value beside one of
2^127 is held to 2^-150, times at most sqrt(512) < 2^5 and a weight below 2^2.  Subnormal bf16 results are 2^-133 apart, so
their rounding is off by up to 2^-134 however small they are."""
import pytest

from test_gpu_rope import _reference, gpu                            # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rotate", [False, True])
@pytest.mark.parametrize("eps", [0.0, 1e-38, 1e-6])
@pytest.mark.parametrize("src,dst", [("float32", "float32"), ("bfloat16", "bfloat16"), ("bfloat16", "float32")])
@pytest.mark.parametrize("M,H,D,rot", [(1, 7, 64, 64), (9, 5, 128, 128), (4000, 9, 128, 64), (5, 3, 30, 30), (3000, 9, 42, 10),
                                       (3, 4, 512, 512), (2000, 3, 320, 160), (3001, 6, 72, 72)])
def test_rows_far_from_one(gpu, M, H, D, rot, src, dst, eps, rotate):                # noqa: F811
    torch, b = gpu
    src, dst = getattr(torch, src), getattr(torch, dst)
    g = torch.Generator(device="cuda").manual_seed(M + D)
    x = torch.randn((M, H, D), generator=g, device="cuda").clamp(-4, 4)
    ordinary = x.to(src)
    size = torch.tensor([1.0, 2.0 ** 60, 1.0, 2.0 ** 90, 2.0 ** 125, 2.0 ** -60, 2.0 ** -75, 2.0 ** -100, 2.0 ** -135], device="cuda",
                        dtype=torch.float64)
    which = torch.randint(0, len(size), (M, H), generator=g, device="cuda")
    x = (ordinary.double() * size[which][..., None]).to(src)
    x[0, H - 1, : D // 2] = 3.0e38                                   # the type's largest, beside ordinary values
    x[0, 0, 0] = -3.0e38
    which[0, 0] = which[0, H - 1] = 1
    w = 1 + 0.3 * torch.randn(D, generator=g, device="cuda").clamp(-3, 3)
    pos = torch.randint(0, 100000, (M,), generator=g, device="cuda", dtype=torch.int32)
    inv_freq, amp = b.w2a8_rope_frequencies(rot, 10000.0)
    args = (pos, inv_freq, amp) if rotate else ()
    got, = b.w2a8_qk_norm_rope(b.Heads([x], weight=[w], out_dtype=dst), eps, *args)
    plain, = b.w2a8_qk_norm_rope(b.Heads([ordinary], weight=[w], out_dtype=dst), eps, *args)
    eps32 = float(torch.tensor(eps, dtype=torch.float32))
    want, tol = _reference(torch, x, w, eps32, pos, inv_freq if rotate else None, amp, False, dst == torch.bfloat16)
    none = (x == 0).all(-1) & (eps32 == 0)                           # of 2^-135 bf16 may leave a row of zeros: 0 / 0 without eps
    assert bool(want[~none].isfinite().all()) and bool(want[none].isnan().all())
    assert bool(got[none].isnan().all())
    err = (got.double() - want).abs()
    least = 2.0 ** -140 + (2.0 ** -134 if dst == torch.bfloat16 else 0.0)
    assert bool((err <= tol + least)[~none].all()), float((err - tol)[~none].max())
    if src == dst:                                                   # in place: the same bits
        z, bits = x.clone(), torch.int32 if src == torch.float32 else torch.int16
        b.w2a8_qk_norm_rope(b.Heads([z], [z], weight=[w]), eps, *args)
        assert torch.equal(z.view(bits), got.view(bits))
    same = (which == 0) | (which == 2)                               # ordinary rows: not a bit is changed by those beside them
    assert torch.equal(got[same], plain[same])


@pytest.mark.parametrize("D", [128, 30])
def test_zeros_infinities_and_nan(gpu, D):                           # noqa: F811
    """Without eps a row of zeros is 0 / 0; finite / inf is zero, inf / inf and NaN are NaN; the rows beside them are not touched."""
    torch, b = gpu
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((6, 3, D), generator=g, device="cuda")
    plain, = b.w2a8_qk_norm_rope(b.Heads([x.clone()]), 0.0)
    x[0, 0] = 0
    x[1, 1, 3] = float("inf")
    x[2, 2, 4] = float("nan")
    x[3, 0], x[3, 0, 7] = 1e30, -float("inf")
    x[4, 1], x[4, 1, 2] = 1e-30, float("nan")
    y, = b.w2a8_qk_norm_rope(b.Heads([x]), 0.0)
    for m, h in [(0, 0), (2, 2), (4, 1)]:
        assert bool(y[m, h].isnan().all())
    for m, h, k in [(1, 1, 3), (3, 0, 7)]:
        rest = [i for i in range(D) if i != k]
        assert bool(y[m, h, k].isnan()) and bool((y[m, h][rest] == 0).all())
    touched = torch.zeros((6, 3), dtype=torch.bool, device="cuda")
    for m, h in [(0, 0), (1, 1), (2, 2), (3, 0), (4, 1)]:
        touched[m, h] = True
    assert torch.equal(y[~touched], plain[~touched])
