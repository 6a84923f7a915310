"""Rotary positions and head norms for as many tokens as make a CTA take several, whose rows are then copied ahead into
shared memory: every piece size (four fp32 values, four and eight bf16 ones, two chunks per lane), both layouts, token
counts that no CTA's share divides, in place and into other strides.  Bounds: see test_gpu_rope.py."""
import pytest

from test_gpu_rope import _reference, gpu                            # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("src,dst", [("float32", "bfloat16"), ("bfloat16", "bfloat16"), ("bfloat16", "float32"), ("float32", "float32")])
@pytest.mark.parametrize("M,heads,D,rot", [(4003, (20, 5), 128, 128), (3001, (18,), 64, 48), (2500, (30, 2), 80, 32),
                                           (2999, (12,), 72, 24), (1501, (9, 2), 512, 256), (5000, (3,), 256, 256)])
def test_against_64_bits(gpu, M, heads, D, rot, src, dst, interleaved, norm):    # noqa: F811
    torch, b = gpu
    src, dst = getattr(torch, src), getattr(torch, dst)
    g = torch.Generator(device="cuda").manual_seed(M + D)
    rows = [torch.randn((M, h + 1, D), generator=g, device="cuda").to(src) for h in heads]
    x = [t[:, :h] for t, h in zip(rows, heads)]
    pos = torch.randint(-1000, 200000, (M,), generator=g, device="cuda", dtype=torch.int32)
    inv_freq, amp = b.w2a8_rope_frequencies(rot, 10000.0, "linear", factor=2.0)
    weight = [1 + 0.3 * torch.randn(D, generator=g, device="cuda") for _ in heads]
    out = [torch.full((h, M + 1, D), 5.0, dtype=dst, device="cuda") for h in heads]          # heads before tokens, a row spare
    grp = b.Heads(x, [o[:, :M].transpose(0, 1) for o in out], weight=weight)
    run = (lambda hd: b.w2a8_qk_norm_rope(hd, 1e-5, pos, inv_freq, amp, interleaved=interleaved)) if norm else \
        (lambda hd: b.w2a8_rope(hd, pos, inv_freq, amp, interleaved=interleaved))
    got = run(grp)
    for y, t, w, o in zip(got, x, weight, out):
        want, tol = _reference(torch, t, w if norm else None, 1e-5 if norm else None, pos, inv_freq, amp, interleaved, dst == torch.bfloat16)
        err = (y.double() - want).abs()
        assert bool((err <= tol).all()), float((err - tol).max())
        assert bool((o[:, M] == 5.0).all())
    if src == dst:                                                   # in place gives the same bits, and leaves what is beside
        beside = [t[:, -1].clone() for t in rows]
        keep = [y.clone() for y in got]
        run(b.Heads(x, x, weight=weight))
        assert all(torch.equal(u, v) for u, v in zip(x, keep))
        assert all(torch.equal(t[:, -1], v) for t, v in zip(rows, beside))


def test_few_and_many_tokens_give_the_same_bits(gpu):                # noqa: F811
    """A token's bits do not depend on how many tokens its CTA takes."""
    torch, b = gpu
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn((6000, 16, 128), generator=g, device="cuda").to(torch.bfloat16)
    pos = torch.randint(0, 100000, (6000,), generator=g, device="cuda", dtype=torch.int32)
    inv_freq, amp = b.w2a8_rope_frequencies(128, 10000.0)
    w = torch.randn(128, generator=g, device="cuda")
    many, = b.w2a8_qk_norm_rope(b.Heads([x], weight=[w]), 1e-6, pos, inv_freq, amp)
    for a, z in [(0, 1), (17, 40), (5990, 6000)]:
        few, = b.w2a8_qk_norm_rope(b.Heads([x[a:z]], weight=[w]), 1e-6, pos[a:z].clone(), inv_freq, amp)
        assert torch.equal(few, many[a:z])
