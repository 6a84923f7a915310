"""Norms of heads without a rotation (w2a8_qk_norm_rope with rot_dim 0): strides, types, several tokens per CTA, several results,
in place.  Bounds: see test_gpu_rope.py."""
import pytest

from test_gpu_rope import _reference, _rows, gpu                     # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("src,dst", [("float32", "bfloat16"), ("bfloat16", "bfloat16"), ("bfloat16", "float32"), ("float32", "float32")])
@pytest.mark.parametrize("layout", ["plain", "packed", "heads"])
@pytest.mark.parametrize("M,heads,D", [(1, (1,), 2), (1, (32, 8), 128), (7, (3, 1, 2, 5), 96), (33, (4,), 72), (5, (2,), 512),
                                       (9, (3,), 30), (3000, (20, 5), 128), (4001, (9,), 80), (2500, (7, 2), 256),
                                       (1501, (5,), 512), (2003, (6, 3), 42)])
def test_against_64_bits(gpu, M, heads, D, layout, src, dst):        # noqa: F811
    torch, b = gpu
    src, dst = getattr(torch, src), getattr(torch, dst)
    g = torch.Generator(device="cuda").manual_seed(M + D)
    x = [3 * _rows(torch, g, M, h, D, src, layout) if layout == "plain" else _rows(torch, g, M, h, D, src, layout) for h in heads]
    before = [t.clone() for t in x]
    weight = [1 + 0.3 * torch.randn(D, generator=g, device="cuda") if i != 1 else None for i in range(len(heads))]
    got = b.w2a8_qk_norm_rope(b.Heads(x, weight=weight, out_dtype=dst), 1e-5)
    for y, t, t0, w in zip(got, x, before, weight):
        assert torch.equal(t, t0)
        want, tol = _reference(torch, t, w, 1e-5, None, None, 1.0, False, dst == torch.bfloat16)
        err = (y.double() - want).abs()
        assert bool((err <= tol).all()), float((err - tol).max())
    if src == dst:
        b.w2a8_qk_norm_rope(b.Heads(x, x, weight=weight), 1e-5)
        assert all(torch.equal(t, y) for t, y in zip(x, got))
