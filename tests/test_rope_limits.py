"""Sizes at the ends of what the rope entry points count in: refused before anything is launched."""
import ctypes

import pytest

SHAPE, ALIGN = -2, -3


@pytest.fixture(scope="module")
def lib():
    from paper_2508_06753_b200 import build, binding
    build.build()
    return binding.lib()


@pytest.fixture(scope="module")
def mem():
    buf = ctypes.create_string_buffer(1 << 20)
    return buf, (ctypes.addressof(buf) + 255) // 256 * 256


def _call(lib, norm, x, out, pos, freq, M, heads, D, rot, xs, os, x16=0, o16=0, weight=None):
    """One entry of x, out, heads, xs and os per result."""
    n = len(x)
    flat = lambda v: (ctypes.c_int64 * (2 * n))(*[k for pair in v for k in pair])
    ptrs = lambda v: (ctypes.c_void_p * n)(*v)
    args = [n, ptrs(x), x16, ptrs(out), o16]
    if norm:
        args += [ptrs(weight) if weight else None, 1e-6]
    args += [(ctypes.c_int * n)(*heads), flat(xs), flat(os), M, D, rot, 0, pos, freq, 1.0, None]
    return (lib.w2a8_qk_norm_rope if norm else lib.w2a8_rope)(*args)


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("M", [(1 << 30) + 1, (1 << 31) - 8, (1 << 31) - 4, (1 << 31) - 1])
def test_tokens(lib, mem, M, norm):
    """One head of two values: memory would hold that many."""
    _, p = mem
    far = p + (1 << 40)
    assert _call(lib, norm, [p], [far], p, p, M, [1], 2, 2, [(2, 2)], [(2, 2)], x16=1, o16=1) == SHAPE


@pytest.mark.parametrize("norm", [False, True])
def test_strides(lib, mem, norm):
    """Rows whose last lies 2^64 bytes and more behind the first, where sums of 64 bits come round: two results over each
    other, a result over its input, an input and a result alone."""
    _, p = mem
    D, far = 64, p + 65536
    call = lambda *a: _call(lib, norm, *a[:2], p, p, *a[2:])
    M, wide, sane = 1 << 30, (1 << 40, D), (2 * D, D)
    assert call([p, p + (1 << 41)], [far, far], M, [2, 2], D, D, [sane] * 2, [wide] * 2) == SHAPE
    assert call([p], [p], M, [2], D, D, [sane], [wide]) == SHAPE
    assert call([p], [far], M, [2], D, D, [wide], [wide]) == SHAPE
    assert call([p], [far], M, [2], D, D, [wide], [sane]) == SHAPE
    heads = 1 << 17                                                     # the same by heads
    assert call([p], [p], 2, [heads], D, D, [(D, 2 * D)], [(D, 1 << 47)]) == SHAPE
