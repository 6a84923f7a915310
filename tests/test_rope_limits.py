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


@pytest.mark.parametrize("norm", [False, True])
def test_alignment_of_single_values(lib, mem, norm):
    """Heads, rotated parts or strides that are no multiple of 8 go value by value: as aligned as their type, so that a view
    behind odd heads of the same rows is taken.  Of others every one has to be 16-byte aligned."""
    _, p = mem
    far, arrays = p + 65536, p + 131072
    call = lambda x, out, D, rot, xs, os, **t: _call(lib, norm, [x], [out], arrays, arrays + 4096, 3, [2], D, rot, [xs], [os], **t)
    for t, e in (dict(x16=1, o16=1), 2), (dict(x16=0, o16=0), 4):
        fine = call(p, far, 30, 30, (150, 30), (60, 30), **t)       # whatever a call without a fault returns here
        assert fine not in (SHAPE, ALIGN)
        for D, rot, xs, os in [(30, 30, (150, 30), (60, 30)), (64, 36, (320, 64), (128, 64)), (64, 64, (324, 64), (128, 64)),
                               (64, 64, (320, 64), (132, 66))]:
            assert call(p + e, far, D, rot, xs, os, **t) == fine and call(p, far + e, D, rot, xs, os, **t) == fine
            assert call(p + 1, far, D, rot, xs, os, **t) == ALIGN and call(p, far + e // 2, D, rot, xs, os, **t) == ALIGN
        assert call(p + 8, far, 64, 64, (320, 64), (128, 64), **t) == ALIGN
        assert call(p, far + 8, 64, 64, (320, 64), (128, 64), **t) == ALIGN
