"""Results of the adapters and of the rotary positions that would lie over something else that the call reads: refused
before anything is launched."""
import ctypes

import pytest

SHAPE = -2


@pytest.fixture(scope="module")
def lib():
    from paper_2508_06753_b200 import build, binding
    build.build()
    return binding.lib()


@pytest.fixture(scope="module")
def mem():
    buf = ctypes.create_string_buffer(1 << 20)
    return buf, (ctypes.addressof(buf) + 255) // 256 * 256


def _ptrs(*p):
    return (ctypes.c_void_p * len(p))(*p)


def test_adapters_result_over_another_input(lib, mem):
    _, p = mem
    M, K, Ns, L, r = 5, 64, (16, 32), 3, 8
    x, adapter, rank, scale, A0, A1, B0, B1, y0, y1 = (p + i * 65536 for i in range(10))
    e = 4

    def call(y):
        return lib.w2a8_lora_grouped(x, adapter, L, r, rank, scale, 2, _ptrs(A0, A1), _ptrs(B0, B1), None, _ptrs(*y), 0,
                                     (ctypes.c_int * 2)(*Ns), M, K, None)

    # bytes of each input; a result that ends in its first or begins in its last 16 bytes
    sizes = {x: M * K * 2, adapter: M * 4, rank: L * 4, scale: L * 4, A0: L * r * K * 2, A1: L * r * K * 2,
             B0: L * Ns[0] * r * 2, B1: L * Ns[1] * r * 2}
    for at, n in sizes.items():
        last = at + (n - 1) // 16 * 16
        assert call((last, y1)) == SHAPE and call((y0, last)) == SHAPE
        for i, first in enumerate((at + 16 - M * Ns[0] * e, at + 16 - M * Ns[1] * e)):
            assert call((first, y1) if i == 0 else (y0, first)) == SHAPE


@pytest.mark.parametrize("norm", [False, True])
def test_rotated_result_over_another_input(lib, mem, norm):
    """Positions, frequencies and weights; beside the rows of a wider result they are not refused for it."""
    _, p = mem
    M, H, D, wide = 5, 2, 64, 256                           # rows of 256 values, 128 of them the result's
    x, pos, freq, w, out = (p + i * 65536 for i in range(5))

    def call(out, pos=pos, freq=freq, w=w, rot=D):
        s = lambda *v: (ctypes.c_int64 * 2)(*v)
        mid = [_ptrs(w), 1e-6] if norm else []
        return (lib.w2a8_qk_norm_rope if norm else lib.w2a8_rope)(
            1, _ptrs(x), 0, _ptrs(out), 0, *mid, (ctypes.c_int * 1)(H), s(H * D, D), s(wide, D), M, D, rot, 0, pos, freq, 1.0, None)

    free = call(out)                                        # whatever a call without a fault returns here
    assert free != SHAPE
    row = wide * 4
    for name, at, n in [("pos", pos, M * 4), ("freq", freq, D // 2 * 8)] + ([("w", w, D * 4)] if norm else []):
        assert call(at) == SHAPE
        assert call(at + (n - 1) // 16 * 16) == SHAPE       # the first row begins in its last bytes
        assert call(at + 16 - H * D * 4) == SHAPE           # the first row ends in its first
        assert call(at - 3 * row - 64) == SHAPE             # inside the fourth row
        kept = {name: out + 2 * row + H * D * 4}            # behind the third row, before the fourth
        assert call(out, **kept) == free
        kept = {name: out + 2 * row + H * D * 4 - 16}
        assert call(out, **kept) == SHAPE
        kept = {name: out + 3 * row - 16}
        assert call(out, **kept) == (free if n <= 16 else SHAPE)
    if norm:
        assert call(out, pos=out, freq=out, rot=0) != SHAPE            # not read without a rotation
