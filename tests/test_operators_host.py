"""Adapters, rotary positions and head norms: refusals and host logic, without a GPU.  Every refused call returns before
anything is launched."""
import ctypes
import math

import pytest

NULLP, SHAPE, ALIGN = -1, -2, -3


@pytest.fixture(scope="module")
def lib():
    from paper_2508_06753_b200 import build, binding
    build.build()
    return binding.lib()


@pytest.fixture(scope="module")
def mem():
    buf = ctypes.create_string_buffer(1 << 20)
    p = (ctypes.addressof(buf) + 255) // 256 * 256
    return buf, p


def _ptrs(*p):
    return (ctypes.c_void_p * len(p))(*p)


def test_lora_refusals(lib, mem):
    _, p = mem
    M, K, N = 2, 64, 16
    x, ad, A, B, base, y = (p + i * 65536 for i in range(6))
    n = (ctypes.c_int * 1)(N)

    def call(x=x, ad=ad, adapters=2, rank_max=8, rank=None, scale=None, count=1, A=_ptrs(A), B=_ptrs(B),
             base=_ptrs(base), y=_ptrs(y), bf16=0, n=n, M=M, K=K):
        return lib.w2a8_lora_grouped(x, ad, adapters, rank_max, rank, scale, count, A, B, base, y, bf16, n, M, K, None)

    assert call(x=None) == NULLP and call(ad=None) == NULLP
    assert call(A=None) == NULLP and call(B=None) == NULLP and call(y=None) == NULLP and call(n=None) == NULLP
    assert call(A=_ptrs(None)) == NULLP and call(B=_ptrs(None)) == NULLP
    assert call(y=_ptrs(None)) == NULLP and call(base=_ptrs(None)) == NULLP
    assert call(count=0) == SHAPE and call(count=5) == SHAPE
    assert call(adapters=0) == SHAPE and call(adapters=1025) == SHAPE
    assert call(rank_max=0) == SHAPE and call(rank_max=12) == SHAPE and call(rank_max=136) == SHAPE
    assert call(M=0) == SHAPE and call(M=-1) == SHAPE and call(M=(1 << 30) + 1) == SHAPE and call(K=96) == SHAPE and call(K=0) == SHAPE
    assert call(n=(ctypes.c_int * 1)(24)) == SHAPE and call(n=(ctypes.c_int * 1)(0)) == SHAPE
    assert call(x=x + 8) == ALIGN and call(ad=ad + 2) == ALIGN and call(rank=ad + 1) == ALIGN and call(scale=ad + 2) == ALIGN
    assert call(A=_ptrs(p + 8)) == ALIGN and call(B=_ptrs(p + 8)) == ALIGN
    assert call(y=_ptrs(y + 8)) == ALIGN and call(base=_ptrs(base + 4)) == ALIGN
    # a result over the activations, over part of its base, over another result or another base
    assert call(y=_ptrs(x)) == SHAPE and call(y=_ptrs(x + M * K * 2 - 16)) == SHAPE
    assert call(base=_ptrs(y + 16)) == SHAPE and call(base=_ptrs(y - 16)) == SHAPE
    n2 = (ctypes.c_int * 2)(N, N)
    two = dict(count=2, A=_ptrs(A, A), B=_ptrs(B, B), n=n2)
    assert call(base=None, y=_ptrs(y, y), **two) == SHAPE
    assert call(base=_ptrs(y + 4096, y), y=_ptrs(y, y + 4096), **two) == SHAPE


def _rope(lib, norm=False, x=None, out=None, x16=0, o16=0, heads=2, xs=None, os=None, M=3, D=64, rot=64, pos=None,
          freq=None, count=1, eps=1e-6, weight=None):
    s = lambda v: (ctypes.c_int64 * len(v))(*v)
    args = [count, x, x16, out, o16]
    if norm:
        args += [weight, eps]
    args += [(ctypes.c_int * 4)(*[heads] * 4), s(xs or [heads * D, D]), s(os or [heads * D, D]), M, D, rot, 0, pos, freq, 1.0, None]
    return (lib.w2a8_qk_norm_rope if norm else lib.w2a8_rope)(*args)


@pytest.mark.parametrize("norm", [False, True])
def test_rope_refusals(lib, mem, norm):
    _, p = mem
    x, out, pos, freq = p, p + 65536, p + 131072, p + 196608
    ok = dict(norm=norm, x=_ptrs(x), out=_ptrs(out), pos=pos, freq=freq)
    call = lambda **kw: _rope(lib, **{**ok, **kw})
    assert call(x=None) == NULLP and call(out=None) == NULLP and call(x=_ptrs(None)) == NULLP and call(out=_ptrs(None)) == NULLP
    assert call(pos=None) == NULLP and call(freq=None) == NULLP
    assert call(count=0) == SHAPE and call(count=5) == SHAPE and call(M=0) == SHAPE and call(heads=0) == SHAPE
    assert call(D=63, rot=62) == SHAPE and call(D=0, rot=0) == SHAPE and call(D=514, rot=64) == SHAPE
    assert call(rot=63) == SHAPE and call(rot=66) == SHAPE and call(rot=-2) == SHAPE
    if not norm:
        assert call(rot=0) == SHAPE
    else:
        assert call(eps=-1.0) == SHAPE and call(eps=math.nan) == SHAPE
        assert call(weight=_ptrs(p + 2)) == ALIGN
    assert call(x=_ptrs(x + 8)) == ALIGN and call(out=_ptrs(out + 8)) == ALIGN
    assert call(pos=pos + 2) == ALIGN and call(freq=freq + 4) == ALIGN
    # rows of the result that share elements, negative strides
    assert call(os=[0, 64]) == SHAPE and call(os=[64, 64]) == SHAPE and call(os=[128, 32]) == SHAPE
    assert call(xs=[-128, 64]) == SHAPE and call(os=[128, -64]) == SHAPE
    # over its input, but not in place
    assert call(out=_ptrs(x), o16=1) == SHAPE and call(out=_ptrs(x), os=[256, 64]) == SHAPE
    assert call(out=_ptrs(x + 16)) == SHAPE


def test_rope_refuses_a_result_over_another_result(lib, mem):
    _, p = mem
    s4 = (ctypes.c_int64 * 4)(128, 64, 128, 64)
    h2 = (ctypes.c_int * 2)(2, 2)
    args = lambda x, out: [2, _ptrs(*x), 0, _ptrs(*out), 0, h2, s4, s4, 3, 64, 64, 0, p + 400000, p + 500000, 1.0, None]
    assert lib.w2a8_rope(*args((p, p + 65536), (p + 131072, p + 131072))) == SHAPE
    assert lib.w2a8_rope(*args((p, p + 65536), (p + 131072, p + 131072 + 256))) == SHAPE
    # results that change places would be read after they were written
    assert lib.w2a8_rope(*args((p, p + 65536), (p + 65536, p))) == SHAPE


def test_frequencies(lib):
    from paper_2508_06753_b200 import binding as b
    D, base, n = 128, 500000.0, 8192
    f = [base ** (-2 * i / D) for i in range(D // 2)]
    got = lambda *a, **k: b.w2a8_rope_frequencies(D, base, *a, device="cpu", **k)
    close = lambda t, want: all(abs(u - v) <= 1e-13 * v for u, v in zip(t.tolist(), want))
    t, amp = got()
    assert close(t, f) and amp == 1.0 and len(t) == 64
    t, amp = got("linear", factor=4.0)
    assert close(t, [v / 4 for v in f]) and amp == 1.0
    t, _ = got("ntk", factor=4.0)
    nb = base * 4.0 ** (D / (D - 2))
    assert close(t, [nb ** (-2 * i / D) for i in range(D // 2)])
    assert abs(t[-1] * 4 / f[-1] - 1) < 1e-12                      # the slowest pair is stretched by the factor
    t, _ = got("llama3", factor=8.0, low=1.0, high=4.0, original_length=n)
    for u, v in zip(t.tolist(), f):
        wave = 2 * math.pi / v
        if wave < n / 4.0:
            want = v
        elif wave > n / 1.0:
            want = v / 8
        else:
            m = (n / wave - 1.0) / (4.0 - 1.0)
            want = (1 - m) * v / 8 + m * v
        assert abs(u - want) <= 1e-12 * want
    t, amp = got("yarn", factor=8.0, low=1.0, high=32.0, original_length=n)
    assert abs(amp - (0.1 * math.log(8.0) + 1)) < 1e-6
    dim = lambda turns: D * math.log(n / (turns * 2 * math.pi)) / (2 * math.log(base))
    lo, hi = math.floor(dim(32.0)), math.ceil(dim(1.0))
    for i, (u, v) in enumerate(zip(t.tolist(), f)):
        m = min(max((i - lo) / (hi - lo), 0.0), 1.0)
        want = v * (1 - m) + v / 8 * m
        assert abs(u - want) <= 1e-12 * want
    assert 0 < lo < hi < D // 2 and t[lo] == f[lo] and abs(t[hi] * 8 / f[hi] - 1) < 1e-12


def test_frequency_refusals(lib):
    from paper_2508_06753_b200 import binding as b
    out = (ctypes.c_double * 64)()
    amp = ctypes.c_float()
    call = lambda rot=64, base=1e4, s=0, f=1.0, lo=1.0, hi=4.0, n=4096, o=ctypes.addressof(out), a=ctypes.addressof(amp): \
        lib.w2a8_rope_frequencies(rot, base, s, f, lo, hi, n, o, a)
    assert call() == 0
    assert call(o=None) == NULLP and call(a=None) == NULLP
    assert call(rot=0) == SHAPE and call(rot=7) == SHAPE and call(rot=514) == SHAPE
    assert call(base=1.0) == SHAPE and call(base=math.nan) == SHAPE and call(base=math.inf) == SHAPE
    assert call(s=5) == SHAPE and call(s=-1) == SHAPE and call(s=1, f=0.5) == SHAPE and call(s=1, f=math.nan) == SHAPE
    for s in (3, 4):
        assert call(s=s, f=2.0, n=0) == SHAPE and call(s=s, f=2.0, lo=0.0) == SHAPE and call(s=s, f=2.0, lo=4.0, hi=4.0) == SHAPE
        assert call(s=s, f=2.0) == 0
    assert call(s=2, rot=2, f=2.0) == SHAPE
    with pytest.raises(ValueError):
        b.w2a8_rope_frequencies(64, 1e4, "dynamic", device="cpu")


def test_binding_refusals(lib):
    """Types, shapes, gaps and devices are looked at before the library is called."""
    import torch
    from paper_2508_06753_b200 import binding as b
    bf, L, r, K, N = torch.bfloat16, 2, 8, 64, 16
    A, B = torch.zeros((L, r, K), dtype=bf), torch.zeros((L, N, r), dtype=bf)
    with pytest.raises(TypeError):
        b.LoraGroup([A.float()], [B])
    with pytest.raises(ValueError):
        b.LoraGroup([A], [B, B])
    with pytest.raises(ValueError):
        b.LoraGroup([A], [torch.zeros((L + 1, N, r), dtype=bf)])
    with pytest.raises(ValueError):
        b.LoraGroup([A], [torch.zeros((L, r, N), dtype=bf).transpose(1, 2)])
    with pytest.raises(TypeError):
        b.LoraGroup([A], [B], rank=torch.zeros(L, dtype=torch.int64))
    with pytest.raises(ValueError):
        b.LoraGroup([A], [B], scale=torch.zeros(L + 1))
    with pytest.raises(ValueError):                                # not on a GPU
        b.w2a8_lora_grouped(torch.zeros((1, K), dtype=bf), torch.zeros(1, dtype=torch.int32), b.LoraGroup([A], [B]))
    x = torch.zeros((3, 2, 64))
    with pytest.raises(TypeError):
        b.Heads([x.half()])
    with pytest.raises(TypeError):
        b.Heads([x, x.to(bf)])
    with pytest.raises(ValueError):
        b.Heads([x, torch.zeros((4, 2, 64))])
    with pytest.raises(ValueError):
        b.Heads([x], [torch.zeros((3, 2, 32))])
    with pytest.raises(ValueError):
        b.Heads([x.transpose(1, 2)])
    with pytest.raises(ValueError):
        b.Heads([x] * 5)
    with pytest.raises(TypeError):
        b.Heads([x], weight=[torch.zeros(64, dtype=bf)])
    with pytest.raises(ValueError):
        b.w2a8_rope(b.Heads([x]), torch.zeros(3, dtype=torch.int32), torch.zeros(32, dtype=torch.float64))
