"""Rotary positions and per-head norms (w2a8_rope, w2a8_qk_norm_rope) against a plain 64-bit computation.

Bound of a value, from the roundings on its way.  Angle: the rest of a turn is held to 2^-26 of a turn (2 pi 2^-26 =
9.4e-8 radians); sincospif is within 2 units in the last place (2^-23); the amplitude and the two products and the sum add
2^-24 each, four in all: together below 5e-7 of amplitude * (|u| + |v|).  Norm: the sum of up to 512 squares is a chain of
at most 16 additions in a lane and 5 between lanes (21 2^-24, halved by the root), mean, root, division, product and
weight 2^-24 each: below 1e-6 of the value.  A bf16 result is rounded by at most 2^-8 of it."""
import pytest

from conftest import Guarded

pytestmark = pytest.mark.gpu
ROTATION, NORM = 5e-7, 1e-6


@pytest.fixture(scope="module")
def gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2508_06753_b200 import binding, build
    build.build()
    binding.lib()
    return torch, binding


def _reference(torch, x, weight, eps, pos, inv_freq, amp, interleaved, bf16):
    """(result in 64 bits, bound)"""
    z = x.double().clone()
    rel = 0.0
    if eps is not None:
        z = z / torch.sqrt((z * z).mean(-1, keepdim=True) + eps)
        if weight is not None:
            z = z * weight.double()
        rel = NORM
    bound = z.abs() * rel
    if inv_freq is not None:
        half = inv_freq.shape[0]
        i, j = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
        angle = (pos.double()[:, None] * inv_freq)[:, None]
        c, s = amp * angle.cos(), amp * angle.sin()
        u, v = z[..., i].clone(), z[..., j].clone()
        z[..., i], z[..., j] = u * c - v * s, v * c + u * s
        bound[..., i] = (u.abs() + v.abs()) * amp * (ROTATION + rel)
        bound[..., j] = bound[..., i]
    if bf16:
        bound = bound + (z.abs() + bound) * 2.0 ** -8
    return z, bound


def _rows(torch, g, M, H, D, dtype, layout):
    """[M][H][D] views: contiguous, columns of wider rows, or heads before tokens."""
    if layout == "packed":
        return torch.randn((M, H + 3, D), generator=g, device="cuda").to(dtype)[:, 2:2 + H] if D % 8 == 0 else \
            torch.randn((M, H, D), generator=g, device="cuda").to(dtype)
    if layout == "heads":
        return torch.randn((H, M, D), generator=g, device="cuda").to(dtype).transpose(0, 1)
    return torch.randn((M, H, D), generator=g, device="cuda").to(dtype)


CASES = [
    # M, heads, head_dim, rot, interleaved, layout
    (1, (1,), 2, 2, False, "plain"),                 # the smallest head, no vectors
    (1, (32, 8), 128, 128, False, "plain"),
    (3, (2, 1), 128, 128, True, "packed"),
    (5, (4, 2), 64, 48, True, "packed"),             # part of the head
    (7, (3,), 80, 32, False, "heads"),               # no power of two
    (2, (5, 1, 2, 3), 96, 96, False, "heads"),       # four results
    (9, (2, 2), 10, 6, False, "plain"),              # no multiple of 8: single values
    (4, (3,), 30, 30, True, "plain"),
    (6, (2,), 128, 36, False, "plain"),              # a rotated part that is no multiple of 8
    (3, (2,), 512, 512, False, "packed"),            # the largest head
    (3, (2,), 512, 512, True, "plain"),
    (2, (1,), 510, 510, False, "plain"),
    (300, (7, 3), 128, 64, False, "heads"),          # many tokens: all rows of a token in one CTA
    (700, (40,), 64, 64, False, "plain"),
    (500, (64, 8), 128, 128, True, "packed"),
]


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("src,dst", [("float32", "float32"), ("float32", "bfloat16"), ("bfloat16", "bfloat16"), ("bfloat16", "float32")])
@pytest.mark.parametrize("M,heads,D,rot,interleaved,layout", CASES)
def test_against_64_bits(gpu, M, heads, D, rot, interleaved, layout, src, dst, norm):
    torch, b = gpu
    src, dst = getattr(torch, src), getattr(torch, dst)
    g = torch.Generator(device="cuda").manual_seed(M + D + rot)
    x = [_rows(torch, g, M, h, D, src, layout) for h in heads]
    before = [t.clone() for t in x]
    pos = torch.randint(0, 200000, (M,), generator=g, device="cuda", dtype=torch.int32)
    inv_freq, amp = b.w2a8_rope_frequencies(rot, 10000.0, "yarn", factor=4.0, low=1.0, high=32.0, original_length=4096)
    outs = [Guarded(torch, (M, h, D), dst, fill=3.0) for h in heads]
    weight = [1 + 0.3 * torch.randn(D, generator=g, device="cuda") if i != 1 else None for i in range(len(heads))]
    grp = b.Heads(x, [o.view for o in outs], weight=weight)
    if norm:
        got = b.w2a8_qk_norm_rope(grp, 1e-5, pos, inv_freq, amp, interleaved=interleaved)
    else:
        got = b.w2a8_rope(grp, pos, inv_freq, amp, interleaved=interleaved)
    torch.cuda.synchronize()
    for y, t, t0, w, o in zip(got, x, before, weight, outs):
        o.check()
        assert torch.equal(t, t0)
        want, tol = _reference(torch, t, w if norm else None, 1e-5 if norm else None, pos, inv_freq, amp, interleaved,
                               dst == torch.bfloat16)
        err = (y.double() - want).abs()
        assert bool((err <= tol).all()), float((err - tol).max())
        if not norm:                                  # what is not rotated passes through
            assert torch.equal(y[..., rot:], t[..., rot:].to(dst))


@pytest.mark.parametrize("position", [0, 1, 2 ** 20 + 1, 2 ** 31 - 1, -1, -(2 ** 31)])
def test_positions_of_any_size(gpu, position):
    """Angles of far positions: against 64-bit integers of turns (exact modulo one turn for a frequency that is a
    binary fraction of a turn), and the general bound with 2^-53 of the angle added for the product in 64 bits."""
    torch, b = gpu
    D = 64
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn((1, 2, D), generator=g, device="cuda")
    pos = torch.tensor([position], dtype=torch.int32, device="cuda")
    inv_freq, amp = b.w2a8_rope_frequencies(D, 10000.0)
    y, = b.w2a8_rope(b.Heads([x]), pos, inv_freq, amp)
    want, tol = _reference(torch, x, None, None, pos, inv_freq, amp, False, False)
    # both sides round inv_freq / 2 pi and the product: up to 4 half steps of the angle in 64 bits, in radians
    tol = tol + 4 * abs(position) * 2.0 ** -53 * (x.abs().max() * 2).double()
    assert bool(((y.double() - want).abs() <= tol).all())
    if position == 0:
        assert torch.equal(y, x)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_in_place_on_a_wide_result(gpu, dtype, interleaved):
    """q and k are column ranges of one q|k|v result and rotated where they are; v is left as it was."""
    torch, b = gpu
    dtype = getattr(torch, dtype)
    g = torch.Generator(device="cuda").manual_seed(1)
    M, H, Hk, D = 35, 6, 2, 128
    rows = torch.randn((M, H + 2 * Hk, D), generator=g, device="cuda").to(dtype)
    start = rows.clone()
    pos = torch.arange(M, dtype=torch.int32, device="cuda") * 37
    inv_freq, amp = b.w2a8_rope_frequencies(D, 500000.0)
    x = [rows[:, :H], rows[:, H:H + Hk]]
    b.w2a8_qk_norm_rope(b.Heads(x, x), 1e-6, pos, inv_freq, amp, interleaved=interleaved)
    far = b.w2a8_qk_norm_rope(b.Heads([start[:, :H], start[:, H:H + Hk]]), 1e-6, pos, inv_freq, amp, interleaved=interleaved)
    assert torch.equal(x[0], far[0]) and torch.equal(x[1], far[1])
    assert torch.equal(rows[:, H + Hk:], start[:, H + Hk:])


def test_rotation_by_minus_position_undoes_it(gpu):
    torch, b = gpu
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn((11, 4, 64), generator=g, device="cuda")
    pos = torch.randint(0, 100000, (11,), generator=g, device="cuda", dtype=torch.int32)
    inv_freq, amp = b.w2a8_rope_frequencies(64, 10000.0)
    y = b.w2a8_rope(b.Heads([x]), pos, inv_freq, amp)
    z, = b.w2a8_rope(b.Heads(y), -pos, inv_freq, amp)
    pair = x[..., :32].abs() + x[..., 32:].abs()
    tol = torch.cat([pair, pair], -1) * 3 * ROTATION          # |u'| + |v'| <= sqrt(2) (|u| + |v|), two passes
    assert bool(((z - x).abs() <= tol).all())


def test_norm_alone_and_extreme_rows(gpu):
    """rot_dim 0; a row of zeros stays zero; tiny and large rows; NaN and infinity stay in their row."""
    torch, b = gpu
    g = torch.Generator(device="cuda").manual_seed(7)
    x = torch.randn((6, 3, 128), generator=g, device="cuda")
    x[0, 0] = 0
    x[1] *= 1e-12
    x[2] *= 1e15
    x[3, 1, 5] = float("nan")
    x[4, 2, 9] = float("inf")
    w = torch.randn(128, generator=g, device="cuda")
    y, = b.w2a8_qk_norm_rope(b.Heads([x], weight=[w]), 1e-6)
    want, tol = _reference(torch, x, w, 1e-6, None, None, 1.0, False, False)
    fine = torch.ones((6, 3), dtype=torch.bool, device="cuda")
    fine[3, 1] = fine[4, 2] = False
    assert bool(((y.double() - want).abs() <= tol)[fine].all())
    assert bool((y[0, 0] == 0).all()) and bool(y[3, 1].isnan().all())
    assert bool(y[4, 2, 9].isnan()) and bool((y[4, 2, :9] == 0).all())     # inf / inf, and finite / inf


def test_many_tokens_beyond_32_bits(gpu):
    """Offsets of the last tokens pass 2^31 elements."""
    torch, b = gpu
    M, H, D = 70000, 250, 128                           # 2.24e9 values
    x = torch.zeros((M, H, D), dtype=torch.bfloat16, device="cuda")
    x[M - 1, H - 1] = torch.arange(D, device="cuda").to(torch.bfloat16)
    pos = torch.zeros(M, dtype=torch.int32, device="cuda")
    pos[M - 1] = 3
    inv_freq, amp = b.w2a8_rope_frequencies(D, 10000.0)
    small, = b.w2a8_rope(b.Heads([x[M - 1:].clone()]), pos[M - 1:].clone(), inv_freq, amp)
    b.w2a8_rope(b.Heads([x], [x]), pos, inv_freq, amp)
    assert torch.equal(x[M - 1], small[0]) and not bool(x[:M - 1].any())
    del x
    torch.cuda.empty_cache()


def test_projection_adapters_norm_and_rotation_together(gpu):
    """The use: q|k|v of 2-bit matrices, adapters of each request, norms and rotation of q and k, on one stream; eager
    and as a replayed graph, whose every kernel starts while the one before it drains."""
    torch, b = gpu
    M, K, H, Hk, D, g, L, r = 12, 1024, 8, 2, 64, 64, 3, 8
    Ns = [H * D, Hk * D, Hk * D]
    gen = torch.Generator(device="cuda").manual_seed(21)
    codes = [torch.randint(0, 4, (n, K), generator=gen, device="cuda", dtype=torch.uint8) for n in Ns]
    scale = [0.02 * torch.exp(0.5 * torch.randn((n, K // g), generator=gen, device="cuda")) for n in Ns]
    y = [torch.empty((M, n), device="cuda") for n in Ns]
    grp = b.Group([b.w2_pack(c) for c in codes], scale, y)
    ws = b.new_workspace(b.w2a8_grouped_workspace_bytes(Ns, M, K, g))
    a, s_a = torch.empty((M, K), dtype=torch.int8, device="cuda"), torch.empty(M, device="cuda")
    A = [(torch.randn((L, r, K), generator=gen, device="cuda") / 32).to(torch.bfloat16) for _ in Ns]
    B = [(0.1 * torch.randn((L, n, r), generator=gen, device="cuda")).to(torch.bfloat16) for n in Ns]
    lora = b.LoraGroup(A, B)
    x = torch.randn((M, K), generator=gen, device="cuda").to(torch.bfloat16)
    adapter = (torch.arange(M, device="cuda") % 4 - 1).to(torch.int32)
    pos = torch.randint(0, 50000, (M,), generator=gen, device="cuda", dtype=torch.int32)
    w = [1 + 0.1 * torch.randn(D, generator=gen, device="cuda") for _ in range(2)]
    inv_freq, amp = b.w2a8_rope_frequencies(D, 500000.0, "llama3", factor=8.0, low=1.0, high=4.0, original_length=8192)
    heads = b.Heads([y[0].view(M, H, D), y[1].view(M, Hk, D)], weight=w, out_dtype=torch.bfloat16)

    def step():
        b.w2a8_linear_grouped(x, grp, g, ws, a=a, a_scale=s_a)
        b.w2a8_lora_grouped(x, adapter, lora, base=y, y=y)
        b.w2a8_qk_norm_rope(heads, 1e-6, pos, inv_freq, amp)

    step()
    torch.cuda.synchronize()
    eager = [t.clone() for t in heads.out] + [t.clone() for t in y]
    # the steps one by one, with nothing in flight
    base = [torch.empty_like(t) for t in y]
    b.w2a8_gemm_grouped(a, s_a, b.Group(grp.packed, grp.w_scale), g, ws, y=base)
    torch.cuda.synchronize()
    added = b.w2a8_lora_grouped(x, adapter, lora, base=base)
    torch.cuda.synchronize()
    for t, c, s, u in zip(y, codes, scale, added):
        assert bool(((t - u).abs() <= 2e-4 * u.abs().amax(1, keepdim=True)).all())
    for out, src, h, ww in zip(heads.out, y, (H, Hk), w):
        want, tol = _reference(torch, src.view(M, h, D), ww, 1e-6, pos, inv_freq, amp, False, True)
        assert bool(((out.double() - want).abs() <= tol).all())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for _ in range(3):
            step()
    for t in list(heads.out) + y:
        t.fill_(float("nan"))
    graph.replay()
    torch.cuda.synchronize()
    assert b.w2a8_workspace_status(ws) == 0
    for t, e in zip(list(heads.out) + y, eager):
        assert torch.equal(t, e)
