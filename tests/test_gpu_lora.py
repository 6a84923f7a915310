"""Low-rank adapters beside the projections (w2a8_lora_grouped) against a plain 64-bit computation.

Integer inputs make every product and every partial sum an integer that fp32 holds exactly (and h one of 16 bits, which
the two bf16 terms of a bf16 result hold), so results have to be equal whatever the order of the sums: a wrong or missing
k, rank, channel or token cannot hide in a tolerance.  Real-valued inputs then check the accuracy.
"""
import itertools

import numpy as np
import pytest

from conftest import Guarded
from paper_2508_06753_b200 import synth

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2508_06753_b200 import binding, build
    build.build()
    binding.lib()
    return torch, binding


def _reference(torch, x, adapter, A, B, rank, scale, base):
    """y in 64 bits, one adapter at a time."""
    out = []
    for a_, b_, base_ in zip(A, B, base):
        y = base_.double().clone()
        for a in range(a_.shape[0]):
            rows = torch.nonzero(adapter == a)[:, 0]
            r = int(rank[a])
            if len(rows) and r:
                h = x[rows].double() @ a_[a, :r].double().T
                y[rows] += float(scale[a]) * (h @ b_[a, :, :r].double().T)
        out.append(y)
    return out


def _integers(torch, M, Ns, K, L, rank_max, seed, bf16=False, ranks=None, none=0.2):
    g = torch.Generator(device="cuda").manual_seed(seed)
    ri = lambda lo, hi, *s: torch.randint(lo, hi + 1, s, generator=g, device="cuda")
    p = dict(x=ri(-3, 3, M, K).to(torch.bfloat16), A=[ri(-1, 1, L, rank_max, K).to(torch.bfloat16) for _ in Ns],
             B=[ri(-3, 3, L, n, rank_max).to(torch.bfloat16) for n in Ns],
             base=[ri(-200, 200, M, n).to(torch.bfloat16 if bf16 else torch.float32) for n in Ns])
    adapter = ri(0, L - 1, M).to(torch.int32)
    adapter[torch.rand(M, generator=g, device="cuda") < none] = -1
    p["adapter"] = adapter
    if ranks is None:
        ranks = ri(0, rank_max, L)
        ranks[0] = rank_max
    else:
        ranks = torch.tensor([ranks[i % len(ranks)] for i in range(L)], device="cuda")
    p["rank"] = ranks.to(torch.int32)
    p["scale"] = torch.tensor([0.5, 1.0, 2.0], device="cuda")[torch.arange(L, device="cuda") % 3].contiguous()
    # what stands at ranks that an adapter does not have may be anything
    for a in range(L):
        r = int(p["rank"][a])
        for t in p["A"]:
            t[a, r:] = float("nan")
        for t in p["B"]:
            t[a, :, r:] = float("nan")
    return p


def _equal(torch, got, ref):
    for y, r in zip(got, ref):
        assert torch.equal(y, r.float().to(y.dtype))


# M, Ns, K, adapters, rank_max
SHAPES = [
    (1, (16,), 64, 1, 8), (1, (4096, 1024, 1024), 4096, 3, 16), (2, (48, 16), 448, 2, 24), (7, (272,), 1600, 5, 40),
    (16, (64, 64, 32, 16), 256, 1, 64), (17, (128,), 512, 1, 72), (33, (96, 48), 320, 2, 128), (64, (256,), 1024, 1, 32),
    (65, (112,), 192, 1, 16), (130, (64, 80), 704, 9, 64), (200, (32,), 128, 150, 56), (300, (48, 16), 64, 1024, 8),
    (1000, (64,), 256, 6, 120), (5, (16,), 28672, 2, 32), (4097, (16, 32), 64, 3, 16), (9000, (16,), 128, 40, 48),
]


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("M,Ns,K,L,rank_max", SHAPES)
def test_exact_on_integers(gpu, M, Ns, K, L, rank_max, bf16):
    torch, b = gpu
    p = _integers(torch, M, Ns, K, L, rank_max, seed=M + K + L, bf16=bf16)
    lora = b.LoraGroup(p["A"], p["B"], rank=p["rank"], scale=p["scale"])
    y = b.w2a8_lora_grouped(p["x"], p["adapter"], lora, base=p["base"])
    _equal(torch, y, _reference(torch, p["x"], p["adapter"], p["A"], p["B"], p["rank"], p["scale"], p["base"]))


@pytest.mark.parametrize("C", [1, 2, 3, 8])
@pytest.mark.parametrize("M,Ns,K,L,rank_max", [(40, (272, 64), 1088, 2, 32), (150, (96,), 64, 3, 128), (4200, (32,), 64, 5, 16)])
def test_forced_cluster_sizes(gpu, monkeypatch, C, M, Ns, K, L, rank_max):
    """Fewer units of K than CTAs or warps, fewer blocks of channels than CTAs, an odd cluster."""
    torch, b = gpu
    monkeypatch.setenv("W2A8_LORA_C", str(C))
    p = _integers(torch, M, Ns, K, L, rank_max, seed=C + M)
    lora = b.LoraGroup(p["A"], p["B"], rank=p["rank"], scale=p["scale"])
    y = b.w2a8_lora_grouped(p["x"], p["adapter"], lora, base=p["base"])
    _equal(torch, y, _reference(torch, p["x"], p["adapter"], p["A"], p["B"], p["rank"], p["scale"], p["base"]))


@pytest.mark.parametrize("ranks,rank_max", [([1], 8), ([7, 0, 3], 8), ([9, 15, 16, 17], 24), ([63, 64, 1], 64),
                                            ([65, 127, 128, 64], 128), ([5, 33, 40], 40)])
def test_ranks_that_end_inside_a_step(gpu, ranks, rank_max):
    torch, b = gpu
    p = _integers(torch, 50, (48, 32), 192, len(ranks), rank_max, seed=rank_max, ranks=ranks)
    lora = b.LoraGroup(p["A"], p["B"], rank=p["rank"], scale=p["scale"])
    y = b.w2a8_lora_grouped(p["x"], p["adapter"], lora, base=p["base"])
    _equal(torch, y, _reference(torch, p["x"], p["adapter"], p["A"], p["B"], p["rank"], p["scale"], p["base"]))


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("M", [1, 20, 300])
def test_in_place_and_without_a_base(gpu, M, bf16):
    """In place equals out of place; without a base y is the adapters' part; nothing outside y is written; rows of
    tokens without an adapter keep their bits (a NaN and a negative zero among them)."""
    torch, b = gpu
    Ns, K = (64, 16), 256
    p = _integers(torch, M, Ns, K, 3, 16, seed=M, bf16=bf16)
    p["adapter"][M // 2] = -7
    p["adapter"][0] = 3                       # behind the last adapter: none
    for t in p["base"]:
        t[M // 2, 0], t[M // 2, 1] = float("nan"), -0.0
    lora = b.LoraGroup(p["A"], p["B"], rank=p["rank"], scale=p["scale"])
    dtype = p["base"][0].dtype
    bits = torch.int16 if bf16 else torch.int32
    outs = [Guarded(torch, t.shape, dtype, fill=7.0) for t in p["base"]]
    y = b.w2a8_lora_grouped(p["x"], p["adapter"], lora, base=p["base"], y=[o.view for o in outs])
    inplace = [Guarded(torch, t.shape, dtype) for t in p["base"]]
    for o, t in zip(inplace, p["base"]):
        o.view.copy_(t)
    same = [o.view for o in inplace]
    b.w2a8_lora_grouped(p["x"], p["adapter"], lora, base=same, y=same)
    alone = b.w2a8_lora_grouped(p["x"], p["adapter"], lora, out_dtype=dtype)
    torch.cuda.synchronize()
    none = (p["adapter"] < 0) | (p["adapter"] >= 3)
    zero = [torch.zeros_like(t) for t in p["base"]]
    ref0 = _reference(torch, p["x"], p["adapter"], p["A"], p["B"], p["rank"], p["scale"], zero)
    for o, i, a, t, r0 in zip(outs, inplace, alone, p["base"], ref0):
        o.check(); i.check()
        assert torch.equal(o.view.view(bits), i.view.view(bits))
        assert torch.equal(o.view[none].view(bits), t[none].view(bits))
        assert torch.equal(a, r0.float().to(dtype)) and bool((a[none] == 0).all())


def test_no_rank_and_scale_arrays(gpu):
    torch, b = gpu
    p = _integers(torch, 30, (32,), 128, 4, 16, seed=5, ranks=[16])
    y = b.w2a8_lora_grouped(p["x"], p["adapter"], b.LoraGroup(p["A"], p["B"]), base=p["base"])
    one = torch.ones(4, device="cuda")
    _equal(torch, y, _reference(torch, p["x"], p["adapter"], p["A"], p["B"], p["rank"], one, p["base"]))


def test_ranks_outside_are_clamped(gpu):
    torch, b = gpu
    p = _integers(torch, 12, (32,), 128, 2, 8, seed=6, ranks=[8], none=0.0)
    wild = torch.tensor([1 << 30, -5], dtype=torch.int32, device="cuda")
    y = b.w2a8_lora_grouped(p["x"], p["adapter"], b.LoraGroup(p["A"], p["B"], rank=wild), base=p["base"])
    _equal(torch, y, _reference(torch, p["x"], p["adapter"], p["A"], p["B"], [8, 0], [1.0, 1.0], p["base"]))


def test_tokens_do_not_disturb_each_other(gpu):
    """A token's bits are the same alone, in a batch of its adapter, in any order, and beside a token of NaN."""
    torch, b = gpu
    g = torch.Generator(device="cuda").manual_seed(8)
    M, K, N, L, r = 77, 512, 96, 3, 24
    x = torch.randn((M, K), generator=g, device="cuda").to(torch.bfloat16)
    A = [(torch.randn((L, r, K), generator=g, device="cuda") / 22).to(torch.bfloat16)]
    B = [torch.randn((L, N, r), generator=g, device="cuda").to(torch.bfloat16)]
    base = [torch.randn((M, N), generator=g, device="cuda")]
    adapter = (torch.arange(M, device="cuda") % L).to(torch.int32)
    lora = b.LoraGroup(A, B)
    y, = b.w2a8_lora_grouped(x, adapter, lora, base=base)
    again, = b.w2a8_lora_grouped(x, adapter, lora, base=base)
    assert torch.equal(y, again)
    order = torch.randperm(M, generator=g, device="cuda")
    mixed, = b.w2a8_lora_grouped(x[order].contiguous(), adapter[order].contiguous(), lora, base=[base[0][order].contiguous()])
    assert torch.equal(mixed, y[order])
    bad = x.clone()
    bad[5], bad[40, 3] = float("nan"), float("inf")
    part, = b.w2a8_lora_grouped(bad, adapter, lora, base=base)
    rest = [m for m in range(M) if m not in (5, 40)]
    assert torch.equal(part[rest], y[rest])
    assert bool(part[5].isnan().all()) and not bool(part[40].isfinite().any())


def test_infinite_activation_follows_the_formula(gpu):
    """h = +-inf in one token: y is that infinity times B, not NaN (of the ranks that the adapter has not, nor of
    the terms that h is cut into)."""
    torch, b = gpu
    K, N, r = 64, 32, 5
    x = torch.zeros((1, K), dtype=torch.bfloat16, device="cuda")
    x[0, 9] = float("inf")
    A = torch.ones((1, 8, K), dtype=torch.bfloat16, device="cuda")
    B = torch.ones((1, N, 8), dtype=torch.bfloat16, device="cuda")
    B[0, 1::2] = -1
    rank = torch.tensor([r], dtype=torch.int32, device="cuda")
    y, = b.w2a8_lora_grouped(x, torch.zeros(1, dtype=torch.int32, device="cuda"), b.LoraGroup([A], [B], rank=rank))
    want = torch.full((1, N), float("inf"), device="cuda")
    want[0, 1::2] = -float("inf")
    assert torch.equal(y, want)


# Real values.  An mma.sync step adds 16 products to the accumulator; the hardware may truncate where it aligns, which
# is at most 2^-22 of the sum of magnitudes per step.  A value of h passes K / 16 such steps and at most 72 fp32 additions
# (8 warps, 8 CTAs, the warps' sums among them), h * scale one rounding; y passes 3 r / 16 steps (padded ranks: at most
# 24) and two roundings.  Result in bf16: h holds 16 bits (2^-16), and the result is rounded by at most 2^-8.
def _bound(torch, x, adapter, A, B, rank, scale, base, bf16):
    out = []
    for a_, b_, base_ in zip(A, B, base):
        y = base_.double().abs() * 2.0 ** -23
        for a in range(a_.shape[0]):
            rows = torch.nonzero(adapter == a)[:, 0]
            r = int(rank[a])
            K = x.shape[1]
            mag = x[rows].double().abs() @ a_[a, :r].double().abs().T
            h = (x[rows].double() @ a_[a, :r].double().T).abs()
            eh = mag * (K / 16 + 72) * 2.0 ** -22 + h * (2.0 ** -16 if bf16 else 2.0 ** -23)
            w = abs(float(scale[a])) * b_[a, :, :r].double().abs().T
            y[rows] += eh @ w + (h @ w) * 26 * 2.0 ** -22
        out.append(y)
    return out


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("M,Ns,K,L,r", [(1, (4096, 1024, 1024), 4096, 2, 16), (37, (1024, 512), 2048, 5, 64),
                                        (24, (256,), 14336, 3, 128), (500, (512,), 1024, 4, 32)])
def test_real_values(gpu, M, Ns, K, L, r, bf16):
    torch, b = gpu
    g = torch.Generator(device="cuda").manual_seed(M + r)
    rn = lambda *s: torch.randn(s, generator=g, device="cuda")
    x = rn(M, K).to(torch.bfloat16)
    A = [(rn(L, r, K) / K ** 0.5).to(torch.bfloat16) for _ in Ns]
    B = [(0.3 * rn(L, n, r)).to(torch.bfloat16) for n in Ns]
    base = [rn(M, n).to(torch.bfloat16 if bf16 else torch.float32) for n in Ns]
    adapter = torch.randint(0, L, (M,), generator=g, device="cuda", dtype=torch.int32)
    rank = torch.tensor([r - 3 * (i % 2) for i in range(L)], dtype=torch.int32, device="cuda")
    scale = 0.5 + torch.rand(L, generator=g, device="cuda")
    y = b.w2a8_lora_grouped(x, adapter, b.LoraGroup(A, B, rank=rank, scale=scale), base=base)
    ref = _reference(torch, x, adapter, A, B, rank, scale, base)
    for got, want, tol in zip(y, ref, _bound(torch, x, adapter, A, B, rank, scale, base, bf16)):
        tol = tol + (want.abs() + tol) * 2.0 ** -8 if bf16 else tol
        assert bool(((got.double() - want).abs() <= tol).all())
        if not bf16:                         # and no bits of h are lost on the way: far below the worst case on average
            assert float((got.double() - want).norm() / want.norm()) < 1e-6


def test_beside_the_grouped_linear(gpu, oracle):
    """The use: q|k|v from the 2-bit matrices, adapters added in place on the same activations, one stream, captured
    into a graph and replayed with other activations and other owners of the tokens."""
    torch, b = gpu
    M, K, Ns, g, L, r = 9, 1024, [256, 64, 64], 64, 3, 16
    mats = [synth.make_linear(60 + i, K, n, g) for i, n in enumerate(Ns)]
    dev = lambda v: torch.from_numpy(np.ascontiguousarray(v)).cuda()
    grp = b.Group([b.w2_pack(dev(c)) for c, _ in mats], [dev(s) for _, s in mats],
                  [torch.empty((M, n), device="cuda") for n in Ns])
    ws = b.new_workspace(b.w2a8_grouped_workspace_bytes(Ns, M, K, g))
    a, s_a = torch.empty((M, K), dtype=torch.int8, device="cuda"), torch.empty(M, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(4)
    A = [(torch.randn((L, r, K), generator=gen, device="cuda") / 32).to(torch.bfloat16) for _ in Ns]
    B = [(0.1 * torch.randn((L, n, r), generator=gen, device="cuda")).to(torch.bfloat16) for n in Ns]
    lora = b.LoraGroup(A, B)
    x = torch.empty((M, K), dtype=torch.bfloat16, device="cuda")
    adapter = torch.zeros(M, dtype=torch.int32, device="cuda")

    def step():
        b.w2a8_linear_grouped(x, grp, g, ws, a=a, a_scale=s_a)
        b.w2a8_lora_grouped(x, adapter, lora, base=grp.y, y=grp.y)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        x.zero_()
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for trial in range(3):
        bits = synth.activations_bf16(70 + trial, M, K)
        x.copy_(dev(bits.view(np.int16)).view(torch.bfloat16))
        adapter.copy_(torch.randint(-1, L, (M,), generator=gen, device="cuda", dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        assert b.w2a8_workspace_status(ws) == 0
        a_ref, s_ref = oracle.quantize(bits)
        base = [torch.from_numpy(oracle.gemm(a_ref, s_ref, c, s_w, g)).cuda() for c, s_w in mats]
        rank, one = [r] * L, [1.0] * L
        ref = _reference(torch, x, adapter, A, B, rank, one, base)
        tol = _bound(torch, x, adapter, A, B, rank, one, base, False)
        for got, want, t, b0 in zip(grp.y, ref, tol, base):
            # the projection's own tolerance is 1e-4 of its row
            assert bool(((got.double() - want).abs() <= t + 1e-4 * b0.abs().amax(1, keepdim=True)).all())


def test_two_streams_at_once(gpu):
    torch, b = gpu
    p = _integers(torch, 120, (256, 64), 512, 5, 32, seed=9)
    lora = b.LoraGroup(p["A"], p["B"], rank=p["rank"], scale=p["scale"])
    want = b.w2a8_lora_grouped(p["x"], p["adapter"], lora, base=p["base"])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [[torch.zeros_like(t) for t in p["base"]] for _ in streams]
    for _ in range(20):
        for s, o in zip(streams, outs):
            b.w2a8_lora_grouped(p["x"], p["adapter"], lora, base=p["base"], y=o, stream=s)
    torch.cuda.synchronize()
    for o in outs:
        assert all(torch.equal(u, v) for u, v in zip(o, want))


def test_offsets_beyond_32_bits(gpu):
    """y, A and B with more than 2^31 elements: the last rows are reached."""
    torch, b = gpu
    K, N, L, r = 64, 28672, 601, 128                      # B: 601 * 28672 * 128 = 2.2e9 values
    B = torch.zeros((L, N, r), dtype=torch.bfloat16, device="cuda")
    A = torch.zeros((L, r, K), dtype=torch.bfloat16, device="cuda")
    B[L - 1] = 1
    A[L - 1] = 1
    M = 76000                                              # y: 76000 * 28672 = 2.2e9 values
    x = torch.ones((M, K), dtype=torch.bfloat16, device="cuda")
    adapter = torch.full((M,), -1, dtype=torch.int32, device="cuda")
    adapter[M - 1] = L - 1
    adapter[7] = L - 1
    y = torch.zeros((M, N), dtype=torch.bfloat16, device="cuda")
    b.w2a8_lora_grouped(x, adapter, b.LoraGroup([A], [B]), base=[y], y=[y])
    assert bool((y[M - 1] == K * r).all()) and bool((y[7] == K * r).all())
    assert not bool(y[8:M - 1].any()) and not bool(y[:7].any())
    del x, y, A, B
    torch.cuda.empty_cache()
