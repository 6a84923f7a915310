"""Infinite values among the adapters' weights (w2a8_lora_grouped): the formula's infinity or NaN, and nothing of it in other
channels, tokens or adapters.  h is cut into bf16 terms inside; whichever of them are zero, 0 * inf of a term must not show."""
import pytest

from test_gpu_lora import gpu                                        # noqa: F401

pytestmark = pytest.mark.gpu
INF = float("inf")


def _want(torch, x, adapter, A, B, rank, scale, base):
    """The formula in 64 bits, product by product."""
    y = base.double().clone()
    for m, a in enumerate(adapter.tolist()):
        if 0 <= a < A.shape[0] and rank[a] > 0:
            r = int(rank[a])
            h = (x[m].double()[None] * A[a, :r].double()).sum(1) * float(scale[a])
            y[m] += (h[None] * B[a, :, :r].double()).sum(1)
    return y


def _same(torch, got, want):
    """Equal, NaN in the same places."""
    got = got.double()
    return torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(nan=0.0, posinf=INF, neginf=-INF),
                                                                  want.nan_to_num(nan=0.0, posinf=INF, neginf=-INF))


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("h", [1.0, -3.0, 1.0 + 2.0 ** -12, 1.0 + 2.0 ** -20, 2.0 ** -100, 0.0, INF])
def test_one_rank(gpu, h, bf16):                                     # noqa: F811
    """h that one term holds, that two and that three terms hold; nothing and infinity.  x and A give h exactly."""
    torch, b = gpu
    K, N = 64, 32
    x = torch.zeros((1, K), dtype=torch.bfloat16, device="cuda")
    A = torch.zeros((1, 8, K), dtype=torch.bfloat16, device="cuda")
    high = h if h in (0.0, INF) else float(torch.tensor(h).bfloat16())
    x[0, 0], x[0, 1] = high, h - high if h != INF else 0.0
    A[0, :, :2] = 1
    B = torch.ones((1, N, 8), dtype=torch.bfloat16, device="cuda")
    B[0, 3, 0], B[0, 8, 0], B[0, 31, 0] = INF, -INF, INF
    rank = torch.tensor([1], dtype=torch.int32, device="cuda")
    owner = torch.zeros(1, dtype=torch.int32, device="cuda")
    y, = b.w2a8_lora_grouped(x, owner, b.LoraGroup([A], [B], rank=rank), out_dtype=torch.bfloat16 if bf16 else torch.float32)
    sign = 1.0 if h >= 0 else -1.0
    want = torch.full((N,), h, dtype=torch.float64, device="cuda")
    for n, w in ((3, INF), (8, -INF), (31, INF)):
        want[n] = sign * w if h != 0 else float("nan")
    if h != INF:                             # h is a multiple of 2^-12 or 2^-20 below 4: fp32 holds it
        assert float(torch.tensor(h)) == h
    assert _same(torch, y[0], want.to(y.dtype).double())


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("M,Ns,K,L,rank_max,tile", [(1, (48,), 64, 1, 8, 16), (40, (528, 16), 192, 3, 16, 16), (37, (272,), 128, 2, 64, 16),
                                                    (9, (144,), 64, 1, 128, 16), (150, (400, 32), 192, 3, 16, 64), (130, (272,), 64, 2, 32, 64),
                                                    (70, (144,), 128, 1, 64, 64), (90, (80,), 64, 2, 128, 64)])
def test_batches(gpu, monkeypatch, M, Ns, K, L, rank_max, tile, in_place, bf16):       # noqa: F811
    """Integers, so that finite results are exact, with infinite weights of both signs here and there (in one channel both
    signs), a last infinite one behind the adapter's rank, and h of zero and of infinity among the tokens."""
    torch, b = gpu
    monkeypatch.setenv("W2A8_LORA_TILE", str(tile))
    g = torch.Generator(device="cuda").manual_seed(M + rank_max)
    ri = lambda lo, hi, *s: torch.randint(lo, hi + 1, s, generator=g, device="cuda")
    dtype = torch.bfloat16 if bf16 else torch.float32
    x = ri(-3, 3, M, K).to(torch.bfloat16)
    A = [ri(-1, 1, L, rank_max, K).to(torch.bfloat16) for _ in Ns]
    B = [ri(-3, 3, L, n, rank_max).to(torch.bfloat16) for n in Ns]
    base = [ri(-200, 200, M, n).to(dtype) for n in Ns]
    rank = torch.tensor([max(1, rank_max - 3 * i) for i in range(L)], dtype=torch.int32, device="cuda")
    scale = torch.tensor([0.5, 1.0, 2.0], device="cuda")[:L].contiguous()
    owner = (torch.arange(M, device="cuda") % (L + 1) - 1 if M > 1 else torch.zeros(1, device="cuda")).to(torch.int32)
    for t in A:
        t[..., 0] = 0                        # h does not see x[:, 0] ...
        t[0, 0, 0] = 1                       # ... but for the first rank of adapter 0
    x[M // 2] = 0                            # h = 0
    x[M - 1, 0] = INF
    for t in A:
        t[0, 1:, 0] = 1                      # infinite h in all ranks of adapter 0, 0 * inf = NaN in those of others
    finite = [t.clone() for t in B]
    for t, n in zip(B, Ns):
        r = int(rank[0])
        t[0, 5 % n, 0], t[0, (n - 1), r - 1], t[0, n // 2, r // 2] = INF, -INF, INF
        if r > 1:
            t[0, 2, 0], t[0, 2, 1] = INF, -INF
        t[L - 1, n // 3, 0] = -INF
        if int(rank[L - 1]) < rank_max:
            t[L - 1, 1, rank_max - 1] = INF  # behind the rank: not used
    run = lambda w: b.w2a8_lora_grouped(x, owner, b.LoraGroup(A, w, rank=rank, scale=scale),
                                        **(lambda c: dict(base=c, y=c if in_place else None))([t.clone() for t in base]))
    got, without = run(B), run(finite)
    for y, y0, a_, b_, f_, c in zip(got, without, A, B, finite, base):
        want = _want(torch, x, owner, a_, b_, rank, scale, c).to(dtype).double()
        assert _same(torch, y, want)
        # channels that no infinite weight of the token's adapter touches have the bits that they have without
        for a in range(L):
            rows = torch.nonzero(owner == a)[:, 0]
            plain = (b_[a, :, :int(rank[a])] == f_[a, :, :int(rank[a])]).all(1)
            u, v = y[rows][:, plain], y0[rows][:, plain]
            assert torch.equal(u.isnan(), v.isnan()) and torch.equal(u.nan_to_num(), v.nan_to_num())
        none = owner < 0
        assert torch.equal(y[none], c[none])
