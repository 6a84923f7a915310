"""The operators around the 2-bit projections, as timed cases: low-rank adapters of many requests beside a
shared projection, rotary positions, and the norms of queries and keys with the rotation in the same pass.

A case is a plain dict.
  op "lora":  y[i] = base[i] + scale * (x A[i]^T) B[i]^T with the adapter of each token's request
     K, N0 .. N3 (0: no such matrix)   the matrices that share x;  M tokens of `requests` requests
     adapters, rank    resident adapters and the rank that their storage is laid out for;  ragged: ranks of
                       rank, rank/2, rank/4 and rank - 3 in turn, instead of `rank` for all
     bare              every so manyth request has no adapter (0: none)
     bf16              base and y are bf16 instead of fp32
  op "rope" and "qk": rotary positions on `heads` query and `kv` key heads of `dim` values, after a norm of each
     head for "qk"
     rot, interleaved  values of a head that are rotated, and how they are paired
     scaling           "none", "linear", "llama3" or "yarn"
     packed            q and k are column ranges of one q|k|v result, instead of results of their own
     src, dst          types of the projection's result and of the rotated heads: "fp32" or "bf16"

Every pass reads inputs that it leaves as they were, so that it can be called again.
"""
import math

import torch

own = False

_TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


# ---- the cases ----------------------------------------------------------------------------------------------------
def _lora(name, K, Ns, M, requests, adapters, rank, ragged=False, bare=0, bf16=False):
    Ns = list(Ns) + [0] * (4 - len(Ns))
    return dict(name=name, op="lora", K=K, N0=Ns[0], N1=Ns[1], N2=Ns[2], N3=Ns[3], M=M, requests=requests,
                adapters=adapters, rank=rank, ragged=ragged, bare=bare, bf16=bf16)


def _heads(name, op, M, heads, kv, dim, rot, interleaved=False, scaling="none", packed=False, src="fp32", dst="bf16"):
    return dict(name=name, op=op, M=M, heads=heads, kv=kv, dim=dim, rot=rot, interleaved=interleaved,
                scaling=scaling, packed=packed, src=src, dst=dst)


def listed():
    return [
        # one stream of one adapted model: q|k|v of a decode step, latency only
        _lora("lora_qkv_8b_m1", 4096, (4096, 1024, 1024), 1, 1, 4, 16),
        # a decode batch of 32 streams with 32 adapters of several ranks, some streams without one
        _lora("lora_gateup_8b_m32", 4096, (14336, 14336), 32, 32, 32, 64, ragged=True, bare=8),
        # a decode batch through the longest rows, bf16 results, four adapters shared by all streams
        _lora("lora_down_70b_m64", 28672, (8192,), 64, 64, 4, 32, bf16=True),
        # chunks of seven prompts, ragged
        _lora("lora_qkv_70b_m500", 8192, (8192, 1024, 1024), 500, 7, 7, 128, ragged=True),
        # the largest prefill of the benchmark with the prompts of 16 requests
        _lora("lora_gateup_8b_m8192", 4096, (14336, 14336), 8192, 16, 16, 64),
        # one decode step of one stream
        _heads("rope_8b_m1", "rope", 1, 32, 8, 128, 128, scaling="llama3"),
        # a ragged batch, pairs of neighbours, a quarter of the head unrotated, rows of a wide projection
        _heads("rope_m777_interleaved", "rope", 777, 32, 8, 64, 48, interleaved=True, packed=True, src="bf16"),
        # a long prompt of the larger model, far positions
        _heads("rope_70b_m8192", "rope", 8192, 64, 8, 128, 128, scaling="yarn"),
        # a decode batch with norms
        _heads("qk_8b_m16", "qk", 16, 32, 8, 128, 128),
        # heads whose size is no power of two, kept in fp32
        _heads("qk_m333_dim80", "qk", 333, 20, 5, 80, 32, scaling="linear", packed=True, dst="fp32"),
        # a long prompt of the larger model with norms, bf16 on both sides
        _heads("qk_70b_m8192", "qk", 8192, 64, 8, 128, 128, scaling="yarn", src="bf16"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


# (K, Ns) of linears that share their activations: layers of the benchmark and the paper's small shapes
_GROUPS = [(4096, (4096, 1024, 1024)), (4096, (4096,)), (4096, (14336, 14336)), (14336, (4096,)),
           (8192, (8192, 1024, 1024)), (8192, (28672, 28672)), (28672, (8192,)), (1600, (1600,)),
           (2048, (2048, 2048, 2048)), (2560, (3840,))]


def draw(rng):
    if rng.random() < 0.5:
        K, Ns = rng.choice(_GROUPS)
        rank = rng.choice([8, 16, 32, 64, 128])
        one = 2 * rank * (K * len(Ns) + sum(Ns))                       # bytes of an adapter
        adapters = _log_int(rng, 1, min(64, 500_000_000 // one))
        M = _log_int(rng, 1, min(8192, (1_900_000_000 - adapters * one) // (8 * sum(Ns) + 2 * K)))
        requests = M if M <= 64 else _log_int(rng, 1, 64)
        if M > 2048:
            rank = min(rank, 64)
        c = _lora("", K, Ns, M, requests, adapters, rank, rng.random() < 0.5, rng.choice([0, 0, 3, 8]),
                  rng.random() < 0.4)
    else:
        dim = rng.choice([64, 80, 96, 128, 128, 128, 256])
        heads, kv = rng.choice([(32, 8), (64, 8), (16, 16), (20, 5), (8, 1)])
        rot = rng.choice([dim, dim, dim // 2, dim // 4 * 3])
        most = min(8192, 8192 * 72 * 128 // ((heads + kv) * dim))
        c = _heads("", rng.choice(["rope", "qk"]), _log_int(rng, 1, most), heads, kv, dim, rot, rng.random() < 0.4,
                   rng.choice(["none", "linear", "llama3", "yarn"]), rng.random() < 0.4, rng.choice(["fp32", "bf16"]),
                   rng.choice(["fp32", "bf16", "bf16"]))
    del c["name"]
    return c


def _Ns(case):
    return [case[k] for k in ("N0", "N1", "N2", "N3") if case[k]]


def _used(case):
    """Adapters that the batch uses: one for each request in turn, for the requests that have one."""
    with_one = [j for j in range(case["requests"]) if not (case["bare"] and j % case["bare"] == case["bare"] - 1)]
    return len({j % case["adapters"] for j in with_one})


def _rank(case, order):
    """Rank of the adapter that is the `order`th to be dealt to requests."""
    r = case["rank"]
    return (r, max(r // 2, 1), max(r // 4, 1), max(r - 3, 1))[order % 4] if case["ragged"] else r


def work(case):
    M = case["M"]
    if case["op"] == "lora":
        K, Ns, e = case["K"], _Ns(case), 2 if case["bf16"] else 4
        ranks = [_rank(case, j) for j in range(_used(case))]
        nbytes = 2 * M * K + 4 * M + sum(2 * M * n * e for n in Ns) + sum(2 * r * (K + n) for r in ranks for n in Ns)
        mean = sum(ranks) / max(1, len(ranks))
        return {"bytes": nbytes, "flops": sum(2 * M * mean * (K + n) for n in Ns)}
    values = M * (case["heads"] + case["kv"]) * case["dim"]
    nbytes = values * sum(_TYPES[case[k]].itemsize for k in ("src", "dst")) + 4 * M + 4 * case["rot"]
    return {"bytes": nbytes, "flops": values * (7 if case["op"] == "qk" else 3)}


# ---- what a user's program has in hand -------------------------------------------------------------------------------
class _State:
    pass


def _ragged(g, M, requests):
    """Lengths of `requests` requests that add up to M, none empty."""
    if requests >= M:
        return torch.ones(M, dtype=torch.int64)
    w = torch.rand(requests, generator=g, device="cuda").cpu().double() + 0.05
    n = 1 + torch.floor(w / w.sum() * (M - requests)).to(torch.int64)
    n[-1] += M - int(n.sum())
    return n


def _inv_freq(case):
    """(radians per position [rot / 2] in 64 bits, amplitude) of the case's scaling."""
    rot, base, factor = case["rot"], 500000.0, 8.0
    p = torch.arange(rot // 2, dtype=torch.float64, device="cuda")
    f = base ** (-2.0 * p / rot)
    if case["scaling"] == "linear":
        return f / factor, 1.0
    if case["scaling"] == "llama3":
        turns = 8192 * f / (2 * math.pi)                       # full turns within the trained length
        mix = ((turns - 1.0) / (4.0 - 1.0)).clamp(0, 1)        # below 1: interpolated, above 4: left as it was
        return f * (mix + (1 - mix) / factor), 1.0
    if case["scaling"] == "yarn":
        pair = lambda turns: rot * math.log(8192 / (turns * 2 * math.pi)) / (2 * math.log(base))
        lo, hi = max(math.floor(pair(32.0)), 0), min(math.ceil(pair(1.0)), rot - 1)
        ramp = ((p - lo) / max(hi - lo, 1e-3)).clamp(0, 1)     # 0: left as it was, 1: interpolated
        return f * (1 - ramp) + f / factor * ramp, 0.1 * math.log(factor) + 1.0
    return f, 1.0


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    M = case["M"]
    s = _State()
    s.case = case

    def randn(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    def whole(high, n):
        return torch.randint(0, high, (n,), generator=g, device="cuda", dtype=torch.int64)

    if case["op"] == "lora":
        K, Ns, L, r = case["K"], _Ns(case), case["adapters"], case["rank"]
        n = _ragged(g, M, case["requests"])
        deal = torch.randperm(L, generator=g, device="cuda").cpu()           # who has which slot of the pool
        rank = torch.full((L,), r, dtype=torch.int32)
        for order in range(L):
            rank[deal[order]] = _rank(case, order)
        owner = torch.tensor([-1 if case["bare"] and j % case["bare"] == case["bare"] - 1 else int(deal[j % L])
                              for j in range(len(n))])
        s.adapter = torch.repeat_interleave(owner, n).to(torch.int32).cuda()
        s.rank = rank.cuda()
        s.scale = 0.5 + 1.5 * torch.rand(L, generator=g, device="cuda")
        s.x = randn(M, K).to(torch.bfloat16)
        s.A = [(randn(L, r, K) / math.sqrt(K)).to(torch.bfloat16) for _ in Ns]
        s.B = [(0.03 * randn(L, nn, r)).to(torch.bfloat16) for nn in Ns]
        s.base = [randn(M, nn).to(torch.bfloat16 if case["bf16"] else torch.float32) for nn in Ns]
        if own:
            from paper_2508_06753_b200 import binding as b
            s.lora = b.LoraGroup(s.A, s.B, rank=s.rank, scale=s.scale)
            s.y = [torch.zeros_like(t) for t in s.base]
        return s

    H, Hk, D = case["heads"], case["kv"], case["dim"]
    src, dst = _TYPES[case["src"]], _TYPES[case["dst"]]
    if case["packed"]:
        rows = (2.0 * randn(M, H + 2 * Hk, D)).to(src)
        s.x = [rows[:, :H], rows[:, H:H + Hk]]
    else:
        s.x = [(2.0 * randn(M, h, D)).to(src) for h in (H, Hk)]
    s.weight = [1.0 + 0.2 * randn(D) for _ in range(2)]
    s.eps = 1e-6
    # every request goes on from a position of its own, up to 128 thousand
    n = _ragged(g, M, min(M, 16))
    first = whole(131072 - M, len(n)).cpu()
    at = torch.arange(M) - torch.repeat_interleave(torch.cumsum(n, 0) - n, n)
    s.pos = (at + torch.repeat_interleave(first, n)).to(torch.int32).cuda()
    s.inv_freq, s.amplitude = _inv_freq(case)
    if own:
        from paper_2508_06753_b200 import binding as b
        s.out = [torch.zeros((M, h, D), dtype=dst, device="cuda") for h in (H, Hk)]
        s.grp = b.Heads(s.x, s.out, weight=s.weight if case["op"] == "qk" else None)
    return s


# ---- one pass ---------------------------------------------------------------------------------------------------------
def _tiles(adapter, L, p):
    """Tokens in tiles of up to p of one adapter: (adapter of each tile, tile and place of each token)."""
    M = adapter.shape[0]
    a = torch.where(adapter < 0, L, adapter).long()
    order = torch.argsort(a, stable=True)
    count = torch.bincount(a, minlength=L + 1)
    rank = torch.empty_like(a)
    rank[order] = torch.arange(M, device=a.device) - (torch.cumsum(count, 0) - count)[a[order]]
    ahead = torch.cumsum((count + p - 1) // p, 0)               # tiles up to and with each adapter
    tiles = torch.arange(M // p + min(L + 1, M), device=a.device)
    of = torch.searchsorted(ahead, tiles, right=True)
    return torch.where(of < L, of, -1), ahead[a] - (count[a] + p - 1) // p + rank // p, rank % p


def _plain_lora(s):
    M, p = s.x.shape[0], 64
    if M <= 256:                    # a decode batch: every token is a tile of its own
        of, x = s.adapter.long(), s.x.float()[:, None]
        back = lambda d: d[:, 0]
    else:
        of, tile, place = _tiles(s.adapter, s.rank.shape[0], p)
        x = torch.zeros((of.shape[0], p, s.x.shape[1]), device=of.device)
        x[tile, place] = s.x.float()
        back = lambda d: d[tile, place]
    ad = of.clamp(min=0)
    live = (of >= 0)[:, None] & (torch.arange(s.A[0].shape[1], device=of.device) < s.rank[ad][:, None])
    gain = torch.where(live, s.scale[ad][:, None], 0.0)[:, None]
    return [(base.float() + back((x @ A[ad].float().mT * gain) @ B[ad].float().mT)).to(base.dtype)
            for A, B, base in zip(s.A, s.B, s.base)]


def _plain_heads(s):
    case, rot = s.case, s.case["rot"]
    angle = s.pos.double()[:, None, None] * s.inv_freq
    c, n = (angle.cos() * s.amplitude).float(), (angle.sin() * s.amplitude).float()

    def one(x, w):
        x = x.float()
        if case["op"] == "qk":
            x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + s.eps) * w
        head, rest = x[..., :rot], x[..., rot:]
        if case["interleaved"]:
            u, v = head[..., 0::2], head[..., 1::2]
            head = torch.stack([u * c - v * n, v * c + u * n], -1).flatten(-2)
        else:
            u, v = head[..., :rot // 2], head[..., rot // 2:]
            head = torch.cat([u * c - v * n, v * c + u * n], -1)
        return torch.cat([head, rest], -1).to(_TYPES[case["dst"]])

    return [one(x, w) for x, w in zip(s.x, s.weight)]


def run(s):
    op = s.case["op"]
    if not own:
        return _plain_lora(s) if op == "lora" else _plain_heads(s)
    from paper_2508_06753_b200 import binding as b
    if op == "lora":
        return b.w2a8_lora_grouped(s.x, s.adapter, s.lora, base=s.base, y=s.y)
    if op == "rope":
        return b.w2a8_rope(s.grp, s.pos, s.inv_freq, s.amplitude, interleaved=s.case["interleaved"])
    return b.w2a8_qk_norm_rope(s.grp, s.eps, s.pos, s.inv_freq, s.amplitude, interleaved=s.case["interleaved"])


# ---- the definition in 64 bits ------------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    out = []
    if case["op"] == "lora":
        owner = s.adapter.tolist()
        for A, B, base in zip(s.A, s.B, s.base):
            y = base.double()
            for a in sorted(set(owner) - {-1}):
                rows = torch.nonzero(s.adapter == a)[:, 0]
                r = int(s.rank[a])
                h = torch.einsum("mk,rk->mr", s.x[rows].double(), A[a, :r].double())
                y[rows] += float(s.scale[a]) * torch.einsum("mr,nr->mn", h, B[a, :, :r].double())
            out.append(y)
        return out
    rot = case["rot"]
    for x, w in zip(s.x, s.weight):
        z = x.double().clone()
        if case["op"] == "qk":
            z /= torch.sqrt((z * z).sum(-1) / case["dim"] + s.eps)[..., None]
            z *= w.double()
        # a pair is a complex number, and the rotation a product with another
        first = slice(0, rot, 2) if case["interleaved"] else slice(0, rot // 2)
        second = slice(1, rot, 2) if case["interleaved"] else slice(rot // 2, rot)
        turn = torch.polar(torch.full_like(s.inv_freq, s.amplitude).expand(case["M"], -1).contiguous(),
                           torch.outer(s.pos.double(), s.inv_freq))
        turned = torch.complex(z[..., first], z[..., second]) * turn[:, None]
        z[..., first], z[..., second] = turned.real, turned.imag
        out.append(z)
    return out
