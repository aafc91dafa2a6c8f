"""The quantized key/value cache against plain implementations in binary64: what is written (codes and scales bit for bit), what is
read back, and attention over it."""
from __future__ import annotations

import math

import pytest

ROUND = {"float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}         # half a step, relative


@pytest.fixture(scope="module")
def cq():
    import paper_2410_07505_amd as pkg
    return pkg


@pytest.fixture(scope="module")
def torch():
    import torch
    return torch


# ---- plain implementations ---------------------------------------------------------------------------------------

def row_codes(torch, x, col, alpha, bits):
    """(codes, row scales) of rows [...][heads][dim], binary64 with the definition's binary32 roundings."""
    q_max = 127 if bits == 8 else 7
    x = x.double()
    a = (x.abs().amax(-1).pow(alpha) / q_max).float()
    D = (a.double()[..., None] * col.double()).float().double()
    safe = torch.where(D == 0, torch.ones_like(D), D)
    q = torch.round((x / safe).float().double()).clamp(-q_max, q_max)
    return torch.where(D == 0, torch.zeros_like(q), q), a


def unpack(torch, codes, bits):
    if bits == 8:
        return codes.double()
    c = codes.to(torch.int64)
    return (((torch.stack((c % 16, c // 16), -1).flatten(-2)) ^ 8) - 8).double()


def places(torch, cache, name):
    """(codes [place][head][dim], scales [place][head], column factors) in binary64."""
    codes = unpack(torch, getattr(cache, name + "_codes"), cache.bits).transpose(1, 2).flatten(0, 1)
    scale = getattr(cache, name + "_scale").double().transpose(1, 2).flatten(0, 1)
    col = getattr(cache, name + "_col")
    return codes, scale, (col.double() if col is not None else torch.ones((cache.heads, cache.dim), dtype=torch.float64, device=codes.device))


def values(torch, cache, name, at):
    """The numbers that the places stand for, in binary32 as defined."""
    codes, scale, col = places(torch, cache, name)
    return (codes[at] * (scale[at][..., None] * col).float().double()).float().double()


def attention_oracle(torch, cache, Q, table, lengths, scale, max_length):
    """(out, tolerance) in binary64.

    A score is off by the query's fixed-point step (1.6e-5 of the largest |q b| of its row, times the magnitudes of the keys' codes)
    and a few binary32 roundings; weights are binary16 (half a step, and at worst 2^-39 of the largest scale's power of two where
    they are subnormal); sums over n positions are binary32; the result is rounded once."""
    B, S, HQ, D = Q.shape
    H, page = cache.heads, cache.page_size
    ck, ak, bk = places(torch, cache, "k")
    cv, av, bv = places(torch, cache, "v")
    out = torch.zeros((B, S, HQ, D), dtype=torch.float64, device=Q.device)
    tol = torch.zeros_like(out)
    for b in range(B):
        n = min(int(lengths[b]), max_length + S - 1)
        for s in range(S):
            m = max(0, min(int(lengths[b]) - (S - 1 - s), max_length))
            pos = torch.arange(m, device=Q.device)
            pages = table[b].long()[pos // page]
            ok = (pages >= 0) & (pages < cache.pages)
            at = (pages * page + pos % page)[ok]
            if at.numel() == 0:
                continue
            for h in range(H):
                g = slice(h * (HQ // H), (h + 1) * (HQ // H))
                q = Q[b, s, g].double() * bk[h]
                k = ck[at, h] * ak[at, h, None]
                v = cv[at, h] * av[at, h, None]
                z = scale * (q @ k.t())
                p = torch.softmax(z, -1)
                o = p @ v * bv[h]
                dz = (abs(scale) * 1.6e-5 * q.abs().amax(-1, keepdim=True) * k.abs().sum(-1) + 2.0 ** -21 * z.abs()).amax(-1, keepdim=True)
                size = p @ v.abs() * bv[h]
                n = at.numel()
                R = 2.0 * float(av[at, h].max())
                q_max = 127 if cache.bits == 8 else 7
                out[b, s, g] = o
                tol[b, s, g] = (torch.expm1(2 * dz) + 2.0 ** -11 + 2.0 ** -20 + n * 2.0 ** -24) * size + n * 2.0 ** -39 * R * q_max * bv[h] / torch.exp(z - z.amax(-1, keepdim=True)).sum(-1, keepdim=True)
    return out, tol


def check_attention(torch, cq, cache, Q, table, lengths, scale=None, max_length=None, **kw):
    out = cq.crossquant_cache_attention(cache, Q, table, lengths, scale=scale, max_length=max_length, **kw)
    assert out.dtype == Q.dtype and out.shape == Q.shape
    ref, tol = attention_oracle(torch, cache, Q, table, lengths, cache.dim ** -0.5 if scale is None else scale,
                                table.shape[1] * cache.page_size if max_length is None else max_length)
    kind = str(Q.dtype).split(".")[1]
    bad = ~((out.double() - ref).abs() <= ROUND[kind] * ref.abs() + (1 + 2.0 ** -8) * tol + (2.0 ** -25 if kind == "float16" else 0.0))
    assert not bad.any(), "%d outputs, the first at %s: %s, not %s" % (
        int(bad.sum()), bad.nonzero()[0].tolist(), out[bad][0].item(), ref[bad][0].item())
    return out


def make_cache(torch, cq, bits, pages, heads, page, dim, *, cols=True, alpha=0.3, seed=0, scale_spread=1.0, device="cuda"):
    g = torch.Generator().manual_seed(seed)
    args = []
    for n in range(2):
        if bits == 8:
            c = torch.randint(-127, 128, (pages, heads, page, dim), generator=g).to(torch.int8)
        else:
            c = torch.randint(-7, 8, (pages, heads, page, dim), generator=g) & 15
            c = (c[..., 0::2] | (c[..., 1::2] << 4)).to(torch.uint8)
        s = torch.exp(scale_spread * torch.randn((pages, heads, page), generator=g)) * (0.01 if bits == 8 else 0.2)
        args += [c.to(device), s.to(device)]
    col = [torch.exp(0.7 * torch.randn((heads, dim), generator=g)).to(device) if cols else None for _ in range(2)]
    return cq.crossquant_cache(*args, bits, alpha=alpha, k_col=col[0], v_col=col[1])


def make_table(torch, cache, lengths, seed=0, extra=2):
    """Disjoint pages in no order; -1 behind the last one."""
    need = [-(-n // cache.page_size) for n in lengths]
    ids = torch.randperm(cache.pages, generator=torch.Generator().manual_seed(seed)).to(torch.int32)
    table = torch.full((len(lengths), max(need + [0]) + extra), -1, dtype=torch.int32)
    used = 0
    for b, n in enumerate(need):
        table[b, :n] = ids[used:used + n]
        used += n
    return table.cuda(), torch.tensor(lengths, dtype=torch.int32).cuda()


def queries(torch, B, S, HQ, dim, kind, seed=0):
    g = torch.Generator().manual_seed(seed + 100)
    return torch.randn((B, S, HQ, dim), generator=g).to(getattr(torch, kind)).cuda()


# ---- write and read ------------------------------------------------------------------------------------------------

@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["float16", "bfloat16"])
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("T,heads,dim,page,alpha,cols", [(1, 1, 64, 16, 1.0, False), (37, 3, 64, 32, 0.15, True), (64, 8, 128, 16, 0.15, True),
                                                        (200, 2, 128, 64, 1.0, False), (33, 5, 256, 128, 0.6, True), (9, 1, 256, 16, 0.0, True),
                                                        (700, 4, 128, 256, 0.45, True)])
def test_write_and_read(cq, torch, T, heads, dim, page, alpha, cols, bits, kind):
    print("cache %d rows, %d heads of %d, %d bits" % (T, heads, dim, bits), flush=True)
    pages = T // page + 3
    cache = make_cache(torch, cq, bits, pages, heads, page, dim, cols=cols, alpha=alpha, seed=T)
    before = [t.clone() for t in (cache.k_codes, cache.k_scale, cache.v_codes, cache.v_scale)]
    g = torch.Generator().manual_seed(T)
    qkv = (torch.randn((T, 3 * heads, dim), generator=g) * 2).to(getattr(torch, kind)).cuda()      # K, V: slices of a fused projection
    K, V = qkv[:, heads:2 * heads], qkv[:, 2 * heads:]
    K[0, 0] = 0.0                                                              # a zero row
    slots = torch.randperm(pages * page, generator=g)[:T].to(torch.int32)
    if T > 4:
        slots[1], slots[2], slots[3] = -1, pages * page, -2 ** 31
        slots[4] = pages * page - 1 if not (slots == pages * page - 1).any() else slots[4]
    cq.crossquant_cache_write(cache, K, V, slots.cuda())
    live = (slots >= 0) & (slots < pages * page)
    at = slots[live].long()
    for n, X, codes0, scale0 in (("k", K, before[0], before[1]), ("v", V, before[2], before[3])):
        col = getattr(cache, n + "_col")
        q, a = row_codes(torch, X.cpu()[live], col.cpu() if cols else torch.ones((heads, dim)), alpha, bits)
        old = type("C", (), {"k_codes": codes0, "k_scale": scale0, "k_col": None, "bits": bits, "heads": heads, "dim": dim})
        codes, scale, _ = places(torch, old, "k")
        codes, scale = codes.cpu(), scale.cpu()
        codes[at], scale[at] = q, a.double()
        got_codes, got_scale, _ = places(torch, cache, n)
        assert torch.equal(got_scale.cpu(), scale)
        assert torch.equal(got_codes.cpu(), codes)                              # what was written, and all other places as they were
    # read: any order, a place twice, padding
    want = torch.cat([slots, slots.flip(0), torch.tensor([0, 0, -5, pages * page + 7], dtype=torch.int32)]).cuda()
    for dtype in (torch.float16, torch.bfloat16):
        got = cq.crossquant_cache_read(cache, want, dtype=dtype)
        ok = (want >= 0) & (want < pages * page)
        for n, t in zip("kv", got):
            ref = torch.zeros(t.shape, dtype=torch.float64, device="cuda")
            ref[ok] = values(torch, cache, n, want[ok].long())
            assert torch.equal(t, ref.to(dtype))                                # (binary32 values, rounded once)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["float16", "bfloat16"])
@pytest.mark.parametrize("bits", [8, 4])
def test_write_of_extreme_rows(cq, torch, bits, kind):
    dtype = getattr(torch, kind)
    cache = make_cache(torch, cq, bits, 2, 1, 16, 64, cols=True, alpha=0.15, seed=2)
    cache.k_col[0, :8] = 0.0                                                    # D = 0: code 0
    cache.k_col[0, 8:16] = 1e-6                                                 # clamped
    X = torch.randn((8, 1, 64), generator=torch.Generator().manual_seed(1)).to(dtype)
    X[1] = 0.0
    X[2] = torch.finfo(dtype).max if kind == "float16" else 1e30
    X[3] = torch.finfo(dtype).smallest_normal
    X[4] = 0.0
    X[4, 0, 20] = torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps
    X[5, 0, ::2] = -X[5, 0, 1::2]
    X[6] = 1.0
    slots = torch.arange(8, dtype=torch.int32) + 3
    Xg = X.cuda()
    cq.crossquant_cache_write(cache, Xg, Xg, slots.cuda())
    q, a = row_codes(torch, X, cache.k_col.cpu(), 0.15, bits)
    codes, scale, _ = places(torch, cache, "k")
    assert torch.equal(scale[3:11].cpu(), a.double()) and torch.equal(codes[3:11].cpu(), q)


@pytest.mark.gpu
@pytest.mark.parametrize("bits,kind", [(8, "float16"), (4, "bfloat16")])
@pytest.mark.parametrize("T,heads,dim,page", [(4101, 8, 128, 64), (2100, 33, 64, 16), (1030, 17, 256, 256), (8300, 8, 128, 1024)])
def test_write_and_read_of_many_rows(cq, torch, T, heads, dim, page, bits, kind):
    """Several rows a thread, with a last stretch that is not whole."""
    test_write_and_read(cq, torch, T, heads, dim, page, 0.3, True, bits, kind)


@pytest.mark.gpu
@pytest.mark.parametrize("T,heads,dim,page,bits,kind", [(4101, 32, 64, 64, 8, "bfloat16"), (4099, 17, 128, 64, 4, "float16"), (2051, 17, 256, 64, 8, "float16"),
                                                       (2060, 32, 128, 64, 4, "bfloat16"), (4200, 32, 64, 16, 4, "float16"), (2049, 17, 256, 32, 4, "bfloat16")])
def test_write_and_read_of_more_rows(cq, torch, T, heads, dim, page, bits, kind):
    test_write_and_read(cq, torch, T, heads, dim, page, 0.6, True, bits, kind)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [3, 2000])
@pytest.mark.parametrize("bits,kind", [(8, "float16"), (8, "bfloat16"), (4, "float16"), (4, "bfloat16")])
def test_write_of_quotients_near_ties(cq, torch, bits, kind, T):
    """Every code's quotient at a tie, and a step of the type beside it; negative, tiny and huge column factors."""
    heads, dim, page, dtype = 33, 64, 16, getattr(torch, kind)
    q_max = 127 if bits == 8 else 7
    cache = make_cache(torch, cq, bits, T // page + 1, heads, page, dim, alpha=1.0, seed=3)
    for col in (cache.k_col, cache.v_col):
        col.fill_(1.0)
        col[1] = 3.0
        col[2] = 1.0 / 3.0
        col[3, ::2] = -1.0
        col[4] = 2.0 ** -70
        col[5] = 2.0 ** 70
        col[6, 1::2] = 0.0
        col[7] = 2.0 ** -149
    g = torch.Generator().manual_seed(T + bits)
    half = torch.randint(-q_max, q_max, (T, heads, dim), generator=g).double() + 0.5
    X = (half * torch.tensor([1.0, 3.0, 1.0 / 3.0]).double().repeat(heads // 3)[:, None]).to(dtype)
    away = torch.randint(-1, 2, X.shape, generator=g).to(torch.int16)
    X = (X.view(torch.int16) + away).view(dtype)
    X[:, :, 7] = q_max                                         # the maximum of most rows: a = 1
    Xg = X.cuda()
    slots = torch.randperm(cache.pages * page, generator=g)[:T].to(torch.int32)
    cq.crossquant_cache_write(cache, Xg, Xg, slots.cuda())
    for n in "kv":
        q, a = row_codes(torch, X, cache.k_col.cpu(), 1.0, bits)
        codes, scale, _ = places(torch, cache, n)
        assert torch.equal(scale[slots.long()].cpu(), a.double()) and torch.equal(codes[slots.long()].cpu(), q)


@pytest.mark.gpu
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("T", [4, 2000])
def test_a_row_with_no_number_stands_for_none(cq, torch, T, value):
    heads, dim, page = 33, 64, 16
    cache = make_cache(torch, cq, 8, T // page + 1, heads, page, dim, alpha=0.3, seed=4)
    cache.k_col[2, 9] = 0.0
    X = torch.randn((T, heads, dim), generator=torch.Generator().manual_seed(6)).half()
    plain = X.clone()
    X[T // 2, 2, 11] = value
    slots = torch.arange(T, dtype=torch.int32).cuda()
    cq.crossquant_cache_write(cache, plain.cuda(), plain.cuda(), slots)
    want = [t.clone() for t in cq.crossquant_cache_read(cache, slots)]
    cq.crossquant_cache_write(cache, X.cuda(), X.cuda(), slots)
    for w, t in zip(want, cq.crossquant_cache_read(cache, slots)):
        assert not torch.isfinite(t[T // 2, 2]).any()
        t[T // 2, 2] = w[T // 2, 2]
        assert torch.equal(t, w)


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [8, 4])
def test_places_behind_four_gib(cq, torch, bits):
    """Codes and the elements behind them past 32-bit offsets: the last pages of a cache of over 2^32 bytes a side."""
    heads, page, dim = 8, 128, 256
    pages = (1 << 32) // (heads * page * dim * bits // 8) + 3
    row = dim * bits // 8
    codes = [torch.empty((pages, heads, page, row), dtype=torch.int8 if bits == 8 else torch.uint8, device="cuda") for _ in range(2)]
    scale = [torch.zeros((pages, heads, page), device="cuda") for _ in range(2)]
    cache = cq.crossquant_cache(codes[0], scale[0], codes[1], scale[1], bits)
    T = 3 * page
    slots = (torch.arange(T, dtype=torch.int32) + (pages - 3) * page).cuda()
    g = torch.Generator().manual_seed(8)
    K, V = (torch.randn((T, heads, dim), generator=g).half().cuda() for _ in range(2))
    cq.crossquant_cache_write(cache, K, V, slots)
    got = cq.crossquant_cache_read(cache, slots)
    for X, t in zip((K, V), got):
        q, a = row_codes(torch, X, torch.ones((heads, dim), device="cuda"), 1.0, bits)
        assert torch.equal(t, (q * a.double()[..., None]).float().half())
    small = cq.crossquant_cache(codes[0][-3:].clone(), scale[0][-3:].clone(), codes[1][-3:].clone(), scale[1][-3:].clone(), bits)
    Q = queries(torch, 1, 2, 16, dim, "float16")
    table = torch.tensor([[pages - 1, pages - 3, pages - 2]], dtype=torch.int32).cuda()
    lengths = torch.tensor([T - 5], dtype=torch.int32).cuda()
    out = cq.crossquant_cache_attention(cache, Q, table, lengths)
    assert torch.equal(out, check_attention(torch, cq, small, Q, table - (pages - 3), lengths))


# ---- attention -----------------------------------------------------------------------------------------------------

CASES = [  # lengths, S, heads, group, dim, page, max_length
    ([1], 1, 1, 1, 64, 16, None),
    ([0, 5, 1], 1, 2, 4, 64, 16, None),
    ([31, 32, 33, 63, 64, 65], 1, 2, 8, 128, 32, None),
    ([127, 128, 129, 200], 1, 3, 7, 128, 16, 200),
    ([500], 1, 8, 4, 128, 16, 500),
    ([3, 0, 2, 700], 4, 2, 2, 64, 64, None),               # fewer positions than tokens: rows that see nothing
    ([1000, 257], 5, 2, 8, 128, 64, None),                 # 40 rows: three row tiles
    ([700, 129, 1], 1, 1, 48, 128, 32, None),
    ([300, 40], 2, 2, 16, 128, 16, None),                  # 32 rows
    ([90, 1025, 640], 1, 4, 16, 256, 128, None),
    ([77, 300], 3, 1, 7, 256, 16, 300),
    ([4096, 1, 3000], 1, 2, 1, 64, 256, None),
    ([20000], 1, 1, 8, 128, 1024, None),
    ([9000, 2500, 1, 0], 2, 2, 4, 256, 64, 9000),
]


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["float16", "bfloat16"])
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_attention(cq, torch, case, bits, kind):
    lengths, S, heads, group, dim, page, max_length = CASES[case]
    print("attention %s" % (CASES[case],), flush=True)
    pages = sum(-(-n // page) for n in lengths) + 2
    cache = make_cache(torch, cq, bits, pages, heads, page, dim, cols=case % 3 != 1, seed=case)
    table, lens = make_table(torch, cache, lengths, seed=case)
    Q = queries(torch, len(lengths), S, heads * group, dim, kind, case) / (float(cache.k_col.mean()) if cache.k_col is not None else 1.0)
    out = check_attention(torch, cq, cache, Q, table, lens, max_length=max_length)
    assert torch.equal(out, cq.crossquant_cache_attention(cache, Q, table, lens, max_length=max_length))
    for b, n in enumerate(lengths):
        for s in range(S):
            if n - (S - 1 - s) <= 0:
                assert (out[b, s] == 0).all()


# many sequences: (B, longest, S, heads, group, dim, page, bits, kind)
@pytest.mark.gpu
@pytest.mark.parametrize("B,longest,S,heads,group,dim,page,bits,kind", [
    (300, 500, 1, 2, 2, 64, 16, 8, "float16"),
    (300, 1500, 1, 1, 2, 64, 16, 8, "float16"),                # more sequences than threads of a block, in pieces
    (270, 1300, 1, 1, 1, 256, 64, 4, "bfloat16"),
    (64, 1100, 1, 1, 3, 128, 16, 8, "float16"),                # as many as a wave's lanes, and one more
    (65, 1100, 1, 1, 3, 128, 16, 4, "float16"),
    (130, 2500, 1, 2, 5, 128, 64, 4, "bfloat16"),              # over 1000 rows, of several pieces
    (90, 1500, 1, 2, 7, 256, 32, 8, "bfloat16"),
    (70, 1200, 2, 2, 9, 64, 64, 4, "float16"),                 # the same, 18 rows a pair
    (900, 200, 1, 7, 1, 128, 16, 8, "float16"),                # a block a pair
    (600, 160, 1, 7, 1, 256, 32, 4, "float16"),
    (520, 300, 2, 4, 10, 64, 16, 8, "bfloat16"),
    (70, 2300, 1, 2, 7, 256, 32, 8, "bfloat16"),               # in pieces
    (40, 2400, 2, 4, 9, 64, 64, 4, "float16"),
    (200, 2100, 1, 2, 5, 128, 16, 8, "float16"),
    (64, 2000, 1, 2, 4, 128, 64, 8, "float16"),                # wide blocks
    (32, 1025, 1, 4, 4, 128, 16, 4, "bfloat16"),
    (64, 600, 2, 4, 10, 64, 16, 8, "float16"),
    (130, 1500, 1, 1, 1, 64, 32, 4, "bfloat16"),
    (50, 1700, 3, 5, 6, 256, 64, 8, "bfloat16"),
    (43, 1300, 1, 3, 17, 128, 32, 8, "bfloat16"),
    (20, 1900, 4, 8, 8, 256, 16, 4, "float16"),
])
def test_attention_of_many_sequences(cq, torch, B, longest, S, heads, group, dim, page, bits, kind):
    print("attention of %d sequences up to %d, %d x %d heads of %d" % (B, longest, heads, group, dim), flush=True)
    g = torch.Generator().manual_seed(B)
    lengths = torch.randint(0, longest + 1, (B,), generator=g).tolist()
    lengths[0], lengths[B // 2], lengths[-1] = longest, 0, longest
    cache = make_cache(torch, cq, bits, sum(-(-n // page) for n in lengths) + 1, heads, page, dim, seed=B)
    table, lens = make_table(torch, cache, lengths, seed=B)
    Q = queries(torch, B, S, heads * group, dim, kind, B) / float(cache.k_col.mean())
    out = check_attention(torch, cq, cache, Q, table, lens, max_length=longest)
    assert torch.equal(out, cq.crossquant_cache_attention(cache, Q, table, lens, max_length=longest))


@pytest.mark.gpu
@pytest.mark.parametrize("bits,heads,dim,group,kind", [(8, 8, 128, 4, "float16"), (8, 16, 64, 20, "bfloat16"), (8, 4, 256, 2, "bfloat16"),
                                                       (4, 8, 256, 3, "float16"), (4, 16, 128, 20, "bfloat16"), (4, 16, 64, 1, "float16")])
def test_attention_over_a_large_cache(cq, torch, bits, heads, dim, group, kind):
    """Calls that could read more than 128 MiB, as their max_length says."""
    page = 64
    pages = -(-(130 << 20) // (2 * heads * (dim * bits // 8 + 4) * page))
    lengths = [3000, 0, 1, 1700, 64, 129, 20, 2500, 333]
    cache = make_cache(torch, cq, bits, pages, heads, page, dim, seed=31)
    table, lens = make_table(torch, cache, lengths, seed=31, extra=-(-pages // len(lengths)))
    assert len(lengths) * table.shape[1] >= pages
    Q = queries(torch, len(lengths), 1, heads * group, dim, kind, 31) / float(cache.k_col.mean())
    out = check_attention(torch, cq, cache, Q, table, lens)
    assert torch.equal(out, cq.crossquant_cache_attention(cache, Q, table, lens))


@pytest.mark.gpu
def test_two_graphs_and_eager_calls_of_attention_at_once(cq, torch):
    """Two graphs of one cache, each with its own workspace, on streams of their own beside eager calls; lengths and table change
    between replays."""
    lengths = [3000, 700, 1]
    cache = make_cache(torch, cq, 4, 3 * 220, 2, 16, 128, seed=21)
    table, lens = make_table(torch, cache, [3200, 900, 100], seed=5)
    lens.copy_(torch.tensor(lengths))
    Qs = [queries(torch, 3, s, 8, 128, "float16", s) for s in (1, 2)]
    need = [cq.crossquant_cache_attention_workspace(cache, 3, s, 8, 3200) for s in (1, 2)]
    streams, graphs, outs, works = [torch.cuda.Stream() for _ in range(2)], [], [], []
    for Q, n, stream in zip(Qs, need, streams):
        out, work = torch.empty_like(Q), torch.empty(n, dtype=torch.uint8, device="cuda")
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            cq.crossquant_cache_attention(cache, Q, table, lens, max_length=3200, out=out, workspace=work)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            cq.crossquant_cache_attention(cache, Q, table, lens, max_length=3200, out=out, workspace=work)
        graphs.append(graph), outs.append(out), works.append(work)
    for turn in range(4):
        lens.add_(torch.tensor([40, 1, 7], dtype=torch.int32, device="cuda"))
        table[0, 5 + turn] = -1
        for out in outs:
            out.fill_(9.0)
        torch.cuda.synchronize()
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
        eager = [cq.crossquant_cache_attention(cache, Q, table, lens, max_length=3200) for Q in Qs]
        torch.cuda.synchronize()
        for out, e in zip(outs, eager):
            assert torch.equal(out, e)
    check_attention(torch, cq, cache, Qs[1], table, lens, max_length=3200)


@pytest.mark.gpu
@pytest.mark.parametrize("S,group,dim,bits,kind", [(70, 3, 128, 8, "float16"), (33, 5, 64, 4, "bfloat16"), (40, 2, 256, 4, "float16"), (300, 1, 64, 8, "bfloat16")])
def test_attention_of_a_chunk(cq, torch, S, group, dim, bits, kind):
    """Many tokens at once, most of them in row tiles that see only a part of the sequence, or nothing of it."""
    lengths = [S, S + 1500, 10, 0, S + 129]
    cache = make_cache(torch, cq, bits, sum(-(-n // 32) for n in lengths), 2, 32, dim, seed=S)
    table, lens = make_table(torch, cache, lengths, seed=S)
    Q = queries(torch, 5, 1, 2 * group, dim, kind, S).expand(5, S, 2 * group, dim) / float(cache.k_col.mean())
    check_attention(torch, cq, cache, Q, table, lens)
    one = queries(torch, 1, 1, 2 * group, dim, kind, S + 1)
    assert torch.equal(cq.crossquant_cache_attention(cache, one.expand(5, S, -1, -1), table, lens),
                       cq.crossquant_cache_attention(cache, one.expand(5, S, -1, -1).contiguous(), table, lens))


@pytest.mark.gpu
@pytest.mark.parametrize("longest", [100, 2000])
def test_attention_of_lengths_that_are_none(cq, torch, longest):
    """Negative lengths, the smallest among them, count as zero; neighbours are not touched by them."""
    cache = make_cache(torch, cq, 8, 300, 2, 16, 64, seed=22)
    table, lens = make_table(torch, cache, [longest, 50, 50, 50, longest], seed=22)
    lens[1:4] = torch.tensor([-2 ** 31, -1, -2 ** 31 + 2], dtype=torch.int32)
    Q = queries(torch, 5, 3, 4, 64, "float16")
    out = check_attention(torch, cq, cache, Q, table, lens)
    assert (out[1:4] == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("scale", [0.0, -0.05, 3.0])
def test_attention_scales(cq, torch, scale):
    """A flat, an inverted and a peaked softmax (scores of hundreds)."""
    cache = make_cache(torch, cq, 8, 12, 2, 64, 128, seed=4)
    table, lens = make_table(torch, cache, [300, 333])
    check_attention(torch, cq, cache, queries(torch, 2, 1, 8, 128, "float16"), table, lens, scale=scale)


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [8, 4])
def test_attention_with_scales_far_apart(cq, torch, bits):
    """Rows whose scales differ by ten powers of ten, zero rows, and a later row that outweighs all before it."""
    cache = make_cache(torch, cq, bits, 40, 1, 16, 128, seed=5, scale_spread=3.0)
    table, lens = make_table(torch, cache, [600])
    cache.v_scale[table[0, 3].item()] = 0.0
    cache.v_scale[table[0, 30].item(), 0, 5] = 1e5
    cache.k_scale[table[0, 7].item()] = 0.0
    check_attention(torch, cq, cache, queries(torch, 1, 1, 8, 128, "bfloat16"), table, lens, scale=0.002)


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("S,lengths", [(1, [45, 130, 1]), (3, [45, 260, 2])])
def test_attention_never_uses_what_it_does_not_see(cq, torch, bits, S, lengths):
    """NaN and infinite scales on unseen places of seen pages, on unseen pages, and wild page numbers behind the last visible position."""
    cache = make_cache(torch, cq, bits, 30, 2, 32, 128, seed=6)
    table, lens = make_table(torch, cache, lengths, extra=3)
    Q = queries(torch, len(lengths), S, 4, 128, "float16")
    want = check_attention(torch, cq, cache, Q, table, lens)
    seen = torch.zeros((30, 32), dtype=torch.bool)
    for b, n in enumerate(lengths):
        for p in range(n):
            seen[int(table[b, p // 32]), p % 32] = True
    hide = ~seen[:, None].expand(30, 2, 32).cuda()
    for t, v in ((cache.k_scale, float("nan")), (cache.v_scale, float("inf"))):
        t[hide] = v
    for i, v in enumerate([2 ** 31 - 1, -2 ** 31, 30]):
        table[:, -1 - i][table[:, -1 - i] == -1] = v
    assert torch.equal(cq.crossquant_cache_attention(cache, Q, table, lens), want)


@pytest.mark.gpu
def test_attention_of_early_tokens_is_free_of_later_ones(cq, torch):
    """Of drafted tokens each sees its own positions only: a NaN key or value of the last token stays out of the others' rows."""
    cache = make_cache(torch, cq, 8, 8, 1, 16, 64, seed=7)
    table, lens = make_table(torch, cache, [50])
    Q = queries(torch, 1, 4, 2, 64, "float16")
    want = check_attention(torch, cq, cache, Q, table, lens)
    for t in (cache.k_scale, cache.v_scale):
        t[table[0, 3].item(), 0, 1] = float("nan")
    out = cq.crossquant_cache_attention(cache, Q, table, lens)
    assert torch.equal(out[:, :3], want[:, :3]) and torch.isnan(out[:, 3]).all()


@pytest.mark.gpu
def test_attention_skips_pages_that_do_not_exist(cq, torch):
    cache = make_cache(torch, cq, 8, 10, 2, 16, 64, seed=8)
    table, lens = make_table(torch, cache, [100])
    for i, bad in ((0, -1), (3, 10), (4, 2 ** 30)):
        table[0, i] = bad
    check_attention(torch, cq, cache, queries(torch, 1, 2, 4, 64, "float16"), table, lens)
    table.fill_(-1)
    assert (cq.crossquant_cache_attention(cache, queries(torch, 1, 2, 4, 64, "float16"), table, lens) == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_a_query_that_is_no_number_spoils_its_own_row(cq, torch, value):
    cache = make_cache(torch, cq, 8, 8, 2, 16, 64, seed=9)
    table, lens = make_table(torch, cache, [50, 0])
    Q = queries(torch, 2, 1, 4, 64, "float16")
    want = check_attention(torch, cq, cache, Q, table, lens)
    Q[:, 0, 1, 5] = value
    out = cq.crossquant_cache_attention(cache, Q, table, lens)
    assert torch.isnan(out[0, 0, 1]).all() and (out[1] == 0).all()
    keep = [0, 2, 3]
    assert torch.equal(out[0, 0, keep], want[0, 0, keep])


@pytest.mark.gpu
def test_attention_of_zero_and_tiny_queries(cq, torch):
    cache = make_cache(torch, cq, 4, 8, 1, 16, 64, seed=9)
    table, lens = make_table(torch, cache, [90])
    Q = queries(torch, 1, 1, 3, 64, "bfloat16")
    Q[0, 0, 0] = 0.0
    Q[0, 0, 1] *= 2.0 ** -120                                # counts as zero: its scores are below 2^-100
    check_attention(torch, cq, cache, Q, table, lens)


@pytest.mark.gpu
def test_attention_with_strided_queries_and_buffers_given(cq, torch):
    cache = make_cache(torch, cq, 8, 40, 2, 16, 128, seed=10)
    table, lens = make_table(torch, cache, [500, 33])
    wide = queries(torch, 2, 3, 2 * 8 + 4, 128, "bfloat16")
    Q = wide[:, :2, 2:18]
    need = cq.crossquant_cache_attention_workspace(cache, 2, 2, 16, 544)
    assert need > 0
    out = torch.full((2, 2, 16, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    work = torch.full((need + 256,), 0xFF, dtype=torch.uint8, device="cuda")   # NaN patterns: need not be cleared
    got = check_attention(torch, cq, cache, Q, table, lens, max_length=544, out=out, workspace=work[:need])
    assert got is out and (work[need:] == 0xFF).all()
    assert torch.equal(out, cq.crossquant_cache_attention(cache, Q.contiguous(), table, lens, max_length=544))
    with pytest.raises(cq.CrossQuantError) as e:
        cq.crossquant_cache_attention(cache, Q, table, lens, max_length=544, workspace=work[:need - 16])
    assert e.value.status == -2


@pytest.mark.gpu
def test_attention_up_to_max_length(cq, torch):
    """Positions at and past max_length are not seen, whatever lengths says."""
    cache = make_cache(torch, cq, 8, 20, 1, 16, 64, seed=11)
    table, lens = make_table(torch, cache, [200])
    Q = queries(torch, 1, 2, 2, 64, "float16")
    check_attention(torch, cq, cache, Q, table, lens, max_length=100)
    assert torch.equal(cq.crossquant_cache_attention(cache, Q[:, 1:], table, lens, max_length=100),
                       cq.crossquant_cache_attention(cache, Q[:, 1:], table, torch.full_like(lens, 100)))


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [8, 4])
def test_a_step_of_a_layer(cq, torch, bits):
    """The calls together, as a serving program runs a layer: FP8 projection of the new tokens, keys and values into the cache,
    attention over it, FP8 projection of the result; eager and as one captured graph replayed for the tokens that follow.  Every
    stage is checked on what the stage before gave it."""
    import test_fp8
    B, width, heads, group, dim, page, past = 3, 256, 2, 2, 64, 16, [0, 40, 77]
    g = torch.Generator().manual_seed(12)
    HQ = heads * group
    w_in = cq.crossquant_weight_quantize_fp8((torch.randn((width, (HQ + 2 * heads) * dim), generator=g) * 0.05).half().cuda())
    w_out = cq.crossquant_weight_quantize_fp8((torch.randn((HQ * dim, width), generator=g) * 0.05).half().cuda())
    cache = make_cache(torch, cq, bits, 30, heads, page, dim, alpha=0.15, seed=13)
    table, lens = make_table(torch, cache, [n + 8 for n in past], seed=3)
    lens.copy_(torch.tensor(past))
    X = torch.zeros((B, width), dtype=torch.float16, device="cuda")
    slots = torch.zeros(B, dtype=torch.int32, device="cuda")

    def step():
        qx = cq.crossquant_quantize_fp8(X)
        qkv = cq.crossquant_fp8_linear(*qx, *w_in).view(B, HQ + 2 * heads, dim)
        cq.crossquant_cache_write(cache, qkv[:, HQ:HQ + heads], qkv[:, HQ + heads:], slots)
        att = cq.crossquant_cache_attention(cache, qkv[:, None, :HQ], table, lens)
        qa = cq.crossquant_quantize_fp8(att.view(B, HQ * dim))
        return qx, qkv, att, qa, cq.crossquant_fp8_linear(*qa, *w_out)

    def inputs(i):
        X.copy_(torch.randn((B, width), generator=g))
        lens.add_(1)
        pos = lens.long() - 1
        slots.copy_(table[torch.arange(B, device="cuda"), pos // page] * page + pos % page)

    def check(qx, qkv, att, qa, Y):
        for (q, s), x in ((qx, X), (qa, att.view(B, HQ * dim))):
            q_ref, s_ref = test_fp8.rows_oracle(torch, x.cpu())
            assert torch.equal(q.cpu().double(), q_ref) and torch.equal(s.cpu().double(), s_ref)
        for q, w, y in ((qx, w_in, qkv.view(B, -1)), (qa, w_out, Y)):
            ref, slack = test_fp8.linear_oracle(*q, *w)
            assert ((y.double() - ref).abs() <= test_fp8.tolerance(ref, slack, "float16")).all()
        for n, x in (("k", qkv[:, HQ:HQ + heads]), ("v", qkv[:, HQ + heads:])):
            q_ref, a_ref = row_codes(torch, x, getattr(cache, n + "_col"), 0.15, bits)
            codes, scale, _ = places(torch, cache, n)
            assert torch.equal(codes[slots.long()], q_ref) and torch.equal(scale[slots.long()], a_ref.double())
        ref, tol = attention_oracle(torch, cache, qkv[:, None, :HQ], table, lens, dim ** -0.5, table.shape[1] * page)
        assert ((att.double() - ref).abs() <= 2.0 ** -11 * ref.abs() + (1 + 2.0 ** -8) * tol + 2.0 ** -25).all()

    inputs(0)
    check(*step())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        results = step()
    for i in range(1, 5):
        inputs(i)
        graph.replay()
        torch.cuda.synchronize()
        check(*results)
        assert torch.equal(results[-1], step()[-1])


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["float16", "bfloat16"])
def test_the_calls_without_the_native_part(cq, torch, monkeypatch, kind):
    """The Python checks and ctypes make the same calls as the binding's native part: same outputs, new or into given buffers."""
    from paper_2410_07505_amd import binding
    assert binding._fast is not binding._NoFastcall
    dtype = getattr(torch, kind)
    g = torch.Generator().manual_seed(21)
    X = torch.randn((33, 300), generator=g).to(dtype).cuda()
    W = torch.randn((300, 70), generator=g).to(dtype).cuda()
    KV = torch.randn((20, 6, 64), generator=g).to(dtype).cuda()
    slots = torch.randperm(80, generator=g)[:20].to(torch.int32).cuda()
    Q = queries(torch, 2, 2, 4, 64, kind)

    def calls():
        q, xs = cq.crossquant_quantize_fp8(X)
        w, ws = cq.crossquant_weight_quantize_fp8(W)
        cache = make_cache(torch, cq, 8, 20, 2, 16, 64, seed=22)
        table, lens = make_table(torch, cache, [150, 31])
        cq.crossquant_cache_write(cache, KV[:, 2:4], KV[:, 4:], slots)
        out = [q.view(torch.uint8), xs, w.view(torch.uint8), ws, cq.crossquant_fp8_linear(q, xs, w, ws, dtype=dtype), cq.crossquant_fp8_linear(q, xs, w, ws),
               cache.k_codes, cache.v_scale, *cq.crossquant_cache_read(cache, slots), *cq.crossquant_cache_read(cache, slots, dtype=dtype),
               cq.crossquant_cache_attention(cache, Q, table, lens), cq.crossquant_cache_attention(cache, Q, table, lens, scale=1, max_length=140)]
        given = [torch.zeros_like(q), torch.zeros_like(xs), torch.zeros_like(w), torch.zeros_like(ws), torch.zeros_like(out[4]), torch.zeros_like(Q)]
        a = cq.crossquant_quantize_fp8(X, codes=given[0], scale=given[1])
        b = cq.crossquant_weight_quantize_fp8(W, qw=given[2], w_scale=given[3])
        c = cq.crossquant_fp8_linear(*a, *b, Y=given[4])
        d = cq.crossquant_cache_attention(cache, Q, table, lens, out=given[5])
        k, v = torch.zeros((20, 2, 64), dtype=dtype, device="cuda"), torch.zeros((20, 2, 64), dtype=dtype, device="cuda")
        e = cq.crossquant_cache_read(cache, slots, K=k, V=v)
        for x, y in zip((*a, *b, c, d, *e), (*given, k, v)):
            assert x is y
        return out + [t.view(torch.uint8) if t.dtype == torch.float8_e4m3fn else t for t in (*given, k, v)]

    native = calls()
    monkeypatch.setattr(binding, "_fast", binding._NoFastcall)
    for x, y in zip(native, calls()):
        assert x.dtype == y.dtype and torch.equal(x, y)


# ---- refusals (no GPU) -----------------------------------------------------------------------------------------------

P = 0x10000


def fields(**kw):
    f = dict(k_codes=P, v_codes=P, k_scale=P, v_scale=P, k_col=0, v_col=0, pages=4, page_size=16, heads=2, dim=64, bits=8, alpha=0.5)
    f.update(kw)
    return f


def descriptor(cq, **kw):
    import ctypes
    from paper_2410_07505_amd import binding
    return ctypes.byref(binding._CacheStruct(*fields(**kw).values()))


DESCRIPTOR_ERRORS = [(dict(k_codes=0), -1), (dict(v_codes=0), -1), (dict(k_scale=0), -1), (dict(v_scale=0), -1), (dict(pages=0), -2),
                     (dict(heads=0), -2), (dict(page_size=0), -2), (dict(dim=0), -2), (dict(pages=1 << 24, page_size=128), -2),
                     (dict(pages=1 << 20, heads=1 << 24, dim=256), -2), (dict(bits=5), -3), (dict(alpha=-0.1), -4), (dict(alpha=float("nan")), -4),
                     (dict(page_size=8), -6), (dict(page_size=48), -6), (dict(page_size=1 << 17), -6), (dict(dim=96), -6),
                     (dict(k_codes=P + 8), -5), (dict(v_scale=P + 4), -5), (dict(k_col=P + 8), -5)]


@pytest.mark.parametrize("change,status", DESCRIPTOR_ERRORS)
def test_descriptor_errors(cq, change, status):
    c = descriptor(cq, **change)
    assert cq.raw.crossquant_cache_write(c, P, 128, 64, P, 128, 64, 0, P, 4, None) == status
    assert cq.raw.crossquant_cache_read(c, P, 4, P, P, 0, None) == status
    assert cq.raw.crossquant_cache_attention_workspace(c, 1, 1, 2, 64) == -1
    assert cq.raw.crossquant_cache_attention(c, P, 128, 128, 64, 0, 1, 1, 2, P, 4, P, 64, 0.1, P, P, 1 << 30, None) == status


def test_write_and_read_argument_errors(cq):
    c = descriptor(cq)
    assert cq.raw.crossquant_cache_write(None, P, 128, 64, P, 128, 64, 0, P, 4, None) == -1

    def write(K=P, kt=128, kh=64, V=P, vt=128, vh=64, kind=0, slots=P, T=4):
        return cq.raw.crossquant_cache_write(c, K, kt, kh, V, vt, vh, kind, slots, T, None)
    assert write(K=0) == -1 and write(V=0) == -1 and write(slots=0) == -1
    assert write(T=0) == -2 and write(T=1 << 25) == -2 and write(kt=-8) == -2
    assert write(kind=2) == -9
    assert write(K=P + 8) == -5 and write(slots=P + 2) == -5 and write(kt=129) == -5 and write(vh=4) == -5

    def read(slots=P, T=4, K=P, V=P, kind=0):
        return cq.raw.crossquant_cache_read(c, slots, T, K, V, kind, None)
    assert read(slots=0) == -1 and read(K=0) == -1 and read(V=0) == -1
    assert read(T=0) == -2 and read(kind=7) == -9 and read(K=P + 8) == -5


def test_attention_argument_errors(cq):
    c = descriptor(cq)

    def call(Q=P, qb=128, qs=128, qh=64, kind=0, B=1, S=1, HQ=2, table=P, width=4, lengths=P, most=64, scale=0.1, out=P, work=P, have=1 << 30):
        return cq.raw.crossquant_cache_attention(c, Q, qb, qs, qh, kind, B, S, HQ, table, width, lengths, most, scale, out, work, have, None)
    for name in ("Q", "table", "lengths", "out"):
        assert call(**{name: 0}) == -1
    assert call(B=0) == -2 and call(S=0) == -2 and call(HQ=0) == -2 and call(HQ=3) == -2 and call(width=0) == -2
    assert call(most=0) == -2 and call(most=65) == -2 and call(S=1 << 23, HQ=4) == -2
    assert call(scale=float("nan")) == -2 and call(scale=float("inf")) == -2
    assert call(kind=2) == -9
    assert call(Q=P + 8) == -5 and call(out=P + 2) == -5 and call(work=P + 4) == -5 and call(qs=100) == -5
    # a sequence that several blocks share needs its workspace
    assert call(width=64, most=1024, work=0) == -1
    need = cq.raw.crossquant_cache_attention_workspace(c, 1, 1, 2, 1024)
    assert need > 0 and call(width=64, most=1024, have=need - 1) == -2
    assert cq.raw.crossquant_cache_attention_workspace(c, 1, 1, 2, 64) == 0
    assert cq.raw.crossquant_cache_attention_workspace(c, 1, 1, 3, 64) == -1


def test_wrappers_check_what_they_are_given(cq, torch):
    z = torch.zeros
    codes, scale = z((4, 2, 16, 64), dtype=torch.int8), z((4, 2, 16))
    with pytest.raises(ValueError, match="v_codes must have shape"):
        cq.crossquant_cache(codes, scale, codes[:3], scale, 8)
    with pytest.raises(TypeError, match="k_codes must have dtype"):
        cq.crossquant_cache(codes, scale, codes, scale, 4)
    with pytest.raises(ValueError, match="k_scale must have shape"):
        cq.crossquant_cache(codes, z((4, 16, 2)), codes, scale, 8)
    with pytest.raises(cq.CrossQuantError):
        cq.crossquant_cache(codes, scale, codes, scale, 6)
    with pytest.raises(cq.CrossQuantError):
        cq.crossquant_cache(codes, scale, codes, scale, 8, alpha=1.5)


def test_calls_check_what_they_are_given(cq, torch):
    """The checks that come before the device check, on CPU tensors."""
    z = torch.zeros
    codes, scale = z((4, 2, 16, 64), dtype=torch.int8), z((4, 2, 16))
    cache = cq.crossquant_cache(codes, scale, codes, scale, 8)
    K = z((5, 2, 64), dtype=torch.float16)
    slots = z(5, dtype=torch.int32)
    with pytest.raises(TypeError, match="slots"):
        cq.crossquant_cache_write(cache, K, K, z((5, 1), dtype=torch.int32))
    with pytest.raises(TypeError, match="slots must have dtype"):
        cq.crossquant_cache_write(cache, K, K, slots.long())
    with pytest.raises(ValueError, match="V must have shape"):
        cq.crossquant_cache_write(cache, K, K[:4], slots)
    with pytest.raises(TypeError, match="V must be a tensor of dtype"):
        cq.crossquant_cache_write(cache, K, K.bfloat16(), slots)
    with pytest.raises(TypeError, match="float16 or bfloat16"):
        cq.crossquant_cache_write(cache, K.float(), K.float(), slots)
    with pytest.raises(ValueError, match="unit stride"):
        cq.crossquant_cache_write(cache, z((5, 64, 2), dtype=torch.float16).transpose(1, 2), K, slots)
    with pytest.raises(ValueError, match="GPU"):
        cq.crossquant_cache_write(cache, K, K, slots)
    with pytest.raises(ValueError, match="K must have shape"):
        cq.crossquant_cache_read(cache, slots, K=K[:4])
    with pytest.raises(ValueError, match="GPU"):
        cq.crossquant_cache_read(cache, slots)
    Q, table, lens = z((3, 1, 4, 64), dtype=torch.float16), z((3, 2), dtype=torch.int32), z(3, dtype=torch.int32)
    for q in (z((3, 1, 3, 64), dtype=torch.float16), z((3, 1, 4, 128), dtype=torch.float16)):
        with pytest.raises(ValueError, match="Q must be"):
            cq.crossquant_cache_attention(cache, q, table, lens)
    with pytest.raises(ValueError, match="lengths must have shape"):
        cq.crossquant_cache_attention(cache, Q, table, lens[:2])
    with pytest.raises(ValueError, match="page_table must have shape"):
        cq.crossquant_cache_attention(cache, Q, table[:2], lens)
    with pytest.raises(TypeError, match="page_table must have dtype"):
        cq.crossquant_cache_attention(cache, Q, table.long(), lens)
    with pytest.raises(ValueError, match="GPU"):
        cq.crossquant_cache_attention(cache, Q, table, lens)
    with pytest.raises(TypeError, match="crossquant_cache"):
        cq.crossquant_cache_read(None, slots)


def test_the_longest_max_length(cq):
    c = descriptor(cq)
    assert cq.raw.crossquant_cache_attention_workspace(c, 1, 1, 2, (1 << 31) - 256) > 0
    assert cq.raw.crossquant_cache_attention_workspace(c, 1, 1, 2, (1 << 31) - 255) == -1


def test_a_cache_with_an_empty_axis_is_refused(cq, torch):
    for shape in ((0, 2, 16, 64), (4, 0, 16, 64), (4, 2, 0, 64), (4, 2, 16, 0)):
        codes, scale = torch.zeros(shape, dtype=torch.int8), torch.zeros(shape[:3])
        with pytest.raises(cq.CrossQuantError) as e:
            cq.crossquant_cache(codes, scale, codes, scale, 8)
        assert e.value.status == -2


def test_a_cache_keeps_its_tensors(cq, torch):
    codes, scale = torch.zeros((4, 2, 16, 64), dtype=torch.int8), torch.zeros((4, 2, 16))
    cache = cq.crossquant_cache(codes, scale, codes, scale, 8)
    for name in ("k_codes", "v_scale", "k_col", "alpha", "_struct", "other"):
        with pytest.raises(AttributeError):
            setattr(cache, name, codes)
        with pytest.raises(AttributeError):
            delattr(cache, name)
    assert cache.k_codes is codes and (cache.pages, cache.heads, cache.page_size, cache.dim) == (4, 2, 16, 64)


@pytest.mark.gpu
def test_a_cache_with_an_empty_axis_is_refused_on_the_gpu(cq, torch):
    for shape in ((0, 2, 16, 64), (4, 0, 16, 64)):
        codes, scale = torch.zeros(shape, dtype=torch.int8, device="cuda"), torch.zeros(shape[:3], device="cuda")
        with pytest.raises(cq.CrossQuantError) as e:
            cq.crossquant_cache(codes, scale, codes, scale, 8)
        assert e.value.status == -2
