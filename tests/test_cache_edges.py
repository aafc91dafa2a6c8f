"""The quantized cache where single numbers decide: rows that hold no number, tokens that see nothing, values whose scales
lie far apart, queries with a channel far above the others, and the largest calls."""
from __future__ import annotations

import math

import pytest

from test_cache import ROUND, attention_oracle, check_attention, cq, descriptor, make_cache, make_table, places, queries, torch  # noqa: F401 (fixtures)

P = 0x10000


# ---- rows that hold no number --------------------------------------------------------------------------------------

@pytest.mark.gpu
@pytest.mark.parametrize("value", [float("inf"), -float("inf"), float("nan")])
@pytest.mark.parametrize("T,bits,kind,alpha", [(4, 8, "float16", 0.3), (4200, 8, "float16", 0.3), (3, 4, "bfloat16", 1.0), (4200, 4, "bfloat16", 1.0),
                                               (5, 8, "bfloat16", 0.0), (4300, 4, "float16", 0.0)])
def test_a_row_with_no_number_has_no_factor(cq, torch, T, bits, kind, alpha, value):
    """Its factor is NaN whatever alpha is (one row a thread, and eight); all other rows are as without it."""
    heads, dim, page = 33, 64, 16
    cache = make_cache(torch, cq, bits, T // page + 1, heads, page, dim, alpha=alpha, seed=4)
    X = torch.randn((T, heads, dim), generator=torch.Generator().manual_seed(6)).to(getattr(torch, kind)).cuda()
    slots = torch.arange(T, dtype=torch.int32).cuda()
    cq.crossquant_cache_write(cache, X, X, slots)
    before = {n: getattr(cache, n).clone() for n in ("k_codes", "k_scale", "v_codes", "v_scale")}
    K = X.clone()
    K[T // 2, 2, 11] = value
    cq.crossquant_cache_write(cache, K, X, slots)
    at = (T // 2 // page, 2, T // 2 % page)
    assert torch.isnan(cache.k_scale[at])
    cache.k_scale[at], cache.k_codes[at] = before["k_scale"][at], before["k_codes"][at]
    for n, t in before.items():
        assert torch.equal(getattr(cache, n), t)


# (lengths, key/value heads, query heads of each, tokens, dim, page, max_length): a block a pair, of four and of eight waves; two
# register tiles of rows; in pieces, joined by half waves and by blocks
FORMS = [([40, 3], 2, 8, 1, 64, 16, 40), ([600] * 64, 2, 2, 1, 128, 64, 600), ([90, 50], 1, 20, 2, 128, 32, 100),
         ([1500, 30], 2, 6, 1, 256, 64, None), ([2500, 600, 30], 2, 4, 3, 128, 16, None), ([1300] * 70, 1, 20, 1, 64, 32, 2100)]


@pytest.mark.gpu
@pytest.mark.parametrize("value", [float("inf"), -float("inf")])
@pytest.mark.parametrize("bits,kind", [(8, "float16"), (4, "bfloat16")])
@pytest.mark.parametrize("form", range(len(FORMS)))
@pytest.mark.parametrize("side", ["k", "v"])
def test_an_infinite_key_or_value_shows(cq, torch, side, form, bits, kind, value):
    """Queries of either sign: all rows that see the place are NaN, no other row changes."""
    lengths, heads, group, S, dim, page, max_length = FORMS[form]
    cache = make_cache(torch, cq, bits, sum(-(-n // page) for n in lengths) + 1, heads, page, dim, seed=form)
    table, lens = make_table(torch, cache, lengths, seed=form, extra=30)
    Q = queries(torch, len(lengths), S, heads * group, dim, kind, form)
    Q[:, :, 1::2] = -Q[:, :, ::2]
    pos = lengths[0] * 2 // 3
    slots = (table[0, pos // page] * page + pos % page).view(1)
    X = torch.randn((1, heads, dim), generator=torch.Generator().manual_seed(form)).to(getattr(torch, kind)).cuda()
    bad = X.clone()
    bad[0, 0, 5] = value
    cq.crossquant_cache_write(cache, X, X, slots)
    want = cq.crossquant_cache_attention(cache, Q, table, lens, max_length=max_length)
    assert torch.isfinite(want).all()
    cq.crossquant_cache_write(cache, *((bad, X) if side == "k" else (X, bad)), slots)
    out = cq.crossquant_cache_attention(cache, Q, table, lens, max_length=max_length)
    assert torch.isnan(out[0, :, :group]).all()
    out[0, :, :group] = want[0, :, :group]
    assert torch.equal(out, want)


@pytest.mark.gpu
@pytest.mark.parametrize("group", [4, 20])
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("n", [20, 40, 700])
def test_a_value_with_no_number_shows_at_any_weight(cq, torch, n, bits, group):
    """A visible position whose softmax weight is 0 in binary32 and whose value is no number: zero times that is none either, in the
    sequence's last tile as in those before it.  An earlier token, which does not see it, is free of it."""
    cache = make_cache(torch, cq, bits, n // 16 + 1, 1, 16, 64, cols=False, seed=41)
    table, lens = make_table(torch, cache, [n], seed=41, extra=0)
    Q = torch.zeros((1, 2, group, 64), dtype=torch.float16, device="cuda")
    Q[..., 0] = 1.0
    cache.k_codes.zero_()
    cache.k_scale.fill_(1.0)
    for pos in (0, n - 2, n - 1):
        page, place = int(table[0, pos // 16]), pos % 16
        cache.k_codes[page, 0, place, 0] = -7 if bits == 8 else 9
        kept = cache.v_scale[page, 0, place].clone()
        cache.v_scale[page, 0, place] = float("nan")
        out = cq.crossquant_cache_attention(cache, Q, table, lens, scale=100.0)
        assert torch.isnan(out[0, 1]).all()
        assert torch.isfinite(out[0, 0]).all() if pos == n - 1 else torch.isnan(out[0, 0]).all()
        cache.v_scale[page, 0, place] = kept


# ---- tokens that see nothing ---------------------------------------------------------------------------------------

@pytest.mark.gpu
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("bits,heads,group,dim,lengths,max_length", [
    (8, 2, 2, 64, [2, 50, 3], 64), (4, 1, 20, 128, [2, 100, 1], 100), (8, 2, 2, 256, [2, 2000, 3], None), (4, 1, 3, 64, [2, 1500, 40], 4096),
    (8, 4, 2, 128, [2, 600] * 32, 600)])
def test_a_token_that_sees_nothing_is_zero_whatever_its_query(cq, torch, bits, heads, group, dim, lengths, max_length, value):
    S, page = 4, 16
    cache = make_cache(torch, cq, bits, sum(-(-n // page) for n in lengths) + 300, heads, page, dim, seed=40)
    table, lens = make_table(torch, cache, lengths, seed=40, extra=260)
    Q = queries(torch, len(lengths), S, heads * group, dim, "float16")
    want = cq.crossquant_cache_attention(cache, Q, table, lens, max_length=max_length)
    blind = torch.arange(S, device="cuda") < S - lens[:, None]
    assert blind[0].tolist() == [True, True, False, False]
    Q[:, :, ::2, 5] = value
    out = cq.crossquant_cache_attention(cache, Q, table, lens, max_length=max_length)
    assert (out[blind] == 0).all()
    assert torch.isnan(out[~blind][:, ::2]).all()
    assert torch.equal(out[:, :, 1::2], want[:, :, 1::2])


@pytest.mark.gpu
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("length", [50, 1500])
def test_a_token_whose_pages_do_not_exist_is_zero_whatever_its_query(cq, torch, length, value):
    cache = make_cache(torch, cq, 8, 10, 2, 16, 64, seed=8)
    table = torch.full((1, length // 16 + 1), -1, dtype=torch.int32, device="cuda")
    table[0, 1::2] = 10
    lens = torch.tensor([length], dtype=torch.int32, device="cuda")
    Q = queries(torch, 1, 2, 4, 64, "float16")
    Q[0, 1, 1, 7] = value
    assert (cq.crossquant_cache_attention(cache, Q, table, lens) == 0).all()
    table[0, 1] = 3
    out = cq.crossquant_cache_attention(cache, Q, table, lens)
    assert torch.isnan(out[0, 1, 1]).all()
    out[0, 1, 1] = 0.0
    assert torch.isfinite(out).all()


# ---- weights -------------------------------------------------------------------------------------------------------

def weight_tolerance(torch, cache, Q, table, lengths, scale, max_length, ref):
    """How far a result may be off where no digit of a query is lost, before its own rounding.

    A score z passes seven roundings to binary32 (the integer product, the key's factor, three of the row's factor, the product, the
    exponent), each 2^-24 of it: dz = 2^-21 |z|, in numerator and denominator.  The exponential, its product with the value's factor and
    the weights' common factor (reciprocal included) are 6 times 2^-23; the two numbers of a weight keep it to 2^-22 of itself, and to
    2^-25 of the unit R / 65504 where they are subnormal, R at most eight times the largest product of a softmax weight and a factor of
    the row: 2^-38 of that.  Sums are binary32: a rounding (counted twice: the matrix instruction may truncate) for each value that is not zero, the
    8 waves, the pieces, and the factors that join them."""
    B, S, HQ, D = Q.shape
    H, page, q_max = cache.heads, cache.page_size, 127 if cache.bits == 8 else 7
    ck, ak, bk = places(torch, cache, "k")
    cv, av, bv = places(torch, cache, "v")
    tol = torch.zeros_like(ref)
    for b in range(B):
        for s in range(S):
            m = max(0, min(int(lengths[b]) - (S - 1 - s), max_length))
            pos = torch.arange(m, device=Q.device)
            at = table[b].long()[pos // page] * page + pos % page
            if m == 0:
                continue
            for h in range(H):
                g = slice(h * (HQ // H), (h + 1) * (HQ // H))
                z = scale * ((Q[b, s, g].double() * bk[h]) @ (ck[at, h] * ak[at, h, None]).t())
                p = torch.softmax(z, -1)
                size = p @ (cv[at, h] * av[at, h, None]).abs()
                terms = (cv[at, h] != 0).sum(0)                              # of each channel
                most = (p * av[at, h]).amax(-1, keepdim=True)
                dz = 2.0 ** -21 * z.abs().amax(-1, keepdim=True)
                tol[b, s, g] = bv[h] * ((torch.expm1(2 * dz) + 6 * 2.0 ** -23 + 2.0 ** -22 + (2 * terms + 64) * 2.0 ** -24) * size
                                        + m * 2.0 ** -38 * q_max * most)
    return tol


def check_weights(torch, cq, cache, Q, table, lengths, scale=None, max_length=None):
    scale = cache.dim ** -0.5 if scale is None else scale
    most = table.shape[1] * cache.page_size if max_length is None else max_length
    out = cq.crossquant_cache_attention(cache, Q, table, lengths, scale=scale, max_length=max_length)
    ref, _ = attention_oracle(torch, cache, Q, table, lengths, scale, most)
    tol = weight_tolerance(torch, cache, Q, table, lengths, scale, most, ref)
    kind = str(Q.dtype).split(".")[1]
    bad = ~((out.double() - ref).abs() <= ROUND[kind] * ref.abs() + (1 + ROUND[kind]) * tol + (2.0 ** -25 if kind == "float16" else 0.0))
    assert not bad.any(), "%d of %d outputs, the first at %s: %s, not %s" % (
        int(bad.sum()), bad.numel(), bad.nonzero()[0].tolist(), out[bad][0].item(), ref[bad][0].item())


def set_values(torch, cache, codes, scale, at):
    """Values and their factors of the places `at`, from [place][head][dim] and [place][head]."""
    page = cache.page_size
    c = codes.to(torch.int64) & 15
    c = codes.to(torch.int8) if cache.bits == 8 else (c[..., 0::2] | (c[..., 1::2] << 4)).to(torch.uint8)
    cache.v_codes[at // page, :, at % page] = c.to(cache.v_codes.device)
    cache.v_scale[at // page, :, at % page] = scale.to(cache.v_scale)


def cancelling_values(torch, n, heads, dim, q_max, seed):
    """Values of n positions, 16 of which are not zero: pairs of opposite codes whose factors differ by some per cent, so that sums are
    a few hundredths of their terms and a weight's own rounding shows in them."""
    g = torch.Generator().manual_seed(seed)
    codes, scale = torch.zeros((n, heads, dim)), torch.ones((n, heads))
    at = torch.randperm(n, generator=g)[:16]
    half = torch.randint(1, q_max + 1, (8, heads, dim), generator=g) * (2 * torch.randint(0, 2, (8, heads, dim), generator=g) - 1)
    codes[at[:8]], codes[at[8:]] = half.float(), -half.float()
    first = 0.01 * (1.0 + torch.rand((8, heads), generator=g))
    scale[at[:8]], scale[at[8:]] = first, first * (1.0 + 0.05 * torch.rand((8, heads), generator=g))
    return codes, scale


FLAT = [(40, 2, 4, 1, 64, 16, 64), (300, 2, 20, 1, 128, 16, 400), (500, 1, 4, 2, 256, 32, None), (1500, 2, 3, 1, 128, 64, None), (1400, 1, 20, 1, 64, 32, 2000)]


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["float16", "bfloat16"])
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("form", range(len(FLAT)))
def test_weights_keep_their_bits(cq, torch, form, bits, kind):
    """scale 0: every score is exactly 0, and sums that cancel show the weights' own rounding (one binary16 number a weight is off by
    some 20 times the tolerance, see the test of the two forms on the CPU)."""
    n, heads, group, S, dim, page, max_length = FLAT[form]
    cache = make_cache(torch, cq, bits, n // page + 1, heads, page, dim, cols=False, seed=form)
    table, lens = make_table(torch, cache, [n], seed=form, extra=30)
    pos = torch.arange(n)
    at = (table[0].cpu().long()[pos // page] * page + pos % page).cuda()
    set_values(torch, cache, *cancelling_values(torch, n, heads, dim, 127 if bits == 8 else 7, form), at)
    check_weights(torch, cq, cache, queries(torch, 1, S, heads * group, dim, kind), table, lens, scale=0.0, max_length=max_length)


def test_one_number_a_weight_is_not_enough(torch):
    """On the CPU: the weights of the test above as two binary16 numbers stay within its tolerance, as one they do not."""
    n, dim = 40, 64
    codes, scale = cancelling_values(torch, n, 1, dim, 127, 0)
    codes, a = codes[:, 0].double(), scale[:, 0].double()
    R = 2.0 ** math.ceil(math.log2(float(a.max())) + 1e-9)
    w = a * 2.0 ** 14 / R
    first = w.half().double()
    both = first + (w - first).half().double()
    exact, size = (w @ codes), (w @ codes.abs())
    terms = (codes != 0).sum(0)
    tol = ROUND["float16"] * exact.abs() + (6 * 2.0 ** -23 + 2.0 ** -22 + (2 * terms + 64) * 2.0 ** -24) * size
    assert ((both @ codes - exact).abs() <= 2.0 ** -22 * size).all()
    off = (first @ codes - exact).abs() / tol
    assert off.max() > 2 and (off > 1).sum() > dim // 8


@pytest.mark.gpu
@pytest.mark.parametrize("binades", [20, 33, 45, 80])
@pytest.mark.parametrize("bits,n,heads,group,S,dim,page,max_length,kind", [
    (8, 30, 2, 2, 1, 64, 16, 64, "float16"), (4, 300, 1, 20, 2, 128, 16, 400, "bfloat16"), (8, 400, 1, 4, 1, 256, 32, None, "float16"),
    (8, 1500, 2, 4, 1, 128, 64, None, "bfloat16"), (4, 1400, 1, 20, 1, 64, 32, 2000, "float16")])
def test_a_value_that_no_weight_asks_for_takes_no_bits(cq, torch, bits, n, heads, group, S, dim, page, max_length, kind, binades):
    """Positions with enormous values and a softmax weight of 2^-101 beside others of ordinary values: results are the others'.  Early
    and late ones, in one tile with the others and in tiles of their own; every second query has the opposite sign, and the enormous
    values are all that it attends to."""
    cache = make_cache(torch, cq, bits, n // page + 1, heads, page, dim, cols=False, seed=51)
    table, lens = make_table(torch, cache, [n], seed=51, extra=30)
    q_max = 127 if bits == 8 else 7
    g = torch.Generator().manual_seed(n + binades)
    big = torch.zeros(n, dtype=torch.bool)
    big[torch.randperm(n, generator=g)[:3]] = True
    big[n // 2:n // 2 + 40] = True
    big[[0, n - 1]] = True
    pos = torch.arange(n)
    at = (table[0].cpu().long()[pos // page] * page + pos % page).cuda()
    cache.k_codes.zero_()
    cache.k_scale.fill_(1.0)
    sign = torch.where(big, -q_max, q_max)
    cache.k_codes[at // page, :, at % page, 0] = (sign if bits == 8 else sign & 15).to(cache.k_codes)[:, None]
    scale = 0.01 * torch.exp(0.3 * torch.randn((n, heads), generator=g)) * torch.where(big, 2.0 ** binades, 1.0)[:, None]
    set_values(torch, cache, torch.randint(-q_max, q_max + 1, (n, heads, dim), generator=g).float(), scale, at)
    Q = torch.zeros((1, S, heads * group, dim), dtype=getattr(torch, kind), device="cuda")
    Q[..., 0] = 1.0
    Q[:, :, 1::2, 0] = -1.0
    if kind == "float16":
        Q[:, :, 1::2, 0] = 1.0                                               # (no binary16 result of that size)
    check_weights(torch, cq, cache, Q, table, lens, scale=35.0 / q_max, max_length=max_length)


@pytest.mark.gpu
@pytest.mark.parametrize("binades", [20, 45, 80])
@pytest.mark.parametrize("n", [100, 400, 3000])
def test_weights_that_later_scores_outweigh(cq, torch, n, binades):
    """Scores rise along the sequence, in small steps and in one large one, while the values' factors fall: what was the largest
    product at first is nothing at the end."""
    cache = make_cache(torch, cq, 8, n // 16 + 1, 1, 16, 64, cols=False, seed=52)
    table, lens = make_table(torch, cache, [n], seed=52)
    pos = torch.arange(n)
    at = (table[0].cpu().long()[pos // 16] * 16 + pos % 16).cuda()
    g = torch.Generator().manual_seed(n)
    cache.k_codes.zero_()
    cache.k_scale.fill_(1.0)
    for steps in (127, 1):
        rise = torch.div(pos * steps, n - 1, rounding_mode="floor") * (254 // steps) - 127
        cache.k_codes[at // 16, :, at % 16, 0] = rise.to(cache.k_codes)[:, None]
        scale = 0.01 * torch.exp2(-binades * (rise + 127) / 254.0)[:, None] * (1.0 + torch.rand((n, 1), generator=g)) * 2.0 ** binades
        set_values(torch, cache, torch.randint(-127, 128, (n, 1, 64), generator=g).float(), scale, at)
        Q = torch.zeros((1, 1, 2, 64), dtype=torch.bfloat16, device="cuda")
        Q[..., 0] = torch.tensor([1.0, 0.5])
        check_weights(torch, cq, cache, Q, table, lens, scale=80.0 / 254.0)


# ---- queries with a channel far above the others -------------------------------------------------------------------

@pytest.mark.gpu
@pytest.mark.parametrize("factor", [100.0, 1000.0])
@pytest.mark.parametrize("bits,n,heads,group,dim,kind", [(8, 300, 2, 4, 128, "float16"), (4, 90, 1, 20, 64, "bfloat16"), (8, 1500, 2, 3, 256, "bfloat16"),
                                                         (4, 2000, 1, 4, 128, "float16")])
def test_a_query_with_an_outlying_channel(cq, torch, bits, n, heads, group, dim, kind, factor):
    """The row's fixed point is relative to the outlier: results are those of the query rounded to it (each element off by at most
    1.6e-5 of the largest, as documented), with no further loss."""
    cache = make_cache(torch, cq, bits, n // 16 + 1, heads, 16, dim, seed=61)
    cache.k_col.fill_(1.0)
    table, lens = make_table(torch, cache, [n], seed=61)
    Q = queries(torch, 1, 1, heads * group, dim, kind, 61)
    Q[..., 9] = factor * (1.0 + Q[..., 9].abs()) * Q[..., 9].sign()
    x = Q.float()
    top = x.abs().amax(-1, keepdim=True)
    fixed = torch.round(x * (torch.full_like(top, 32512.0) / top)).double() * (top.double() / 32512.0)
    assert ((fixed - x.double()).abs() <= 1.6e-5 * top).all()
    scale = 1.0 / factor
    most = table.shape[1] * 16
    out = cq.crossquant_cache_attention(cache, Q, table, lens, scale=scale)
    ref, _ = attention_oracle(torch, cache, fixed, table, lens, scale, most)
    tol = weight_tolerance(torch, cache, fixed, table, lens, scale, most, ref)
    assert ((out.double() - ref).abs() <= ROUND[kind] * ref.abs() + (1 + ROUND[kind]) * tol + 2.0 ** -25).all()


# ---- scores that are billions ----------------------------------------------------------------------------------------

@pytest.mark.gpu
@pytest.mark.parametrize("bits,n,group,dim,kind,size", [(8, 40, 4, 128, "float16", 6e4), (4, 300, 20, 64, "float16", 6e4), (8, 1500, 4, 256, "float16", 6e4),
                                                        (4, 100, 3, 128, "bfloat16", 1e9), (8, 700, 20, 128, "bfloat16", 1e9)])
def test_scores_of_the_types_largest_numbers(cq, torch, bits, n, group, dim, kind, size):
    """Keys of one size and queries of either sign: equal scores of 2^33 and more are a mean over the values; with some keys half as
    large, over the larger scores alone."""
    cache = make_cache(torch, cq, bits, n // 16 + 1, 1, 16, dim, cols=False, alpha=1.0, seed=44)
    table, lens = make_table(torch, cache, [n], seed=44)
    pos = torch.arange(n)
    at = table[0].cpu().long()[pos // 16] * 16 + pos % 16
    dtype = getattr(torch, kind)
    Q = torch.full((1, 1, group, dim), size, dtype=dtype, device="cuda")
    Q[:, :, 1::2] = -size
    Q[:, :, 2] /= 3.0
    V = torch.randn((n, 1, dim), generator=torch.Generator().manual_seed(n)).to(dtype).cuda()
    half = torch.zeros(n, dtype=torch.bool)
    for part in (None, slice(0, 3), slice(n - 9, n), slice(0, n, 2)):
        if part is not None:
            half[part] = True
        K = torch.full((n, 1, dim), size, dtype=dtype)
        K[half] /= 2.0
        cq.crossquant_cache_write(cache, K.cuda(), V, at.to(torch.int32).cuda())
        codes, scale, _ = places(torch, cache, "v")
        v = codes[at, 0] * scale[at, 0, None]
        out = cq.crossquant_cache_attention(cache, Q, table, lens)[0, 0].double()
        large = v[~half].mean(0)
        small = v[half].mean(0) if part is not None else large
        for h in range(group):
            ref = small if h % 2 else large
            # (every weight is the same: its two numbers, n sums of values and of ones, one quotient)
            tol = ROUND[kind] * ref.abs() + (1 + ROUND[kind]) * (2.0 ** -21 + 2 * n * 2.0 ** -24) * v.abs().mean(0) * n / max(1, int((half if h % 2 and part is not None else ~half).sum())) + 2.0 ** -25
            assert ((out[h] - ref).abs() <= tol).all()


@pytest.mark.gpu
@pytest.mark.parametrize("bits,n,group,dim", [(8, 60, 4, 128), (4, 900, 20, 64)])
@pytest.mark.parametrize("k_size,q_size", [(1e34, 1e-29), (1e-30, 1e30)])
def test_scores_of_huge_keys_and_tiny_queries(cq, torch, bits, n, group, dim, k_size, q_size):
    """Scores of ordinary size from factors at the ends of bfloat16."""
    cache = make_cache(torch, cq, bits, n // 16 + 1, 2, 16, dim, cols=False, alpha=1.0, seed=45)
    table, lens = make_table(torch, cache, [n], seed=45)
    pos = torch.arange(n)
    at = table[0].cpu().long()[pos // 16] * 16 + pos % 16
    g = torch.Generator().manual_seed(n)
    K, V = (torch.randn((n, 2, dim), generator=g) for _ in range(2))
    cq.crossquant_cache_write(cache, (K * k_size).bfloat16().cuda(), V.bfloat16().cuda(), at.to(torch.int32).cuda())
    Q = (torch.randn((1, 1, 2 * group, dim), generator=g) * q_size).bfloat16().cuda()
    check_attention(torch, cq, cache, Q, table, lens, scale=0.3 / (k_size * q_size))


# ---- the largest calls ---------------------------------------------------------------------------------------------

def test_size_limits_are_the_same_for_workspace_and_call(cq):
    c = descriptor(cq, heads=1)

    def both(B, S, HQ, most=64, width=4):
        need = cq.raw.crossquant_cache_attention_workspace(c, B, S, HQ, most)
        status = cq.raw.crossquant_cache_attention(c, P, 64, 64, 64, 0, B, S, HQ, P, width, P, most, 0.1, P, P, need - 1, None)
        return need, status
    for B, S, HQ in ((1 << 24, 8, 1), (2048, 1024, 64), (1 << 24, 128, 1)):
        assert both(B, S, HQ) == (-1, -2)
    for B, S, HQ in ((64, 4096, 64), (1 << 24, 1, 1), (1 << 24, 7, 1), (2047, 1024, 64)):
        need, status = both(B, S, HQ, 1 << 20, 1 << 16)
        assert need > 0 and status == -2                                     # (a byte too few)


@pytest.mark.parametrize("size", [(1 << 64) + 64, 1 << 63, -(1 << 64) + 64])
def test_sizes_past_64_bits_are_refused(cq, torch, size):
    codes, scale = torch.zeros((4, 2, 16, 64), dtype=torch.int8), torch.zeros((4, 2, 16))
    cache = cq.crossquant_cache(codes, scale, codes, scale, 8)
    for sizes in ((size, 1, 2, 64), (1, size, 2, 64), (1, 1, size, 64), (1, 1, 2, size)):
        with pytest.raises(cq.CrossQuantError) as e:
            cq.crossquant_cache_attention_workspace(cache, *sizes)
        assert e.value.status == -2
    Q, table, lens = torch.zeros((1, 1, 4, 64), dtype=torch.float16), torch.zeros((1, 4), dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    with pytest.raises(cq.CrossQuantError) as e:
        cq.crossquant_cache_attention(cache, Q, table, lens, max_length=size)
    assert e.value.status == -2


@pytest.mark.gpu
@pytest.mark.parametrize("B,S,heads,group,max_length", [(64, 4096, 1, 64, 64), (64, 4096, 1, 64, 1 << 18), ((1 << 20) + 3, 1, 16, 1, 64)])
def test_calls_of_more_than_sixteen_million_rows(cq, torch, B, S, heads, group, max_length):
    """One query row for all, so that a few small calls say what each row is."""
    dim, page = 64, 65536 if max_length > 64 else 16
    cache = make_cache(torch, cq, 8, 4, heads, page, dim, seed=70)
    width = -(-max_length // page)
    table = torch.arange(width, dtype=torch.int32, device="cuda").expand(B, width).contiguous()
    lens = (torch.arange(B, device="cuda") % 61).to(torch.int32)
    one = queries(torch, 1, 1, heads * group, dim, "bfloat16")
    out = cq.crossquant_cache_attention(cache, one.expand(B, S, -1, -1), table, lens, max_length=max_length)
    few = torch.arange(61, dtype=torch.int32, device="cuda")
    want = cq.crossquant_cache_attention(cache, one.expand(61, 1, -1, -1), table[:61].contiguous(), few, max_length=64)[:, 0]
    size = -(-B // 8)
    for b in range(0, B, size):
        seen = (lens[b:b + size, None] - (S - 1 - torch.arange(S, device="cuda"))).clamp(min=0)
        assert torch.equal(out[b:b + size].view(torch.int16), want[seen].view(torch.int16))


@pytest.mark.gpu
def test_column_factors_behind_two_to_the_31(cq, torch):
    """More heads than 32-bit offsets into their factors reach (about 60 GiB)."""
    heads, dim, page, few = (1 << 23) + 3, 256, 16, 5
    small = make_cache(torch, cq, 4, 1, few, page, dim, alpha=0.3, seed=71)
    tensors, cols = [], []
    for n in "kv":
        codes = torch.zeros((1, heads, page, dim // 2), dtype=torch.uint8, device="cuda")
        scale = torch.zeros((1, heads, page), device="cuda")
        col = torch.zeros((heads, dim), device="cuda")
        for t, name in ((codes, "_codes"), (scale, "_scale")):
            t[:, -few:] = getattr(small, n + name)
        col[-few:] = getattr(small, n + "_col")
        tensors += [codes, scale]
        cols.append(col)
    cache = cq.crossquant_cache(*tensors, 4, alpha=0.3, k_col=cols[0], v_col=cols[1])
    table, lens = torch.zeros((1, 1), dtype=torch.int32, device="cuda"), torch.full((1,), 13, dtype=torch.int32, device="cuda")
    q = queries(torch, 1, 1, few, dim, "bfloat16")
    Q = torch.zeros((1, 1, heads, dim), dtype=torch.bfloat16, device="cuda")
    Q[:, :, -few:] = q
    out = cq.crossquant_cache_attention(cache, Q, table, lens)
    assert torch.equal(out[:, :, -few:], cq.crossquant_cache_attention(small, q, table, lens))
    assert not out.view(torch.int64)[:, :, :-few].any()
    del cache, tensors, cols, Q, out, codes, scale, col, t
    torch.cuda.empty_cache()
