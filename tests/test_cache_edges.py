"""The quantized cache where single numbers decide: rows that hold no number, tokens that see nothing."""
from __future__ import annotations

import pytest

from test_cache import cq, make_cache, make_table, queries, torch  # noqa: F401 (fixtures)


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
