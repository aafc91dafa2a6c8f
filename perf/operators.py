"""Block-scaled FP8 linear layers and the quantized key/value cache, as measurable cases.

Every case is one pass through the public calls of ``paper_2410_07505_amd`` (``own`` true) or through the same
operators in elementary torch operations (``own`` false), on inputs that a program has in hand already: activations
(a few channels far larger than the rest), FP8 weights with a scale for every 128 x 128 block, a paged cache filled by
earlier steps.  ``kind`` says which calls:

``layer``   quantize_fp8 (a scale for every 128 channels of a token) and fp8_linear: one FP8 layer of a serving program.
``linear``  fp8_linear alone, on codes that several projections share.
``weight``  weight_quantize_fp8: weight preparation when a model is loaded.
``chunk``   cache_write of a chunk's keys and values, then cache_read of a sequence's tokens: what prompt attention over
            a cached prefix needs.
``step``    cache_write of the new tokens, then cache_attention over the cache: attention of one decode step.
``attend``  cache_attention alone (the step's tokens are in the cache already).

Definitions (fl32: rounded to binary32; rne: round to nearest, ties to even):

    FP8 group g of 128:  m = max |x|;  m < 2^-100: s = r = 0, else s = fl32(m / 448), r = fl32(448 / m)
                         code = e4m3(fl32(x r));  the value a code stands for is code s
    linear               Y_ik = sum over blocks b of s_x[b, i] s_w[k / 128, b] (sum over j in b of cx_ij cw_kj)
    cache, row of a token and head:  a = fl32(t^alpha / q_max), t = max |x|;  D_j = fl32(a b_j);
                         q = clamp(rne(fl32(x / D_j)), +-q_max);  the value it stands for is q D_j
    attention            softmax over the visible tokens of scale q.k, times v; a row that sees no token is zero
"""
import math

import torch

own = False

FP8_MAX = 448.0
TINY = 2.0 ** -100
BLOCK = 128


def listed():
    return [
        # the smallest layer: 64 tokens of a test model, all latency and launches
        {"name": "layer_tiny", "kind": "layer", "T": 64, "I": 256, "O": 256, "type": "float16"},
        # decode of 16 sequences through the up-projection of a 70B-shaped MLP: the weights have to be read
        {"name": "layer_decode_70b", "kind": "layer", "T": 16, "I": 8192, "O": 28672, "type": "bfloat16"},
        # prefill of 2048 tokens through the up-projection of a 7B-shaped MLP
        {"name": "layer_prefill_7b", "kind": "layer", "T": 2048, "I": 4096, "O": 11008, "type": "float16"},
        # a pruned layer: token count and widths that are multiples of nothing
        {"name": "layer_ragged", "kind": "layer", "T": 509, "I": 2750, "O": 4090, "type": "bfloat16"},
        # the matrix product of a 70B-shaped MLP up-projection, the largest call there is
        {"name": "linear_70b", "kind": "linear", "T": 4096, "I": 8192, "O": 28672, "type": "bfloat16"},
        # a 7B-shaped weight prepared at load time
        {"name": "weight_7b", "kind": "weight", "I": 4096, "O": 11008, "type": "float16"},
        # the pruned layer's weight
        {"name": "weight_ragged", "kind": "weight", "I": 2750, "O": 4090, "type": "bfloat16"},
        # a short chunk of a small model: odd counts, padding tokens that are not written
        {"name": "chunk8_odd", "kind": "chunk", "bits": 8, "T": 333, "R": 1001, "heads": 3, "dim": 64, "page": 16, "type": "float16"},
        # 2048 prompt tokens written, the 16384 tokens of their sequence read back for the chunk's attention
        {"name": "chunk4_prefix", "kind": "chunk", "bits": 4, "T": 2048, "R": 16384, "heads": 8, "dim": 128, "page": 64, "type": "bfloat16"},
        # one user's decode step early in a conversation: latency
        {"name": "step8_single", "kind": "step", "bits": 8, "B": 1, "S": 1, "L": 500, "heads": 8, "group": 4, "dim": 128, "page": 16, "type": "float16"},
        # decode of 64 sequences of 1024 to 8192 tokens, 64 query heads on 8 key/value heads
        {"name": "attend8_batch", "kind": "attend", "bits": 8, "B": 64, "S": 1, "L": 8192, "heads": 8, "group": 8, "dim": 128, "page": 64, "type": "bfloat16"},
        # four drafted tokens behind each of two long documents, INT4 cache
        {"name": "attend4_long", "kind": "attend", "bits": 4, "B": 2, "S": 4, "L": 131072, "heads": 8, "group": 4, "dim": 128, "page": 128, "type": "float16"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A layer width: mostly whole multiples of 128 as in the usual models, now and then any number (pruned, sharded)."""
    w = _log(rng, lo, hi)
    return max(128, w // 128 * 128) if rng.random() < 0.7 else w


def draw(rng):
    kind = rng.choice(["layer", "layer", "linear", "weight", "chunk", "step", "attend", "attend"])
    case = {"kind": kind, "type": rng.choice(["float16", "bfloat16"])}
    if kind in ("layer", "linear"):
        case.update(T=_log(rng, 1, 4096), I=_width(rng, 100, 8192), O=_width(rng, 100, 28672))
    elif kind == "weight":
        case.update(I=_width(rng, 100, 8192), O=_width(rng, 100, 20480))
    else:
        case.update(bits=rng.choice([8, 4]), heads=rng.randint(1, 16), dim=rng.choice([64, 128, 128, 256]), page=rng.choice([16, 32, 64, 128]))
        if kind == "chunk":
            case.update(T=_log(rng, 1, 4096), R=_log(rng, 1, 16384))
        else:
            B, L = _log(rng, 1, 64), _log(rng, 1, 131072)
            room = (1 << 28) // (case["heads"] * case["dim"] * B)          # about the listed batch's cache
            case.update(B=B, S=rng.choice([1, 1, 1, 2, 5]), L=max(1, min(L, room)), group=rng.choice([1, 2, 4, 7, 8, 16]))
    return case


# ---- inputs -------------------------------------------------------------------------------------------------

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _outliers(g, n, one_in, lo, hi):
    """Per-channel magnitudes: 1, but for one channel in `one_in`."""
    s = torch.ones(n, device="cuda")
    k = max(1, n // one_in)
    s[torch.randperm(n, generator=g, device="cuda")[:k]] = lo + (hi - lo) * torch.rand(k, generator=g, device="cuda")
    return s


def _activation(g, T, I, dtype):
    return (_randn(g, T, I) * _outliers(g, I, 200, 50.0, 100.0)).to(dtype)


def _slots(g, n_slots, n, padding):
    """n different places of the cache in no order; a share of them -1, as for the padding tokens of a batch."""
    s = torch.randperm(n_slots, generator=g, device="cuda")[:n].to(torch.int32)
    if padding:
        s[torch.rand(n, generator=g, device="cuda") < 0.05] = -1
    return s


def _cache(g, pages, case):
    """A cache that earlier steps have filled: codes and scales as keys and values of unit size give them."""
    bits, H, D, page = case["bits"], case["heads"], case["dim"], case["page"]
    q_max, alpha = (127, 0.15) if bits == 8 else (7, 0.15)
    cache = {"bits": bits, "alpha": alpha}
    for n in "kv":
        c = _outliers(g, H * D, 64, 3.0, 8.0).view(H, D) * 3.5
        col = c.double().pow(1.0 - alpha).float()
        t = c.max() * (0.5 + 0.5 * torch.rand((pages, H, page), generator=g, device="cuda"))
        a = (t.double().pow(alpha) / q_max).float()
        if bits == 8:
            codes = torch.randint(-90, 91, (pages, H, page, D), generator=g, device="cuda", dtype=torch.int8)
        else:
            codes = torch.randint(0, 256, (pages, H, page, D // 2), generator=g, device="cuda", dtype=torch.uint8)
            codes = torch.where(codes % 16 == 8, codes ^ 1, codes)         # -8 is no code
            codes = torch.where(codes // 16 == 8, codes ^ 16, codes)
        cache.update({n + "_codes": codes, n + "_scale": a, n + "_col": col})
    return cache


def _lengths(case):
    """Lengths of the batch: from an eighth of L to L, evenly (the same set for every seed)."""
    B, L = case["B"], case["L"]
    return [max(1, L // 8 + (L - L // 8) * (i + 1) // B) for i in range(B)]


def prepare(case, seed):
    g = _generator(seed)
    kind, dtype = case["kind"], getattr(torch, case["type"])
    s = {"kind": kind, "dtype": dtype}
    if kind in ("layer", "linear", "weight"):
        I, O = case["I"], case["O"]
        W = (_randn(g, I, O) * 0.02 * _outliers(g, O, 100, 2.0, 8.0)).to(dtype)
        if kind == "weight":
            s["W"] = W
            return s
        s["qw"], s["w_scale"] = _weight_fp8(W)
        del W
        X = _activation(g, case["T"], I, dtype)
        if kind == "layer":
            s["X"] = X
        else:
            s["qx"], s["x_scale"] = _rows_fp8(X)
        return s
    H, D, page = case["heads"], case["dim"], case["page"]
    if kind == "chunk":
        T, R = case["T"], case["R"]
        pages = (max(T, R) + T) // page + 2
        s.update(_cache(g, pages, case))
        s["K"], s["V"] = ((_randn(g, T, H, D) * s[n + "_col"] / 3.5).to(dtype) for n in "kv")
        s["slots"] = _slots(g, pages * page, T, True)
        s["read"] = _slots(g, pages * page, R, True)
        return s
    B, S = case["B"], case["S"]
    need = [-(-n // page) for n in _lengths(case)]
    order = torch.randperm(B, generator=g, device="cuda")
    lengths = torch.tensor(_lengths(case), device="cuda", dtype=torch.int32)[order].contiguous()
    pages = sum(need) + 3
    s.update(_cache(g, pages, case))
    # pages are handed out in no order; a sequence's row of the table ends in -1
    width = max(need) + 1
    at = torch.arange(width, device="cuda")
    used = at < (-(-lengths // page))[:, None]
    table = torch.full((B, width), -1, device="cuda", dtype=torch.int32)
    table[used] = torch.randperm(pages, generator=g, device="cuda")[:sum(need)].to(torch.int32)
    s.update(table=table, lengths=lengths, max_length=int(max(_lengths(case))))
    s["Q"] = (_randn(g, B, S, H * case["group"], D) / _col_heads(s["k_col"], case["group"]).sqrt()).to(dtype)
    if kind == "step":
        pos = lengths[:, None].long() - S + torch.arange(S, device="cuda")
        slot = table.gather(1, pos.clamp(min=0) // page).long() * page + pos.clamp(min=0) % page
        s["slots"] = torch.where(pos >= 0, slot, -1).to(torch.int32).view(-1)
        s["K"], s["V"] = ((_randn(g, B * S, H, D) * s[n + "_col"] / 3.5).to(dtype) for n in "kv")
    return s


def _col_heads(col, group):
    return col.repeat_interleave(group, 0)


# ---- the operators in plain form ----------------------------------------------------------------------------

def _over(a, b):
    """a / b of binary32 numbers, correctly rounded (a scalar operand would be turned into a product with its reciprocal)."""
    a, b = (v if isinstance(v, torch.Tensor) else torch.full((), v, device="cuda") for v in (a, b))
    return torch.div(a, b)


def _scales_fp8(m):
    live = m >= TINY
    return torch.where(live, _over(m, FP8_MAX), 0.0), torch.where(live, _over(FP8_MAX, m.clamp(min=TINY)), 0.0)


def _pad(X, rows, cols):
    return torch.nn.functional.pad(X, (0, cols - X.shape[1], 0, rows - X.shape[0]))


def _up(n):
    return -(-n // BLOCK) * BLOCK


def _rows_fp8(X):
    """Codes [T][I up to a multiple of 128] and scales [blocks][T]."""
    T, I = X.shape
    x = _pad(X, T, _up(I)).float().view(T, -1, BLOCK)
    s, r = _scales_fp8(x.abs().amax(2))
    return (x * r[:, :, None]).to(torch.float8_e4m3fn).view(T, -1), s.t().contiguous()


def _weight_fp8(W):
    """W [I][O] -> codes [O][I up to a multiple of 128] and scales [blocks of O][blocks of I]."""
    I, O = W.shape
    w = _pad(W, _up(I), _up(O)).float().view(_up(I) // BLOCK, BLOCK, _up(O) // BLOCK, BLOCK)
    s, r = _scales_fp8(w.abs().amax((1, 3)))
    codes = (w * r[:, None, :, None]).view(_up(I), _up(O))[:, :O].t().contiguous().to(torch.float8_e4m3fn)
    return codes, s.t().contiguous()


def _linear_fp8(qx, x_scale, qw, w_scale, dtype):
    T, K = qx.shape
    O = qw.shape[0]
    x = (qx.float().view(T, -1, BLOCK) * x_scale.t()[:, :, None]).view(T, K)
    w = (qw.float().view(O, -1, BLOCK) * w_scale.repeat_interleave(BLOCK, 0)[:O, :, None]).view(O, K)
    return (x @ w.t()).to(dtype)


def _pack(q):
    q = q.to(torch.int32) & 15
    return (q[..., 0::2] | (q[..., 1::2] << 4)).to(torch.uint8)


def _unpack(p):
    p = p.to(torch.int32)
    return (torch.stack((p & 15, p >> 4), -1).flatten(-2) ^ 8) - 8


def _write(s):
    q_max = 127.0 if s["bits"] == 8 else 7.0
    page = s["k_scale"].shape[2]
    live = s["slots"] >= 0
    slots = s["slots"][live].long()
    at = (slots // page, slice(None), slots % page)
    for X, n in ((s["K"], "k"), (s["V"], "v")):
        x = X[live].float()
        a = (x.abs().amax(2).double().pow(s["alpha"]) / q_max).float()
        step = a[:, :, None] * s[n + "_col"]
        q = torch.where(step == 0, 0.0, _over(x, step)).round().clamp(-q_max, q_max)
        s[n + "_scale"][at] = a
        s[n + "_codes"][at] = q.to(torch.int8) if s["bits"] == 8 else _pack(q)


def _values(s, n, page, off):
    """Values of a cache's places (page, off), [...][heads][dim], zero where the page is negative."""
    at = (page.clamp(min=0), slice(None), off)
    codes = s[n + "_codes"][at]
    q = (codes if s["bits"] == 8 else _unpack(codes)).float()
    v = q * (s[n + "_scale"][at][..., None] * s[n + "_col"])
    return torch.where((page >= 0)[..., None, None], v, 0.0)


def _read(s):
    page = s["k_scale"].shape[2]
    r = s["read"].long()
    p = torch.where(r < 0, -1, r // page)
    return [_values(s, n, p, r.clamp(min=0) % page).to(s["dtype"]) for n in "kv"]


def _attend(s):
    Q, lengths, L = s["Q"], s["lengths"].long(), s["max_length"]
    B, S, HQ, D = Q.shape
    page = s["k_scale"].shape[2]
    H = s["k_scale"].shape[1]
    at = torch.arange(L, device="cuda")
    p = s["table"].long()[:, at // page]
    K, V = (_values(s, n, p, (at % page).expand(B, L)).permute(0, 2, 1, 3) for n in "kv")
    q = Q.float().view(B, S, H, HQ // H, D).permute(0, 2, 1, 3, 4).reshape(B, H, -1, D)
    scores = (q @ K.transpose(2, 3).contiguous()).view(B, H, S, HQ // H, L) / math.sqrt(D)
    seen = at < (lengths[:, None] - S + 1 + torch.arange(S, device="cuda"))[:, :, None]
    seen = (seen & (p >= 0)[:, None])[:, None, :, None]
    scores = scores.masked_fill(~seen, -math.inf)
    top = scores.amax(-1, keepdim=True)
    e = torch.exp(scores - torch.where(top == -math.inf, 0.0, top))
    total = e.sum(-1, keepdim=True)
    out = (e / torch.where(total == 0, 1.0, total)).view(B, H, -1, L) @ V.contiguous()
    return out.view(B, H, S, HQ // H, D).permute(0, 2, 1, 3, 4).reshape(B, S, HQ, D).to(s["dtype"])


# ---- one pass -----------------------------------------------------------------------------------------------

def run(s):
    kind = s["kind"]
    if own:
        import paper_2410_07505_amd as cq
        if kind == "layer":
            qx, x_scale = cq.crossquant_quantize_fp8(s["X"])
            return cq.crossquant_fp8_linear(qx, x_scale, s["qw"], s["w_scale"], dtype=s["dtype"]), qx, x_scale
        if kind == "linear":
            return cq.crossquant_fp8_linear(s["qx"], s["x_scale"], s["qw"], s["w_scale"], dtype=s["dtype"])
        if kind == "weight":
            return cq.crossquant_weight_quantize_fp8(s["W"])
        cache = cq.crossquant_cache(s["k_codes"], s["k_scale"], s["v_codes"], s["v_scale"], s["bits"], alpha=s["alpha"],
                                    k_col=s["k_col"], v_col=s["v_col"])
        if kind in ("chunk", "step"):
            cq.crossquant_cache_write(cache, s["K"], s["V"], s["slots"])
        if kind == "chunk":
            out = list(cq.crossquant_cache_read(cache, s["read"], dtype=s["dtype"]))
        else:
            out = [cq.crossquant_cache_attention(cache, s["Q"], s["table"], s["lengths"], max_length=s["max_length"])]
    else:
        if kind == "layer":
            qx, x_scale = _rows_fp8(s["X"])
            return _linear_fp8(qx, x_scale, s["qw"], s["w_scale"], s["dtype"]), qx, x_scale
        if kind == "linear":
            return _linear_fp8(s["qx"], s["x_scale"], s["qw"], s["w_scale"], s["dtype"])
        if kind == "weight":
            return _weight_fp8(s["W"])
        if kind in ("chunk", "step"):
            _write(s)
        out = _read(s) if kind == "chunk" else [_attend(s)]
    if kind != "attend":
        out += [s["k_scale"], s["v_scale"]]
        if s["bits"] == 8:                        # packed INT4 codes show in what is read back, and in the attention
            out += [s["k_codes"], s["v_codes"]]
    return out


def work(case):
    kind = case["kind"]
    if kind in ("layer", "linear", "weight"):
        I, O = case["I"], case["O"]
        K, nb, ob = _up(I), _up(I) // BLOCK, _up(O) // BLOCK
        if kind == "weight":
            return {"bytes": 2 * I * O + O * K + 4 * nb * ob, "flops": 0}
        T = case["T"]
        codes = T * K + 4 * T * nb                # read by the linear; in a layer they are an output of it
        x = 2 * T * I if kind == "layer" else 0
        return {"bytes": x + codes + O * K + 4 * nb * ob + 2 * T * O, "flops": 2 * T * I * O}
    H, D = case["heads"], case["dim"]
    row = 2 * H * (D * case["bits"] // 8 + 4)     # a token's codes and scales, keys and values
    if kind == "chunk":
        T, R = case["T"], case["R"]
        return {"bytes": T * (4 * H * D + row + 4) + R * (4 * H * D + row + 4), "flops": 0}
    B, S, HQ = case["B"], case["S"], H * case["group"]
    total = sum(_lengths(case))
    w = {"bytes": total * row + 4 * B * S * HQ * D + 4 * sum(-(-n // case["page"]) for n in _lengths(case)) + 4 * B, "flops": 4 * S * HQ * D * total}
    if kind == "step":
        w["bytes"] += B * S * (4 * H * D + row + 4)
    return w


# ---- the definitions in 64 bits -----------------------------------------------------------------------------

def _fl32(v):
    return v.float().double()


def _e4m3(v):
    """Nearest e4m3 value (ties to even) of |v| <= 448 and a little more: 3 fraction bits, exponents from -6."""
    _, e = torch.frexp(v)
    unit = torch.exp2((e - 1).clamp(min=-6).double() - 3.0)
    return (torch.round(v / unit) * unit).clamp(-448.0, 448.0)


def _exact_fp8(x, axes):
    """Codes and scales of x [...] with a group along `axes`, the axes kept."""
    m = x.abs().amax(axes, keepdim=True)
    dead = m < TINY
    m = torch.where(dead, torch.ones_like(m), m)
    r, s = _fl32(448.0 / m), _fl32(m / 448.0)
    return torch.where(dead, 0.0, _e4m3(_fl32(x * r))), torch.where(dead, 0.0, s)


def exact(case, seed):
    kind = case["kind"]
    if kind == "linear" and 2 * case["T"] * case["I"] * case["O"] > 4e14:
        return None                               # half a minute of binary64 products
    s = prepare(case, seed)
    if kind == "weight":
        W = s["W"].double()
        I, O = W.shape
        full = W.new_zeros(_up(I), _up(O))
        full[:I, :O] = W
        q, sc = _exact_fp8(full.view(_up(I) // BLOCK, BLOCK, -1, BLOCK), (1, 3))
        return q.reshape(_up(I), _up(O)).t()[:O].contiguous(), sc[:, 0, :, 0].t().contiguous()
    if kind in ("layer", "linear"):
        if kind == "layer":
            X = s["X"].double()
            T, I = X.shape
            full = X.new_zeros(T, _up(I))
            full[:, :I] = X
            q, sc = _exact_fp8(full.view(T, -1, BLOCK), (2,))
        else:
            T = s["qx"].shape[0]
            q, sc = s["qx"].double().view(T, -1, BLOCK), s["x_scale"].double().t()[:, :, None]
        cw = s["qw"].double()
        O, K = cw.shape
        Y = cw.new_zeros(T, O)
        per_row = s["w_scale"].double().repeat_interleave(BLOCK, 0)[:O]
        for b in range(K // BLOCK):
            Y += (q[:, b] * sc[:, b]) @ (cw[:, b * BLOCK:(b + 1) * BLOCK] * per_row[:, b, None]).t()
        return Y if kind == "linear" else (Y, q.reshape(T, K), sc[:, :, 0].t().contiguous())
    q_max = 127 if s["bits"] == 8 else 7
    values, scales = {}, {}
    for n in "kv":                                # codes and scales of the whole cache, the new tokens among them
        codes, a, col = s[n + "_codes"], s[n + "_scale"].double(), s[n + "_col"].double()
        if s["bits"] == 4:
            low, high = codes % 16, codes // 16
            codes = torch.stack((low, high), -1).flatten(-2).to(torch.int16)
            codes = torch.where(codes > 7, codes - 16, codes)
        codes = codes.transpose(1, 2).flatten(0, 1)                          # [place][head][dim]
        a = a.transpose(1, 2).flatten(0, 1)
        if kind != "attend":
            at = s["slots"][s["slots"] >= 0].long()
            x = s[n.upper()][s["slots"] >= 0].double()
            new = _fl32(x.abs().amax(2).pow(s["alpha"]) / q_max)
            D = _fl32(new[:, :, None] * col)
            q = torch.where(D > 0, torch.round(_fl32(x / D)), 0.0).clamp(-q_max, q_max)
            a[at], codes[at] = new, q.to(codes.dtype)
        values[n], scales[n] = (codes, a, col), a
    def take(n, places):
        codes, a, col = values[n]
        return codes[places].double() * (a[places][..., None] * col)
    page = s["k_scale"].shape[2]
    if kind == "chunk":
        out = []
        for n in "kv":
            v = take(n, s["read"].clamp(min=0).long())
            out.append(torch.where((s["read"] >= 0)[:, None, None], v, 0.0))
    else:
        B, S, HQ, D = s["Q"].shape
        H = s["k_col"].shape[0]
        O = torch.zeros(B, S, HQ, D, device="cuda", dtype=torch.float64)
        for b, n in enumerate(s["lengths"].tolist()):
            at = torch.arange(n, device="cuda")
            places = s["table"][b].long()[at // page] * page + at % page
            for h in range(H):
                K, V = ((values[c][0][places, h].double() * values[c][1][places, h, None]) * values[c][2][h] for c in "kv")
                for i in range(S):
                    m = n - S + 1 + i
                    if m > 0:
                        g = slice(h * (HQ // H), (h + 1) * (HQ // H))
                        z = s["Q"][b, i, g].double() @ K[:m].t() / math.sqrt(D)
                        O[b, i, g] = torch.softmax(z, -1) @ V[:m]
        out = [O]
    if kind != "attend":
        shape = s["k_scale"].shape
        out += [scales[n].view(shape[0], page, -1).transpose(1, 2).contiguous() for n in "kv"]
        if s["bits"] == 8:
            out += [values[n][0].view(shape[0], page, shape[1], -1).transpose(1, 2).contiguous() for n in "kv"]
    return out
