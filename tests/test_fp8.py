"""The FP8 calls (e4m3 codes with a scale for every block of 128) against plain implementations: codes and scales bit for bit, the
linear layer against a binary64 product."""
from __future__ import annotations

import numpy as np
import pytest

ROUND = {"float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}         # half a step, relative
TINY = 2.0 ** -100


@pytest.fixture(scope="module")
def cq():
    import paper_2410_07505_amd as pkg
    return pkg


@pytest.fixture(scope="module")
def torch():
    import torch
    return torch


# ---- plain implementations (CPU) -----------------------------------------------------------------------------

def e4m3(torch, v):
    """Nearest e4m3 value of binary64 numbers within the format's range, ties to even."""
    _, e = torch.frexp(v)
    unit = torch.exp2((e - 1).clamp(min=-6).double() - 3.0)
    return torch.round(v / unit) * unit


def block_codes(torch, x, axes):
    """(values of the codes, scales with `axes` kept), binary64 with the definition's binary32 roundings."""
    m = x.double().abs().amax(axes, keepdim=True)
    dead = m < TINY
    safe = torch.where(dead, torch.ones_like(m), m)
    r, s = (448.0 / safe).float().double(), (safe / 448.0).float().double()
    return torch.where(dead, torch.zeros_like(x.double()), e4m3(torch, (x.double() * r).float().double())), torch.where(dead, torch.zeros_like(s), s)


def rows_oracle(torch, X):
    T, I = X.shape
    full = torch.zeros((T, -(-I // 128) * 128), dtype=torch.float64)
    full[:, :I] = X.double()
    q, s = block_codes(torch, full.view(T, -1, 128), 2)
    return q.view(T, -1), s[:, :, 0].t().contiguous()


def weight_oracle(torch, W):
    I, O = W.shape
    full = torch.zeros((-(-I // 128) * 128, -(-O // 128) * 128), dtype=torch.float64)
    full[:I, :O] = W.double()
    q, s = block_codes(torch, full.view(full.shape[0] // 128, 128, -1, 128), (1, 3))
    return q.reshape(full.shape)[:, :O].t().contiguous(), s[:, 0, :, 0].t().contiguous()


def linear_oracle(qx, x_scale, qw, w_scale):
    """(Y, how far binary32 sums of it may be off) in binary64.

    Binary32: 128 products of a block, one scaled addition a block, the scales' product and the joining of at most 8 shares; each
    rounding is at most 2^-24 of the terms' magnitudes.
    The matrix instruction sums 8 neighbouring products with the bits from 2^-13 of the largest one's exponent on (ea + eb of its
    operands, -6 for those below 2^-6), and drops what lies below: at most 7 times 2^-13 2^(ea + eb) for each 8 products, as the
    largest loses nothing (4 + 4 significant bits make 8).  2^(ea + eb) <= max(|a|, 2^-6) max(|b|, 2^-6), and the largest of 8
    such numbers is at most the 8th root of the sum of their 8th powers, which is what is added up here."""
    T, O, blocks = qx.shape[0], qw.shape[0], qx.shape[1] // 128
    x, w = qx.double().view(T, blocks, 128), qw.double().view(O, blocks, 128)
    sx, sw = x_scale.double().t().contiguous(), w_scale.double().repeat_interleave(128, 0)[:O].contiguous()
    xs, ws = (x * sx[:, :, None]).flatten(1), (w * sw[:, :, None]).flatten(1)
    Y, slack = xs @ ws.t(), (xs.abs() @ ws.abs().t()) * 2.0 ** -24 * (128 + blocks + 16)
    ex, ew = x.abs().clamp(min=2.0 ** -6).pow(8), w.abs().clamp(min=2.0 ** -6).pow(8)
    for b in range(blocks):
        s = sx[:, b, None] * sw[:, b]
        for g in range(0, 128, 8):
            slack += 7 * 2.0 ** -13 * s * (ex[:, b, g:g + 8] @ ew[:, b, g:g + 8].t()).pow(0.125)
    return Y, slack


def tolerance(Y, slack, kind):
    """Half a step of the result's type (binary16: also below its normal numbers), and what the sums may be off."""
    return ROUND[kind] * (Y.abs() + slack) + slack + (2.0 ** -25 if kind == "float16" else 0.0)


def activation(torch, T, I, kind, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((T, I), generator=g)
    x[:, ::61] *= 70.0
    return x.to(getattr(torch, kind))


# ---- quantizers -----------------------------------------------------------------------------------------------

def check_rows(torch, cq, X, Xg):
    codes, scale = cq.crossquant_quantize_fp8(Xg)
    q, s = rows_oracle(torch, X)
    assert torch.equal(scale.cpu().double(), s)
    assert torch.equal(codes.cpu().double(), q)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["float16", "bfloat16"])
@pytest.mark.parametrize("T,I", [(1, 1), (1, 128), (3, 7), (5, 127), (2, 129), (17, 512), (9, 513), (64, 640), (33, 1000), (1, 8192),
                                 (1000, 8200), (2050, 4098)])
def test_activation_codes(cq, torch, T, I, kind):
    print("quantize_fp8 %d x %d %s" % (T, I, kind), flush=True)
    X = activation(torch, T, I, kind, T + I)
    check_rows(torch, cq, X, X.cuda())


@pytest.mark.gpu
@pytest.mark.parametrize("T,I,kind", [(2051, 4100, "float16"), (16385, 513, "bfloat16"), (4097, 2041, "float16")])
def test_activation_codes_of_many_rows(cq, torch, T, I, kind):
    """Several rows a wave, an odd number of them."""
    test_activation_codes(cq, torch, T, I, kind)


@pytest.mark.gpu
@pytest.mark.parametrize("offset,pitch", [(0, 776), (8, 768), (1, 768), (3, 777)])
def test_activation_codes_of_strided_rows(cq, torch, offset, pitch):
    X = activation(torch, 40, 700, "bfloat16", 5)
    store = torch.full((40 * pitch + 16,), float("nan"), dtype=torch.bfloat16, device="cuda")
    view = store[offset:offset + 40 * pitch].view(40, pitch)[:, :700]
    view.copy_(X)
    check_rows(torch, cq, X, view)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["float16", "bfloat16"])
def test_activation_groups_at_the_edges(cq, torch, kind):
    dtype = getattr(torch, kind)
    X = torch.zeros((8, 256), dtype=dtype)
    X[1, 3] = torch.finfo(dtype).max
    X[1, 4] = -torch.finfo(dtype).max
    X[2] = torch.finfo(dtype).smallest_normal
    X[3, ::2] = torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps     # the smallest subnormal: a zero group of bfloat16
    X[4, :128] = torch.linspace(-448, 448, 128).to(dtype)
    X[5, 128:] = torch.arange(128).to(dtype) / 8 + 1                            # many ties of e4m3
    X[5, 128] = 448.0
    X[6, 7] = -0.0
    X[7] = 1.0
    check_rows(torch, cq, X, X.cuda())


@pytest.mark.gpu
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
def test_a_group_with_no_number_has_no_finite_scale(cq, torch, value):
    X = activation(torch, 20, 300, "float16", 1).cuda()
    clean = cq.crossquant_quantize_fp8(X)
    X[11, 130] = value
    codes, scale = cq.crossquant_quantize_fp8(X)
    assert not torch.isfinite(scale[1, 11])
    keep = torch.ones((3, 20), dtype=torch.bool, device="cuda")
    keep[1, 11] = False
    assert torch.equal(scale[keep], clean[1][keep])
    same = (codes.view(torch.uint8) == clean[0].view(torch.uint8)).view(20, 3, 128).all(2)
    assert same[keep.t()].all()
    W = activation(torch, 384, 200, "float16", 2).cuda()
    Y = cq.crossquant_fp8_linear(codes, scale, *cq.crossquant_weight_quantize_fp8(W))
    assert not torch.isfinite(Y[11]).any()
    Y[11] = 0.0
    assert torch.isfinite(Y).all()


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["float16", "bfloat16"])
@pytest.mark.parametrize("I,O", [(1, 1), (128, 128), (127, 5), (129, 130), (256, 384), (300, 1001), (1000, 7), (513, 1288)])
def test_weight_codes(cq, torch, I, O, kind):
    print("weight_quantize_fp8 %d x %d %s" % (I, O, kind), flush=True)
    W = activation(torch, I, O, kind, I + 3 * O) * 0.02
    if I > 200 and O > 200:
        W[128:256, 128:256] = 0.0
    qw, s = cq.crossquant_weight_quantize_fp8(W.cuda())
    q_ref, s_ref = weight_oracle(torch, W)
    assert torch.equal(s.cpu().double(), s_ref)
    assert torch.equal(qw.cpu().double(), q_ref)


# ---- linear ---------------------------------------------------------------------------------------------------

def operands(torch, T, I, O, seed):
    """Random codes and scales straight away (every finite code occurs), on the GPU."""
    g = torch.Generator().manual_seed(seed)
    def codes(n):
        c = torch.randint(0, 256, (n, I), generator=g).to(torch.uint8)
        c[(c & 127) == 127] = 0x38                                             # no NaN
        return c.view(torch.float8_e4m3fn)
    xs = torch.rand((I // 128, T), generator=g) * 0.1 + 0.01
    ws = torch.rand((-(-O // 128), I // 128), generator=g) * 0.001 + 1e-4
    return [v.cuda() for v in (codes(T), xs, codes(O), ws)]


SHAPES = [(1, 128, 1), (1, 1024, 130), (3, 640, 257), (16, 128, 16), (16, 4096, 512), (17, 384, 100), (31, 256, 33), (64, 1152, 300),
          (100, 256, 96), (128, 640, 1000), (129, 128, 128), (200, 896, 515), (255, 512, 2049), (300, 1280, 520), (513, 384, 4100),
          (1030, 256, 260), (2048, 640, 8200), (4096, 256, 4096), (2500, 8192, 640)]


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["float16", "bfloat16"])
@pytest.mark.parametrize("T,I,O", SHAPES)
def test_linear(cq, torch, T, I, O, kind):
    print("fp8_linear %d x %d x %d %s" % (T, I, O, kind), flush=True)
    qx, xs, qw, ws = operands(torch, T, I, O, T + I + O)
    Y = cq.crossquant_fp8_linear(qx, xs, qw, ws, dtype=getattr(torch, kind))
    assert Y.dtype == getattr(torch, kind)
    ref, slack = linear_oracle(qx, xs, qw, ws)
    bad = (Y.double() - ref).abs() > tolerance(ref, slack, kind)
    assert not bad.any(), "%d outputs, the first at %s" % (int(bad.sum()), bad.nonzero()[0].tolist())
    again = cq.crossquant_fp8_linear(qx, xs, qw, ws, dtype=getattr(torch, kind))
    assert torch.equal(Y.view(torch.int16), again.view(torch.int16))


# one for each way to tile a layer that the shapes above leave out: tiles of 16 x 32, 32 x 64 and 64 x 128 in less than a round and with
# ragged ends; 256 x 256 ones of one, two and three blocks of the contraction, with whole tiles alone (number no multiple of 8), with
# halves alone, and with both
@pytest.mark.gpu
@pytest.mark.parametrize("T,I,O,kind", [(1, 384, 8200, "float16"), (5, 512, 11000, "bfloat16"), (17, 384, 8200, "bfloat16"),
                                        (64, 512, 4100, "float16"), (100, 256, 8200, "float16"), (300, 384, 4100, "bfloat16"),
                                        (2000, 128, 11000, "float16"), (1500, 256, 8200, "bfloat16"), (700, 384, 11000, "float16"),
                                        (1000, 1024, 4100, "bfloat16"), (2000, 384, 4100, "float16")])
def test_linear_by_other_tiles(cq, torch, T, I, O, kind):
    test_linear(cq, torch, T, I, O, kind)


# weights of more than 128 MiB
@pytest.mark.gpu
@pytest.mark.parametrize("T,I,O,kind", [(16, 8192, 16400, "bfloat16"), (30, 8192, 16400, "float16"), (60, 8192, 16400, "bfloat16"),
                                        (100, 8192, 16400, "float16"), (5, 131200, 1030, "bfloat16"), (27, 131200, 1030, "float16"),
                                        (50, 131200, 1100, "bfloat16")])
def test_linear_with_large_weights(cq, torch, T, I, O, kind):
    test_linear(cq, torch, T, I, O, kind)


# the same by the tiles that the shapes above leave out: 16 x 16
@pytest.mark.gpu
@pytest.mark.parametrize("T,I,O,kind", [(8, 53248, 2600, "float16"), (1, 65536, 2100, "bfloat16")])
def test_linear_with_large_weights_by_the_smallest_tiles(cq, torch, T, I, O, kind):
    test_linear(cq, torch, T, I, O, kind)


# by 32 x 32 and 64 x 64 tiles (the rows of the list further up whose contraction is 131200 take 16 x 16 ones, and 32 x 32 without
# the non-temporal form)
@pytest.mark.gpu
@pytest.mark.parametrize("T,I,O,kind", [(27, 16512, 8192, "float16"), (32, 59776, 2260, "bfloat16"), (60, 11008, 12300, "float16"), (64, 8320, 16200, "bfloat16")])
def test_linear_with_large_weights_by_middle_tiles(cq, torch, T, I, O, kind):
    test_linear(cq, torch, T, I, O, kind)


@pytest.mark.gpu
@pytest.mark.parametrize("offset,pitch", [(0, 336), (0, 300), (4, 304), (1, 301), (2, 310)])
@pytest.mark.parametrize("T", [5, 70, 260])
def test_linear_into_padded_rows(cq, torch, T, offset, pitch):
    O, I = 300, 384
    qx, xs, qw, ws = operands(torch, T, I, O, 9)
    store = torch.full((T * pitch + 64,), 77.0, dtype=torch.float16, device="cuda")
    Y = store[offset:offset + T * pitch].view(T, pitch)[:, :O]
    cq.crossquant_fp8_linear(qx, xs, qw, ws, Y=Y)
    assert torch.equal(Y, cq.crossquant_fp8_linear(qx, xs, qw, ws))
    untouched = torch.ones_like(store, dtype=torch.bool)
    untouched[offset:offset + T * pitch].view(T, pitch)[:, :O] = False
    assert (store[untouched] == 77.0).all()


# outputs at every alignment, by every way to tile a layer, against those of an aligned buffer; nothing else is written
@pytest.mark.gpu
@pytest.mark.parametrize("extra", [0, 1, 2, 5])
@pytest.mark.parametrize("T,I,O", [(2000, 128, 11001), (1000, 1024, 4102), (513, 384, 4101), (300, 384, 4099), (64, 512, 4103), (17, 384, 8201),
                                   (1, 384, 8203), (4, 256, 70), (16, 2048, 2101)])
def test_linear_into_rows_of_odd_pitch(cq, torch, T, I, O, extra):
    qx, xs, qw, ws = operands(torch, T, I, O, T + O)
    want = torch.empty((T, (O + 7) // 8 * 8), dtype=torch.bfloat16, device="cuda")[:, :O]
    cq.crossquant_fp8_linear(qx, xs, qw, ws, Y=want)
    assert torch.isfinite(want).all()
    pitch = O + extra
    store = torch.full((T * pitch + 64,), 77.0, dtype=torch.bfloat16, device="cuda")
    Y = store[extra:extra + T * pitch].view(T, pitch)[:, :O]
    cq.crossquant_fp8_linear(qx, xs, qw, ws, Y=Y)
    assert torch.equal(Y, want)
    store[extra:extra + T * pitch].view(T, pitch)[:, :O] = 77.0
    assert (store == 77.0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 40, 300])
def test_linear_at_the_ends_of_the_formats(cq, torch, T):
    """Scales near the ends of binary32, results past binary16 (infinite) and below it, zero scales."""
    I, O = 256, 140
    qx, xs, qw, ws = operands(torch, T, I, O, 3)
    xs[:, 0] = 0.0
    assert (cq.crossquant_fp8_linear(qx, xs, qw, ws)[0] == 0).all()
    xs.fill_(2.0 ** -60)
    ws.fill_(2.0 ** 60)
    ref, slack = linear_oracle(qx, xs, qw, ws)
    Y = cq.crossquant_fp8_linear(qx, xs, qw, ws, dtype=torch.bfloat16)
    assert ((Y.double() - ref).abs() <= tolerance(ref, slack, "bfloat16")).all()
    Y16 = cq.crossquant_fp8_linear(qx, xs, qw, ws)
    over = ref.abs() > 65600.0
    assert over.any() and torch.isinf(Y16[over]).all()
    ws.fill_(2.0 ** -60)
    assert (cq.crossquant_fp8_linear(qx, xs, qw, ws) == 0).all()


@pytest.mark.gpu
def test_layer_on_another_stream_and_captured(cq, torch):
    """quantize_fp8 and fp8_linear captured into one graph, replayed with new inputs between eager calls, and on a side stream."""
    T, I, O = 70, 700, 520
    W = activation(torch, I, O, "float16", 4).cuda() * 0.05
    qw, ws = cq.crossquant_weight_quantize_fp8(W)
    X = torch.zeros((T, I), dtype=torch.float16, device="cuda")
    codes = torch.empty((T, 768), dtype=torch.float8_e4m3fn, device="cuda")
    scale = torch.empty((6, T), device="cuda")
    Y = torch.empty((T, O), dtype=torch.float16, device="cuda")

    def layer():
        cq.crossquant_quantize_fp8(X, codes=codes, scale=scale)
        cq.crossquant_fp8_linear(codes, scale, qw, ws, Y=Y)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer()
    for seed in range(3):
        X.copy_(activation(torch, T, I, "float16", seed))
        graph.replay()
        torch.cuda.synchronize()
        got = Y.clone()
        want = cq.crossquant_fp8_linear(*cq.crossquant_quantize_fp8(X), qw, ws)
        assert torch.equal(got, want)
        with torch.cuda.stream(side):
            side.wait_stream(torch.cuda.current_stream())
            layer()
        side.synchronize()
        assert torch.equal(Y, want)


# ---- refusals (no GPU) ------------------------------------------------------------------------------------------

P = 0x10000


def test_quantizer_argument_errors(cq):
    def call(X=P, kind=0, T=4, I=8, ldx=8, codes=P, scale=P):
        return cq.raw.crossquant_quantize_fp8(X, kind, T, I, ldx, codes, scale, None)
    assert call(X=0) == -1 and call(codes=0) == -1 and call(scale=0) == -1
    assert call(T=0) == -2 and call(I=0) == -2 and call(ldx=7) == -2 and call(T=1 << 25) == -2
    assert call(kind=2) == -9 and call(kind=-1) == -9
    assert call(X=P + 1) == -5 and call(codes=P + 8) == -5 and call(scale=P + 2) == -5

    def weight(W=P, kind=1, I=4, O=8, qw=P, s=P):
        return cq.raw.crossquant_weight_quantize_fp8(W, kind, I, O, qw, s, None)
    assert weight(W=0) == -1 and weight(qw=0) == -1 and weight(s=0) == -1
    assert weight(I=0) == -2 and weight(O=0) == -2 and weight(kind=3) == -9 and weight(qw=P + 4) == -5


def test_linear_argument_errors(cq):
    def call(qx=P, xs=P, qw=P, ws=P, T=4, I=128, O=8, Y=P, kind=0, ldy=8):
        return cq.raw.crossquant_fp8_linear(qx, xs, qw, ws, T, I, O, Y, kind, ldy, None)
    for name in ("qx", "xs", "qw", "ws", "Y"):
        assert call(**{name: 0}) == -1
    assert call(T=0) == -2 and call(O=0) == -2 and call(I=0) == -2 and call(ldy=7) == -2 and call(T=1 << 25) == -2
    assert call(I=64) == -6 and call(I=129) == -6
    assert call(kind=2) == -9
    assert call(qx=P + 8) == -5 and call(qw=P + 1) == -5 and call(xs=P + 2) == -5 and call(Y=P + 1) == -5
    assert "binary16" in cq.crossquant_status_string(-9)


def test_wrappers_check_what_they_are_given(cq, torch):
    X = torch.zeros((4, 130), dtype=torch.float16)
    e4 = lambda *s: torch.zeros(s, dtype=torch.uint8).view(torch.float8_e4m3fn)
    with pytest.raises(ValueError, match="GPU"):
        cq.crossquant_quantize_fp8(X)
    with pytest.raises(TypeError):
        cq.crossquant_quantize_fp8(X.float())
    with pytest.raises(ValueError, match="codes must have shape"):
        cq.crossquant_quantize_fp8(X, codes=e4(4, 130))
    with pytest.raises(ValueError, match="scale must have shape"):
        cq.crossquant_quantize_fp8(X, scale=torch.zeros((4, 2)))
    with pytest.raises(ValueError, match="unit stride"):
        cq.crossquant_quantize_fp8(torch.zeros((130, 4), dtype=torch.float16).t())
    with pytest.raises(ValueError, match="contiguous"):
        cq.crossquant_weight_quantize_fp8(X.t())
    with pytest.raises(ValueError, match="w_scale must have shape"):
        cq.crossquant_weight_quantize_fp8(X, w_scale=torch.zeros((1, 2)))
    with pytest.raises(ValueError, match="GPU"):
        cq.crossquant_weight_quantize_fp8(X)
    qx, xs, qw, ws = e4(4, 256), torch.zeros((2, 4)), e4(130, 256), torch.zeros((2, 2))
    with pytest.raises(ValueError, match="GPU"):
        cq.crossquant_fp8_linear(qx, xs, qw, ws)
    with pytest.raises(ValueError, match="x_scale must have shape"):
        cq.crossquant_fp8_linear(qx, xs.t().contiguous(), qw, ws)
    with pytest.raises(ValueError, match="w_scale must have shape"):
        cq.crossquant_fp8_linear(qx, xs, qw, torch.zeros((130, 2)))
    with pytest.raises(ValueError, match="contraction lengths"):
        cq.crossquant_fp8_linear(qx, xs, e4(130, 128), ws)
    with pytest.raises(cq.CrossQuantError) as e:
        cq.crossquant_fp8_linear(e4(4, 130), xs, e4(130, 130), ws)
    assert e.value.status == -6
    with pytest.raises(TypeError, match="float16 or bfloat16"):
        cq.crossquant_fp8_linear(qx, xs, qw, ws, dtype=torch.float32)
    with pytest.raises(ValueError, match="Y must be"):
        cq.crossquant_fp8_linear(qx, xs, qw, ws, Y=torch.zeros((4, 129), dtype=torch.float16))
    with pytest.raises(ValueError, match="Y must be"):
        cq.crossquant_fp8_linear(qx, xs, qw, ws, Y=torch.zeros((4, 130), dtype=torch.float16), dtype=torch.bfloat16)
    with pytest.raises(TypeError):
        cq.crossquant_fp8_linear(qx.view(torch.uint8), xs, qw, ws)
