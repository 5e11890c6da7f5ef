"""GPU parity of the 8-bit linear layer with the float64 oracle.

The 8-bit forms are exact: codes and scale bytes have to be the oracle's.  Products: a product of two 8-bit values under their
scales is exact in float32, so what is off is the float32 sum of K products (at most K additions, each off by at most 2^-23 of the
sum of magnitudes A = sum |a b| where it truncates) and the rounding to bf16 (2^-8 of the value): |y - y_ref| <= 2^-8 |y_ref| + 1.01 K 2^-23 A.
The bias adds one more float32 rounding of |y| (counted with the K).  GELU has slope below 1.13 and the kernels' own form of it is off by
at most 2e-6 plus a few float32 roundings: 1.13 times the error before it, plus 4e-6 (1 + |x|), plus the rounding to bf16.
Column sums: rows - 1 float32 additions, each off by half a place: rows 2^-24 sum |x|.
"""
import numpy as np
import pytest
import torch
from math import erf

import paper_2009_08065_b200 as bsp
from oracle import fp8_oracle as F
from gpu_util import DEV, bf16_bits_to_f64, bits_of, to_dev

pytestmark = pytest.mark.gpu
PAD = 0x5A
FORMATS = [F.E4M3, F.E5M2]


def bf16_bits(x):
    u = np.ascontiguousarray(x, dtype=np.float32).view(np.uint32).astype(np.uint64)
    return ((u + 0x7FFF + ((u >> 16) & 1)) >> 16).astype(np.uint16)


def random_matrix(rng, rows, cols, spread=3.0):
    """bf16 bits of values of very different sizes, zeros, a row and a column of zeros among them."""
    x = rng.normal(size=(rows, cols)) * np.exp(rng.normal(size=(rows, 1)) * spread) * (rng.random((rows, cols)) < 0.9)
    if rows > 2:
        x[rows // 2] = 0.0
    if cols > 2:
        x[:, cols // 3] = 0.0
    return bf16_bits(x)


class Padded:
    """A device matrix with columns of a pattern behind its own, which have to stay."""

    def __init__(self, rows, cols, ld, dtype=torch.uint8, fill=PAD):
        self.whole = torch.full((rows, ld), fill, dtype=dtype, device=DEV)
        self.fill, self.t = fill, self.whole[:, :cols]

    def host(self):
        assert bool((self.whole[:, self.t.shape[1]:] == self.fill).all()), "columns behind the matrix were written"
        return self.t.cpu().numpy()


def up(n, a):
    return (n + a - 1) // a * a


def widened(bits, ld):
    """bf16 bits on the device with leading dimension ld."""
    wide = np.zeros((bits.shape[0], ld), dtype=np.uint16)
    wide[:, :bits.shape[1]] = bits
    return to_dev(wide)[:, :bits.shape[1]]


def codes(q, s, ld, scales_ld=None):
    """Codes and scales on the device, codes with leading dimension ld and NaN codes behind the rows."""
    whole = torch.full((q.shape[0], ld), 0x7F, dtype=torch.uint8, device=DEV)
    whole[:, :q.shape[1]] = torch.from_numpy(q).to(DEV)
    ws = torch.full((s.shape[0], scales_ld or s.shape[1]), 0xFF, dtype=torch.uint8, device=DEV)
    ws[:, :s.shape[1]] = torch.from_numpy(s).to(DEV)
    return whole[:, :q.shape[1]], ws[:, :s.shape[1]]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 0), (1, 128, 0), (5, 130, 6), (128, 128, 0), (129, 257, 7), (300, 520, 8), (257, 1000, 0), (40, 4096, 16)])
def test_quantize(rows, cols, pad, fmt):
    rng = np.random.default_rng(rows * 1000 + cols)
    bits = random_matrix(rng, rows, cols)
    x = bf16_bits_to_f64(bits)
    X = widened(bits, cols + pad)
    kb, rb = up(cols, 128) // 128, up(rows, 128) // 128
    Q, S = Padded(rows, cols, cols + pad), Padded(rows, kb, kb + 3)
    Qc, Sc = Padded(rows, cols, cols + 2 * pad), Padded(rb, cols, cols + 5)
    sums, ws = torch.empty(cols, dtype=torch.float32, device=DEV), torch.empty(rb * cols * 4, dtype=torch.uint8, device=DEV)
    bsp.bsp_fp8_quantize(X, fmt, Q.t, S.t, Qc.t, Sc.t, sums, ws)
    q, s = F.quantize(x, 1, 128, fmt)
    qc, sc = F.quantize(x, 128, 1, fmt)
    assert np.array_equal(S.host(), s) and np.array_equal(Q.host(), q)
    assert np.array_equal(Sc.host(), sc) and np.array_equal(Qc.host(), qc)
    assert (np.abs(sums.cpu().numpy() - x.sum(0)) <= rows * 2.0 ** -24 * np.abs(x).sum(0)).all()
    # each form by itself
    for kw, a, b, ref, refs in ((dict(), Q, S, q, s), (dict(Qc=Qc.t, Sc=Sc.t), Qc, Sc, qc, sc)):
        a.t.fill_(1)
        b.t.fill_(1)
        bsp.bsp_fp8_quantize(X, fmt, **(kw or dict(Q=Q.t, S=S.t)))
        assert np.array_equal(a.host(), ref) and np.array_equal(b.host(), refs)
    sums.fill_(0)
    bsp.bsp_fp8_quantize(X, fmt, col_sums=sums, ws=ws)
    assert (np.abs(sums.cpu().numpy() - x.sum(0)) <= rows * 2.0 ** -24 * np.abs(x).sum(0)).all()


@pytest.mark.parametrize("n,k,pad", [(1, 1, 0), (128, 128, 0), (130, 257, 7), (96, 1000, 8), (300, 520, 0)])
def test_quantize_weight(n, k, pad):
    rng = np.random.default_rng(n + k)
    bits = random_matrix(rng, n, k, 0.5)
    if n > 128:
        bits[128:, :min(k, 128)] = 0                                  # a whole block of zeros
    Q, S = Padded(n, k, k + pad), Padded(up(n, 128) // 128, up(k, 128) // 128, up(k, 128) // 128 + 1)
    bsp.bsp_fp8_quantize_weight(widened(bits, k + pad), Q.t, S.t)
    q, s = F.quantize(bf16_bits_to_f64(bits), 128, 128, F.E4M3)
    assert np.array_equal(S.host(), s) and np.array_equal(Q.host(), q)


@pytest.mark.parametrize("fmt", FORMATS)
def test_quantize_what_is_not_finite(fmt):
    """Infinities and NaN reach their blocks and no others; the smallest and largest magnitudes of bf16."""
    x = np.ones((130, 260), dtype=np.float32)
    x[3, 5], x[70, 200], x[129, 259] = np.inf, np.nan, -np.inf
    x[10] = 1e-40
    x[11] = 3.3e38
    x[12] = -0.0
    bits = bf16_bits(x)
    bits[70, 200] = 0xFFC1
    ref = bf16_bits_to_f64(bits)
    Q, S, Qc, Sc = Padded(130, 260, 264), Padded(130, 3, 3), Padded(130, 260, 264), Padded(2, 260, 260)
    bsp.bsp_fp8_quantize(to_dev(bits), fmt, Q.t, S.t, Qc.t, Sc.t)
    for got, scales, want in ((Q, S, F.quantize(ref, 1, 128, fmt)), (Qc, Sc, F.quantize(ref, 128, 1, fmt))):
        assert np.array_equal(scales.host(), want[1]) and np.array_equal(got.host(), want[0])
    Wq, WS = Padded(130, 260, 264), Padded(2, 3, 3)
    bsp.bsp_fp8_quantize_weight(to_dev(bits), Wq.t, WS.t)
    want = F.quantize(ref, 128, 128, F.E4M3)
    assert np.array_equal(WS.host(), want[1]) and np.array_equal(Wq.host(), want[0])


def check(y_bits, a, b, bias=None, act=bsp.ACT_NONE, mask=None, what=""):
    """y against a b^T for float64 a [rows, K], b [cols, K]."""
    ref, mag = a @ b.T, np.abs(a) @ np.abs(b).T
    terms = a.shape[1]
    if bias is not None:
        ref, mag, terms = ref + bias, mag + np.abs(bias), terms + 1
    err = 1.01 * terms * 2.0 ** -23 * mag
    if act == bsp.ACT_GELU:
        err = 1.13 * err + 4e-6 * (1 + np.abs(ref))
        ref = ref * 0.5 * (1 + np.vectorize(erf)(ref / np.sqrt(2.0)))
    if mask is not None:
        ref, err = ref * mask, err * mask
        assert not y_bits[~mask].any(), f"{what}: pruned outputs are +0"
    y = bf16_bits_to_f64(y_bits)
    off = np.abs(y - ref) - (2.0 ** -8 * np.abs(ref) + err + 1e-37)
    assert np.isfinite(y).all() and (off <= 0).all(), f"{what}: off by {off.max()} more than allowed at {np.unravel_index(off.argmax(), off.shape)}"


class Layer:
    def __init__(self, t, n, k, seed, fmt=F.E4M3, ld_align=16, out_align=8, block=1):
        rng = np.random.default_rng(seed)
        self.t, self.n, self.k, self.fmt, self.block = t, n, k, fmt, block
        self.x_bits, self.dy_bits = random_matrix(rng, t, k, 1.0), random_matrix(rng, t, n, 1.0)
        self.keep = (rng.random((n // block, k)) < 0.4).astype(np.uint8)
        self.keep[0] = 0
        self.mask = np.repeat(self.keep, block, 0).astype(bool)
        w = bf16_bits_to_f64(bf16_bits(0.02 * rng.normal(size=(n, k)))) * self.mask
        self.bias_bits = bf16_bits(rng.normal(size=n) * 0.1)
        self.wq, self.wsc = F.quantize(w, 128, 128, F.E4M3)
        self.w = F.dequantize(self.wq, self.wsc, 128, 128, F.E4M3)
        self.Wq, self.WS = codes(self.wq, self.wsc, up(k, ld_align) if ld_align else k + 1, self.wsc.shape[1] + 1)
        self.al, self.out_align = ld_align, out_align

    def ld(self, n):
        return up(n, self.al) if self.al else n + 1

    def out(self, rows, cols):
        return Padded(rows, cols, up(cols, self.out_align) + self.out_align, torch.int16, 0x7FC0)

    def rows_form(self, bits, fmt):
        q, s = F.quantize(bf16_bits_to_f64(bits), 1, 128, fmt)
        return F.dequantize(q, s, 1, 128, fmt), codes(q, s, self.ld(q.shape[1]), s.shape[1] + 1)

    def cols_form(self, bits, fmt):
        q, s = F.quantize(bf16_bits_to_f64(bits), 128, 1, fmt)
        return F.dequantize(q, s, 128, 1, fmt), codes(q, s, self.ld(q.shape[1]), s.shape[1] + 1)

    def forward(self, act):
        x, (Xq, XS) = self.rows_form(self.x_bits, self.fmt)
        Y = self.out(self.t, self.n)
        bsp.bsp_linear_fp8_quantized(self.Wq, self.WS, Xq, XS, self.fmt, to_dev(self.bias_bits), act, Y.t)
        bsp.bsp_linear_status()
        check(Y.host().view(np.uint16), x, self.w, bf16_bits_to_f64(self.bias_bits), act, what="forward")

    def backward_input(self):
        dy, (Yq, YS) = self.rows_form(self.dy_bits, self.fmt)
        dX = self.out(self.t, self.k)
        bsp.bsp_linear_fp8_backward_input(self.Wq, self.WS, Yq, YS, self.fmt, dX.t)
        bsp.bsp_linear_status()
        check(dX.host().view(np.uint16), dy, self.w.T, what="dX")

    def backward_weight(self, masked):
        dy, (Yq, YS) = self.cols_form(self.dy_bits, self.fmt)
        x, (Xq, XS) = self.cols_form(self.x_bits, F.E4M3)
        dW = self.out(self.n, self.k)
        keep = torch.from_numpy(self.keep).to(DEV) if masked else None
        bsp.bsp_linear_fp8_backward_weight(Yq, YS, self.fmt, Xq, XS, F.E4M3, self.block, keep, dW.t)
        bsp.bsp_linear_status()
        check(dW.host().view(np.uint16), dy.T, x.T, mask=self.mask if masked else None, what="dW")


# (rows that begin anywhere go through the plain kernel, the others through the tensor cores)
ANY = [(1, 1, 1, 1), (3, 5, 7, 1), (65, 66, 130, 3), (130, 67, 129, 1), (70, 257, 300, 1)]
TENSOR = [(1, 1, 1, 1), (1, 128, 128, 8), (7, 8, 130, 1), (128, 128, 512, 16), (129, 130, 513, 10), (300, 257, 1000, 1), (257, 520, 136, 8), (1000, 96, 256, 12),
          (64, 2000, 1288, 16), (513, 1288, 640, 8)]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("t,n,k,block", ANY)
def test_products_any_alignment(t, n, k, block, fmt):
    layer = Layer(t, n, k, t + n + k, fmt, ld_align=0, out_align=1, block=block)
    layer.forward(bsp.ACT_GELU)
    layer.backward_input()
    layer.backward_weight(True)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("t,n,k,block", TENSOR)
def test_forward(t, n, k, block, fmt):
    layer = Layer(t, n, k, t + n + k, fmt, block=block)
    layer.forward(bsp.ACT_NONE)
    layer.forward(bsp.ACT_GELU)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("t,n,k,block", TENSOR)
def test_backward_input(t, n, k, block, fmt):
    Layer(t, n, k, t + n + k, fmt, block=block).backward_input()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("t,n,k,block", TENSOR)
def test_backward_weight(t, n, k, block, fmt):
    layer = Layer(t, n, k, t + n + k, fmt, block=block)
    layer.backward_weight(False)
    layer.backward_weight(True)


# Many output tiles (pairs of CTAs), few of them (clusters that share the contraction), contractions of one block to some 260, and whose
# parts are more blocks than a CTA has stages or carries scales for at a time.
LONG = [(1300, 1100, 1050, 10), (40, 96, 33000, 8), (100, 128, 30000, 16), (100, 30000, 128, 16), (9000, 96, 130, 8), (1000, 1000, 1200, 8),
        (33, 1024, 1024, 8), (128, 768, 2300, 8), (200, 70, 5000, 10), (2300, 260, 200, 4)]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("t,n,k,block", LONG)
def test_few_and_many_tiles(t, n, k, block, fmt):
    layer = Layer(t, n, k, t + n + k, fmt, block=block)
    layer.forward(bsp.ACT_GELU if k < 2000 else bsp.ACT_NONE)
    layer.backward_input()
    layer.backward_weight(True)


@pytest.mark.parametrize("t,n,k", [(3, 256, 512), (40, 256, 512), (128, 512, 2304), (700, 1100, 700)])
def test_weight_written_just_before(t, n, k):
    """The weight is quantised anew ahead of every call, with nothing between them; so are X and the workspace used again."""
    rng = np.random.default_rng(9)
    weights = [to_dev(bf16_bits(rng.normal(size=(n, k)) * 2.0 ** i)) for i in range(4)]
    X, bias = to_dev(random_matrix(rng, t, k, 1.0)), to_dev(bf16_bits(rng.normal(size=n)))
    ws = torch.empty(bsp.bsp_linear_fp8_ws_bytes(t, k), dtype=torch.uint8, device=DEV)
    Wq, WS = torch.empty((n, up(k, 16)), dtype=torch.uint8, device=DEV)[:, :k], torch.empty((up(n, 128) // 128, up(k, 128) // 128), dtype=torch.uint8, device=DEV)
    out = [torch.zeros((t, n), dtype=torch.int16, device=DEV) for _ in range(64)]
    ref = []
    for W in weights:
        bsp.bsp_fp8_quantize_weight(W, Wq, WS)
        torch.cuda.synchronize()
        bsp.bsp_linear_fp8(Wq, WS, X, bias, bsp.ACT_NONE, out[0], ws)
        torch.cuda.synchronize()
        ref.append(out[0].clone())
    torch.cuda.synchronize()
    for i, Y in enumerate(out):
        bsp.bsp_fp8_quantize_weight(weights[i % 4], Wq, WS)
        bsp.bsp_linear_fp8(Wq, WS, X, bias, bsp.ACT_NONE, Y, ws)
    bsp.bsp_linear_status()
    for i, Y in enumerate(out):
        assert torch.equal(Y, ref[i % 4]), i


def test_weight_written_just_before_in_a_graph():
    """The same in a captured graph, two layers of different routes one after the other, replayed with other weights in the same place."""
    rng = np.random.default_rng(10)
    shapes = [(40, 256, 512), (128, 512, 2304)]
    layers = []
    for t, n, k in shapes:
        layers.append(dict(
            W=to_dev(bf16_bits(rng.normal(size=(n, k)))), X=to_dev(random_matrix(rng, t, k, 1.0)),
            ws=torch.empty(bsp.bsp_linear_fp8_ws_bytes(t, k), dtype=torch.uint8, device=DEV), Wq=torch.empty((n, k), dtype=torch.uint8, device=DEV),
            WS=torch.empty((up(n, 128) // 128, up(k, 128) // 128), dtype=torch.uint8, device=DEV),
            Y=[torch.zeros((t, n), dtype=torch.int16, device=DEV) for _ in range(4)]))

    def step():
        for i in range(4):
            for L in layers:
                bsp.bsp_fp8_quantize_weight(L["W"], L["Wq"], L["WS"])
                bsp.bsp_linear_fp8(L["Wq"], L["WS"], L["X"], None, bsp.ACT_NONE, L["Y"][i], L["ws"])

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in range(5):
        new = [to_dev(bf16_bits(np.random.default_rng(seed).normal(size=L["W"].shape) * 2.0 ** seed)) for L in layers]
        for L, w in zip(layers, new):
            L["W"].copy_(w)
        graph.replay()
        bsp.bsp_linear_status()
        got = [[y.clone() for y in L["Y"]] for L in layers]
        for L, ys in zip(layers, got):
            bsp.bsp_fp8_quantize_weight(L["W"], L["Wq"], L["WS"])
            torch.cuda.synchronize()
            bsp.bsp_linear_fp8(L["Wq"], L["WS"], L["X"], None, bsp.ACT_NONE, L["Y"][0], L["ws"])
            torch.cuda.synchronize()
            assert all(torch.equal(y, L["Y"][0]) for y in ys)


def test_the_same_bits_every_time():
    """Split contractions are added in a fixed order, whichever CTA is ready first."""
    layer = Layer(130, 512, 4096, 3)
    _, (Xq, XS) = layer.rows_form(layer.x_bits, layer.fmt)
    runs = []
    for _ in range(20):
        Y = layer.out(130, 512)
        bsp.bsp_linear_fp8_quantized(layer.Wq, layer.WS, Xq, XS, layer.fmt, None, bsp.ACT_NONE, Y.t)
        runs.append(Y)
    bsp.bsp_linear_status()
    assert all(np.array_equal(r.host(), runs[0].host()) for r in runs)


@pytest.mark.parametrize("t,n,k", [(1, 16, 128), (1, 1, 1), (1, 1000, 1000), (2, 130, 257), (7, 96, 100), (8, 64, 4096), (9, 200, 384), (15, 257, 1288), (16, 48, 130),
                                   (17, 40, 520), (31, 100, 136), (32, 256, 1024), (33, 128, 256), (64, 520, 768), (200, 130, 1000)])
@pytest.mark.parametrize("pad", [0, 3])
def test_linear(t, n, k, pad):
    """bf16 activations straight in, few and many tokens; pad: rows of X and Y that begin anywhere."""
    layer = Layer(t, n, k, t + n + k)
    x, _ = layer.rows_form(layer.x_bits, F.E4M3)
    ws = torch.empty(bsp.bsp_linear_fp8_ws_bytes(t, k), dtype=torch.uint8, device=DEV)
    X = widened(layer.x_bits, up(k, 8) + pad)
    for act, bias in ((bsp.ACT_NONE, None), (bsp.ACT_GELU, layer.bias_bits)):
        Y = Padded(t, n, up(n, 8) + pad, torch.int16, 0x7FC0)
        bsp.bsp_linear_fp8(layer.Wq, layer.WS, X, None if bias is None else to_dev(bias), act, Y.t, ws)
        bsp.bsp_linear_status()
        check(Y.host().view(np.uint16), x, layer.w, None if bias is None else bf16_bits_to_f64(bias), act, what="linear")


@pytest.mark.parametrize("t", [2, 40, 300])
def test_nan_stays_in_its_token(t):
    layer = Layer(t, 96, 300, 5)
    layer.x_bits[1, 200] = 0x7F80                                      # an infinity
    ws = torch.empty(bsp.bsp_linear_fp8_ws_bytes(t, 300), dtype=torch.uint8, device=DEV)
    Y = layer.out(t, 96)
    bsp.bsp_linear_fp8(layer.Wq, layer.WS, widened(layer.x_bits, 304), None, bsp.ACT_NONE, Y.t, ws)
    bsp.bsp_linear_status()
    y = bf16_bits_to_f64(Y.host().view(np.uint16))
    assert np.isnan(y[1]).all() and np.isfinite(np.delete(y, 1, 0)).all()


def test_scales_of_any_size():
    """Weights and activations whose scales lie far apart: every block's own scale is used, along rows and along columns."""
    t, n, k = 200, 260, 700
    rng = np.random.default_rng(9)
    x = rng.normal(size=(t, k)) * 2.0 ** rng.integers(-30, 30, size=(t, 6)).repeat(128, 1)[:, :k]
    w = rng.normal(size=(n, k)) * 2.0 ** rng.integers(-30, 30, size=(3, 6)).repeat(128, 0)[:n].repeat(128, 1)[:, :k]
    layer = Layer(t, n, k, 9)
    layer.x_bits = bf16_bits(x)
    layer.wq, layer.wsc = F.quantize(bf16_bits_to_f64(bf16_bits(w)), 128, 128, F.E4M3)
    layer.w = F.dequantize(layer.wq, layer.wsc, 128, 128, F.E4M3)
    layer.Wq, layer.WS = codes(layer.wq, layer.wsc, up(k, 16))
    layer.forward(bsp.ACT_NONE)
    layer.backward_input()
    layer.backward_weight(False)


def test_binding_refuses_other_shapes_and_types():
    layer = Layer(9, 40, 200, 1)
    X, Y = widened(layer.x_bits, 200), torch.zeros((9, 40), dtype=torch.int16, device=DEV)
    ws = torch.empty(bsp.bsp_linear_fp8_ws_bytes(9, 200), dtype=torch.uint8, device=DEV)
    call = lambda **c: bsp.bsp_linear_fp8(**{**dict(Wq=layer.Wq, WS=layer.WS, X=X, bias=None, act=0, Y=Y, ws=ws), **c})  # noqa: E731
    call()
    for c in (dict(X=X[:, :199]), dict(Y=Y[:8]), dict(Y=Y.float()), dict(WS=layer.WS[:, :1]), dict(X=X.float()), dict(bias=torch.zeros(39, dtype=torch.int16, device=DEV)),
              dict(Wq=layer.Wq.to(torch.int16))):
        with pytest.raises(ValueError):
            call(**c)
    with pytest.raises(bsp.BspError) as e:
        call(ws=ws[:100])
    assert e.value.status == -3
    with pytest.raises(ValueError):
        bsp.bsp_fp8_quantize(X, 0, torch.zeros((9, 200), dtype=torch.uint8, device=DEV), torch.zeros((9, 1), dtype=torch.uint8, device=DEV))


@pytest.mark.parametrize("t", [5, 300])
def test_captured_and_on_another_stream(t):
    """The calls of a training step, captured on one stream and replayed on new inputs while another stream runs the same step with its own
    buffers: both get what single calls give."""
    n, k, block = 264, 400, 8
    layer = Layer(t, n, k, 17, block=block)
    keep = torch.from_numpy(layer.keep).to(DEV)
    inputs = [(widened(Layer(t, n, k, s, block=block).x_bits, k), widened(Layer(t, n, k, s, block=block).dy_bits, n)) for s in (21, 22, 23)]

    def buffers():
        u8 = lambda r, c: torch.zeros((r, up(c, 16)), dtype=torch.uint8, device=DEV)[:, :c]  # noqa: E731
        i16 = lambda r, c: torch.zeros((r, c), dtype=torch.int16, device=DEV)  # noqa: E731
        b = up(t, 128) // 128
        return dict(xr=u8(t, k), xc=u8(t, k), yr=u8(t, n), yc=u8(t, n), xrs=u8(t, up(k, 128) // 128), xcs=u8(b, k), yrs=u8(t, up(n, 128) // 128), ycs=u8(b, n),
                    X=i16(t, k), dY=i16(t, n), Y=i16(t, n), dX=i16(t, k), dW=i16(n, k), db=torch.zeros(n, dtype=torch.float32, device=DEV),
                    ws=torch.empty(b * n * 4, dtype=torch.uint8, device=DEV))

    def step(b):
        bsp.bsp_fp8_quantize(b["X"], F.E4M3, b["xr"], b["xrs"], b["xc"], b["xcs"])
        bsp.bsp_linear_fp8_quantized(layer.Wq, layer.WS, b["xr"], b["xrs"], F.E4M3, None, bsp.ACT_NONE, b["Y"])
        bsp.bsp_fp8_quantize(b["dY"], F.E5M2, b["yr"], b["yrs"], b["yc"], b["ycs"], b["db"], b["ws"])
        bsp.bsp_linear_fp8_backward_input(layer.Wq, layer.WS, b["yr"], b["yrs"], F.E5M2, b["dX"])
        bsp.bsp_linear_fp8_backward_weight(b["yc"], b["ycs"], F.E5M2, b["xc"], b["xcs"], F.E4M3, block, keep, b["dW"])
        return b

    def fill(b, i):
        b["X"].copy_(inputs[i][0])
        b["dY"].copy_(inputs[i][1])
        return b

    names = ("Y", "dX", "dW", "db")
    want = []
    for i in range(3):
        b = step(fill(buffers(), i))
        torch.cuda.synchronize()
        want.append({k: b[k].clone() for k in names})
    a, c = buffers(), buffers()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(a)
    side = torch.cuda.Stream()
    for i in range(3):
        fill(a, i)
        fill(c, 2 - i)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            for _ in range(3):
                step(c)
        graph.replay()
        torch.cuda.synchronize()
        for k in names:
            assert torch.equal(a[k], want[i][k]), k
            assert torch.equal(c[k], want[2 - i][k]), k
    bsp.bsp_linear_status()
    graph.reset()


@pytest.mark.parametrize("block,t", [(16, 200), (1, 33)])
def test_retraining_in_8_bits(block, t):
    """The operators as a retraining loop uses them: prune, quantise the masked weight, forward and backward in 8 bits, the weight gradient
    and bias gradient into one Adam step with 8-bit moments, whose bf16 copy is quantised for the next forward.  Two iterations; every piece against the oracle."""
    n, k = 96, 200
    rng = np.random.default_rng(block)
    w = 0.02 * rng.normal(size=(n, k))
    keep_np = (rng.random((n // block, k)) < 0.4).astype(np.uint8)
    keep_np[0] = 0
    mask = np.repeat(keep_np, block, 0).astype(bool)
    W = torch.from_numpy((w * mask).astype(np.float32)).to(DEV)
    b = torch.zeros((1, n), dtype=torch.float32, device=DEV)
    Wb, bb = torch.zeros((n, k), dtype=torch.int16, device=DEV), torch.zeros((1, n), dtype=torch.int16, device=DEV)
    keep = torch.from_numpy(keep_np).to(DEV)
    state = lambda r, c: dict(m=torch.zeros((r, c), dtype=torch.uint8, device=DEV), v=torch.zeros((r, c), dtype=torch.uint8, device=DEV),  # noqa: E731
                              m_scale=torch.zeros((r, up(c, 128) // 128), dtype=torch.uint8, device=DEV), v_scale=torch.zeros((r, up(c, 128) // 128), dtype=torch.uint8, device=DEV))
    dW, db = torch.zeros((n, k), dtype=torch.int16, device=DEV), torch.zeros((1, n), dtype=torch.float32, device=DEV)
    jobs = bsp.make_adam_job_array([bsp.AdamJob(W=W, grad=dW, lr=1e-3, weight_decay=0.01, keep=keep, block=block, W_bf16=Wb, **state(n, k)),
                                    bsp.AdamJob(W=b, grad=db, lr=1e-3, W_bf16=bb, **state(1, n))])
    Wb.copy_(torch.from_numpy(bf16_bits(w * mask).view(np.int16)))
    kb, nb, tb = up(k, 128) // 128, up(n, 128) // 128, up(t, 128) // 128
    u8 = lambda r, c: torch.zeros((r, up(c, 16)), dtype=torch.uint8, device=DEV)[:, :c]  # noqa: E731
    Wq, WS = u8(n, k), u8(nb, kb)
    xr, xc, yr, yc, xrs, xcs, yrs, ycs = u8(t, k), u8(t, k), u8(t, n), u8(t, n), u8(t, kb), u8(tb, k), u8(t, nb), u8(tb, n)
    ws = torch.empty(tb * n * 4, dtype=torch.uint8, device=DEV)
    Y, dX = torch.zeros((t, n), dtype=torch.int16, device=DEV), torch.zeros((t, k), dtype=torch.int16, device=DEV)
    for step in (1, 2):
        w_bits, b_bits = bits_of(Wb), bits_of(bb)[0]
        x_bits, dy_bits = random_matrix(rng, t, k, 1.0), random_matrix(rng, t, n, 1.0)
        bsp.bsp_fp8_quantize_weight(Wb, Wq, WS)
        bsp.bsp_fp8_quantize(to_dev(x_bits), F.E4M3, xr, xrs, xc, xcs)
        bsp.bsp_linear_fp8_quantized(Wq, WS, xr, xrs, F.E4M3, bb[0], bsp.ACT_NONE, Y)
        bsp.bsp_fp8_quantize(to_dev(dy_bits), F.E5M2, yr, yrs, yc, ycs, db[0], ws)
        bsp.bsp_linear_fp8_backward_input(Wq, WS, yr, yrs, F.E5M2, dX)
        bsp.bsp_linear_fp8_backward_weight(yc, ycs, F.E5M2, xc, xcs, F.E4M3, block, keep, dW)
        before = W.cpu().numpy()
        bsp.bsp_masked_adam_step_batched(jobs, 0.9, 0.999, 1e-8, step, 7)
        bsp.bsp_linear_status()
        form = lambda bits, rows, cols, fmt: F.dequantize(*F.quantize(bf16_bits_to_f64(bits), rows, cols, fmt), rows, cols, fmt)  # noqa: E731
        w8 = form(w_bits, 128, 128, F.E4M3)
        check(bits_of(Y), form(x_bits, 1, 128, F.E4M3), w8, bf16_bits_to_f64(b_bits), what="Y")
        check(bits_of(dX), form(dy_bits, 1, 128, F.E5M2), w8.T, what="dX")
        check(bits_of(dW), form(dy_bits, 128, 1, F.E5M2).T, form(x_bits, 128, 1, F.E4M3).T, mask=mask, what="dW")
        dy = bf16_bits_to_f64(dy_bits)
        assert (np.abs(db[0].cpu().numpy() - dy.sum(0)) <= t * 2.0 ** -24 * np.abs(dy).sum(0)).all()
        after = W.cpu().numpy()
        assert not after[~mask].any() and (np.abs(after - before)[mask] > 0).mean() > 0.9
        assert np.array_equal(bits_of(Wb), bf16_bits(after)) and b.abs().sum() > 0
