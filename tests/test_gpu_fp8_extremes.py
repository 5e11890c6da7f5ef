"""The 8-bit linear layer with scales at the ends of their range: the same definition and tolerance as test_gpu_fp8.py (what float32 or
bf16 cannot hold at all, below 2^-126, is within its absolute term)."""
import numpy as np
import pytest
import torch

import paper_2009_08065_b200 as bsp
from oracle import fp8_oracle as F
from gpu_util import DEV, bf16_bits_to_f64, to_dev
from test_gpu_fp8 import Padded, bf16_bits, check, codes, up

pytestmark = pytest.mark.gpu


def matrices(t, n, k, fmt, exp_x, exp_w):
    """X and W in 8 bits; a third of W's rows and every other token are zeros beside blocks of these exponents."""
    rng = np.random.default_rng(t + n + k)
    w, x = rng.normal(size=(n, k)) * 2.0 ** exp_w, rng.normal(size=(t, k)) * 2.0 ** exp_x
    w[::3] = 0.0
    x[1::2] = 0.0
    x_bits = bf16_bits(x)
    wq, ws = F.quantize(bf16_bits_to_f64(bf16_bits(w)), 128, 128, F.E4M3)
    xq, xs = F.quantize(bf16_bits_to_f64(x_bits), 1, 128, fmt)
    return x_bits, codes(xq, xs, up(k, 16)), F.dequantize(xq, xs, 1, 128, fmt), codes(wq, ws, up(k, 16)), F.dequantize(wq, ws, 128, 128, F.E4M3)


def both_calls(t, n, k, fmt, x_bits, X8, W8):
    """The output by the call that quantises (e4m3) and by the one that takes 8-bit activations."""
    ws = torch.empty(bsp.bsp_linear_fp8_ws_bytes(t, k), dtype=torch.uint8, device=DEV)
    for quantised in (True, False):
        Y = Padded(t, n, up(n, 8), torch.int16, 0x7FC0)
        if quantised:
            bsp.bsp_linear_fp8_quantized(*W8, *X8, fmt, None, bsp.ACT_NONE, Y.t)
        elif fmt == F.E4M3:
            bsp.bsp_linear_fp8(*W8, to_dev(x_bits), None, bsp.ACT_NONE, Y.t, ws)
        else:
            continue
        bsp.bsp_linear_status()
        yield Y.host().view(np.uint16), f"quantised {quantised}"


@pytest.mark.parametrize("fmt", [F.E4M3, F.E5M2])
@pytest.mark.parametrize("t", [1, 3, 16, 24, 40, 300])
@pytest.mark.parametrize("exp_x,exp_w", [(100, -100), (-100, 100), (60, 60), (-60, -60), (90, -120), (-50, -60)])
def test_far_scales(t, exp_x, exp_w, fmt):
    n, k = 130, 520
    x_bits, X8, x, W8, w = matrices(t, n, k, fmt, exp_x, exp_w)
    for y, what in both_calls(t, n, k, fmt, x_bits, X8, W8):
        check(y, x, w, what=what)


@pytest.mark.parametrize("fmt", [F.E4M3, F.E5M2])
@pytest.mark.parametrize("t", [2, 16, 24, 40, 300])
def test_zeros_beside_values_that_overflow(t, fmt):
    """Scales whose product float32 does not hold: outputs that are sums of zeros are zero, and the others infinite or NaN."""
    n, k = 130, 520
    x_bits, X8, x, W8, w = matrices(t, n, k, fmt, 100, 100)
    for y, what in both_calls(t, n, k, fmt, x_bits, X8, W8):
        y = bf16_bits_to_f64(y)
        zero = (x @ w.T) == 0
        assert zero.any() and (y[zero] == 0).all() and not np.isfinite(y[~zero]).any(), what


def test_small_products_of_far_scales():
    """Both scales' product is 2^129 and more, what it multiplies 2^-18 and less: finite."""
    t, n, k = 4, 32, 256
    x = np.zeros((t, k))
    w = np.zeros((n, k))
    x[:, 0], w[:, 1] = 2.0 ** 73, 2.0 ** 73                         # the blocks' largest: scales of 2^65
    x[:, 2], w[:, 2] = 2.0 ** 56, 2.0 ** 57                         # 2^-9 and 2^-8 of them: 2^-17 2^130 = 2^113
    x_bits = bf16_bits(x)
    wq, wsc = F.quantize(w, 128, 128, F.E4M3)
    xq, xsc = F.quantize(x, 1, 128, F.E4M3)
    assert wsc[0, 0] == xsc[0, 0] == 127 + 65
    for y, what in both_calls(t, n, k, F.E4M3, x_bits, codes(xq, xsc, k), codes(wq, wsc, k)):
        assert (bf16_bits_to_f64(y) == 2.0 ** 113).all(), what
