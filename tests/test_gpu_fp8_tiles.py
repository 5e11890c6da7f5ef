"""8-bit products whose CTAs come round more than once, against float64 on the device: pairs of CTAs with several tiles of several blocks of
128 each, few tokens whose warps take several blocks.  Operands are codes and scales drawn directly (every finite code, scales
that differ from block to block); tolerance as derived in test_gpu_fp8.py."""
import pytest
import torch

import paper_2009_08065_b200 as bsp
from oracle import fp8_oracle as F
from gpu_util import DEV
from test_gpu_fp8 import up

pytestmark = pytest.mark.gpu
FINITE = {F.E4M3: 0x7E, F.E5M2: 0x7B}


def drawn(rows, cols, scale_shape, fmt, g):
    """Codes in a padded matrix whose padding is NaN, scale bytes, and the values in float64 (scales repeated by `wide`)."""
    whole = torch.full((rows, up(cols, 16) + 16), 0x7F, dtype=torch.uint8, device=DEV)
    q = whole[:, :cols]
    code = torch.randint(0, FINITE[fmt] + 1, (rows, cols), generator=g, device=DEV)
    q.copy_(code | (torch.randint(0, 2, (rows, cols), generator=g, device=DEV) << 7))
    top = 8 if fmt == F.E4M3 else 15
    s = torch.randint(127 - top - 4, 127 - top + 5, scale_shape, generator=g, device=DEV).to(torch.uint8)
    values = torch.from_numpy(F.code_values(fmt)).to(DEV)[q.long()]
    per = [1 if n == m else 128 for n, m in zip((rows, cols), scale_shape)]
    wide = torch.exp2(s.double() - 127).repeat_interleave(per[0], 0)[:rows].repeat_interleave(per[1], 1)[:, :cols]
    return q, s, values * wide


def check(Y, fill, a, b, bias=None, gelu=False, mask=None):
    cols = b.shape[0]
    assert bool((Y[:, cols:] == fill).all()), "columns behind the matrix were written"
    y = (Y[:, :cols].to(torch.int32) << 16).view(torch.float32).double()
    ref, mag, terms = a @ b.T, a.abs() @ b.abs().T, a.shape[1]
    if bias is not None:
        ref, mag, terms = ref + bias, mag + bias.abs(), terms + 1
    err = 1.01 * terms * 2.0 ** -23 * mag
    if gelu:
        err = 1.13 * err + 4e-6 * (1 + ref.abs())
        ref = ref * 0.5 * (1 + torch.erf(ref / 2.0 ** 0.5))
    if mask is not None:
        ref, err = ref * mask, err * mask
        assert not bool(Y[:, :cols][mask == 0].any())
    off = (y - ref).abs() - (2.0 ** -8 * ref.abs() + err + 1e-37)
    worst = int(off.argmax())
    assert bool(torch.isfinite(y).all()) and float(off.max()) <= 0, f"off by {float(off.max())} too much at {divmod(worst, cols)}"


def run(form, rows, cols, contraction, fmt, block=1):
    """out [rows, cols] summed over `contraction`, as one of the three products."""
    g = torch.Generator(device=DEV).manual_seed(rows + cols + contraction)
    blocks = lambda n: up(n, 128) // 128  # noqa: E731
    Y = torch.full((rows, up(cols, 8) + 8), 0x7FC0, dtype=torch.int16, device=DEV)
    out = Y[:, :cols]
    if form == "weight":                                            # rows of W x its columns, over the tokens
        yq, ys, y = drawn(contraction, rows, (blocks(contraction), rows), fmt, g)
        xq, xs, x = drawn(contraction, cols, (blocks(contraction), cols), F.E4M3, g)
        keep = (torch.rand(rows // block, cols, generator=g, device=DEV) < 0.4).to(torch.uint8)
        keep[0] = 0
        bsp.bsp_linear_fp8_backward_weight(yq, ys, fmt, xq, xs, F.E4M3, block, keep, out)
        bsp.bsp_linear_status()
        return check(Y, 0x7FC0, y.T, x.T, mask=keep.double().repeat_interleave(block, 0))
    aq, asc, a = drawn(rows, contraction, (rows, blocks(contraction)), fmt, g)
    if form == "input":
        wq, ws, w = drawn(contraction, cols, (blocks(contraction), blocks(cols)), F.E4M3, g)
        bsp.bsp_linear_fp8_backward_input(wq, ws, aq, asc, fmt, out)
        bsp.bsp_linear_status()
        return check(Y, 0x7FC0, a, w.T)
    wq, ws, w = drawn(cols, contraction, (blocks(cols), blocks(contraction)), F.E4M3, g)
    bias = torch.randn(cols, generator=g, device=DEV).to(torch.bfloat16)
    for act in (bsp.ACT_NONE, bsp.ACT_GELU):
        Y.fill_(0x7FC0)
        bsp.bsp_linear_fp8_quantized(wq, ws, aq, asc, fmt, bias, act, out)
        bsp.bsp_linear_status()
        check(Y, 0x7FC0, a, w, bias.double(), act == bsp.ACT_GELU)


# More than twice 74 tiles of 256 x 192 or one and a half times as many, ragged at both ends, blocks of the contraction 2, 3, 5, 6, 8, 9, 11, 13 and 33.
# (The rule of bsp_gemm_fp8.cu takes widths of 128 to 256 for them, 240 and 256 with a last piece that overlaps and with one accumulator among them.)
MANY = [(3500, 4600, 130), (2600, 2200, 260), (1800, 4096, 640), (2570, 4616, 650), (4000, 4090, 1000), (4000, 1900, 1100), (2500, 2050, 1290), (2600, 2200, 1664),
        (4096, 2304, 4100)]


@pytest.mark.parametrize("fmt", [F.E4M3, F.E5M2])
@pytest.mark.parametrize("form", ["linear", "input", "weight"])
@pytest.mark.parametrize("rows,cols,contraction", MANY)
def test_several_tiles_of_several_blocks(form, rows, cols, contraction, fmt):
    run(form, rows, cols, contraction, fmt, block=4 if rows % 4 == 0 else 2)


# 18 and 40 blocks for each CTA of a cluster of four (16 warps), 12 for each of two (12 warps), 20 for one (16)
@pytest.mark.parametrize("fmt", [F.E4M3, F.E5M2])
@pytest.mark.parametrize("t", [1, 5, 8, 13])
@pytest.mark.parametrize("n,k", [(64, 9000), (64, 20000), (50, 3001), (5000, 2560)])
def test_few_tokens_long_contractions(t, n, k, fmt):
    run("linear", t, n, k, fmt)


@pytest.mark.parametrize("t", [5, 8, 13, 24])
@pytest.mark.parametrize("n,k", [(64, 9000), (64, 20000), (5000, 2560)])
def test_few_tokens_long_contractions_from_bf16(t, n, k):
    """The same from bf16 activations: against float64."""
    g = torch.Generator(device=DEV).manual_seed(t + n + k)
    wq, ws, w = drawn(n, k, (up(n, 128) // 128, up(k, 128) // 128), F.E4M3, g)
    X = torch.randn(t, k, generator=g, device=DEV).to(torch.bfloat16)
    q, s = F.quantize(X.double().cpu().numpy(), 1, 128, F.E4M3)
    x = torch.from_numpy(F.dequantize(q, s, 1, 128, F.E4M3)).to(DEV)
    scratch = torch.empty(bsp.bsp_linear_fp8_ws_bytes(t, k), dtype=torch.uint8, device=DEV)
    Y = torch.full((t, n + 8), 0x7FC0, dtype=torch.int16, device=DEV)
    bsp.bsp_linear_fp8(wq, ws, X, None, bsp.ACT_NONE, Y[:, :n], scratch)
    bsp.bsp_linear_status()
    check(Y, 0x7FC0, x, w)
