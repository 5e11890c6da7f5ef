"""The batched Adam step with 8-bit moments and no gaps, with so many chunks that every CTA fills its stages again and again: against the
same tensors with a gap behind their rows, which the kernel for any tensor takes.  Bit for bit: moments, scales, weights and their copy."""
import pytest
import torch

import paper_2009_08065_b200 as bsp
from gpu_util import DEV

pytestmark = pytest.mark.gpu


def tensors(shapes, grad16, mixed):
    """Two sets of the same tensors: without gaps, and with rows 8 elements further apart."""
    g = torch.Generator(device=DEV).manual_seed(7)
    sets = ([], [])
    for i, (rows, cols, block) in enumerate(shapes):
        kb = (cols + 127) // 128
        half = grad16 != (mixed and i % 2 == 1)
        keep = None
        if block:
            keep = (torch.rand(rows // block, cols, generator=g, device=DEV) < 0.4).to(torch.uint8)
        W = 0.02 * torch.randn(rows, cols, generator=g, device=DEV)
        G = (1e-3 * torch.randn(rows, cols, generator=g, device=DEV)).to(torch.bfloat16 if half else torch.float32)
        M, V = (torch.randint(0, 0x78, (rows, cols), generator=g, device=DEV).to(torch.uint8) for _ in range(2))
        MS, VS = (torch.full((rows, kb), b, dtype=torch.uint8, device=DEV) for b in (107, 92))
        for gap, out in zip((0, 8), sets):
            def laid_out(t):
                whole = torch.zeros(rows, cols + gap, dtype=t.dtype, device=DEV)
                whole[:, :cols] = t
                return whole[:, :cols]
            out.append(bsp.AdamJob(W=laid_out(W), grad=laid_out(G), m=laid_out(M), v=laid_out(V), lr=1e-3 * (1 + i % 3), weight_decay=0.01 * (i % 2), m_scale=MS.clone(),
                                   v_scale=VS.clone(), keep=keep, block=max(1, block), W_bf16=laid_out(torch.zeros(rows, cols, dtype=torch.bfloat16, device=DEV))))
    return sets


# Chunks of 2048 weights; three CTAs of each of 148 SMs take one at a time: 4096 of the large tensor are nine turns.  Small and ragged
# tensors between large ones, so that a CTA goes from one tensor to another, and past several, between two of its chunks.
LARGE = [(2048, 4096, 16)]
MIXED = [(1024, 1024, 16), (1, 1024, 0), (3, 136, 3), (1, 8, 0), (1100, 920, 4), (1, 920, 0), (2048, 1024, 0), (1, 4096, 0), (5, 200, 1), (920, 3680, 8), (1, 3680, 0), (700, 1288, 1)]


@pytest.mark.parametrize("shapes,grad16,mixed", [(LARGE, True, False), (LARGE, False, False), (MIXED, True, False), (MIXED, False, True), (MIXED * 9, True, True)],
                         ids=["large bf16", "large float32", "small and large", "both gradients", "two launches"])
def test_many_chunks(shapes, grad16, mixed):
    dense, gaps = tensors(shapes, grad16, mixed)
    a, b = bsp.make_adam_job_array(dense), bsp.make_adam_job_array(gaps)
    scale = torch.full((1,), 0.5, dtype=torch.float32, device=DEV)
    for step in (1, 1000):
        bsp.bsp_masked_adam_step_batched(a, 0.9, 0.999, 1e-8, step, 3, scale)
        bsp.bsp_masked_adam_step_batched(b, 0.9, 0.999, 1e-8, step, 3, scale)
    bsp.bsp_linear_status()
    for i, (x, y) in enumerate(zip(dense, gaps)):
        for name in ("m", "v", "m_scale", "v_scale"):
            assert torch.equal(getattr(x, name), getattr(y, name)), (i, name)
        assert torch.equal(x.W.view(torch.int32), y.W.contiguous().view(torch.int32)), i
        assert torch.equal(x.W_bf16.view(torch.int16), y.W_bf16.contiguous().view(torch.int16)), i
        assert bool(torch.isfinite(x.W).all()) and float(x.W.abs().max()) > 0, i
