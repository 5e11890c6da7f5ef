"""Rows that are 2^32 elements and a row's length apart: their distance has to be refused, not cut to 32 bits (what is left would be a valid
distance, and other memory be read or written)."""
import pytest
import torch

import paper_2009_08065_b200 as bsp
from paper_2009_08065_b200 import binding
from gpu_util import DEV

FAR = 2 ** 32 + 64


@pytest.mark.parametrize("shape,strides", [((2, 64), (FAR, 1)), ((2, 64), (2 ** 31, 1)), ((2 ** 31, 64), (64, 1)), ((1, 2 ** 31), (2 ** 31, 1))])
def test_descriptors_refuse(shape, strides):
    t = torch.empty_strided(shape, strides, dtype=torch.float32, device="meta")
    with pytest.raises(ValueError, match="beyond"):
        binding._ld(t)


def test_largest_distance():
    assert binding._ld(torch.empty_strided((2, 64), (2 ** 31 - 1, 1), device="meta")) == 2 ** 31 - 1


@pytest.mark.gpu
def test_calls_refuse():
    z = lambda r, c, dtype: torch.zeros(r, c, dtype=dtype, device=DEV)  # noqa: E731
    far = torch.empty(FAR + 128, dtype=torch.uint8, device=DEV).as_strided((2, 64), (FAR, 1))
    W, WS, S, Y = z(32, 64, torch.uint8), z(1, 1, torch.uint8), z(2, 1, torch.uint8), z(2, 32, torch.bfloat16)
    bsp.bsp_linear_fp8_quantized(W, WS, z(2, 64, torch.uint8), S, 0, None, 0, Y)
    with pytest.raises(ValueError, match="beyond"):
        bsp.bsp_linear_fp8_quantized(W, WS, far, S, 0, None, 0, Y)
    with pytest.raises(ValueError, match="beyond"):
        bsp.bsp_fp8_quantize(z(2, 64, torch.bfloat16), 0, far, S)
    with pytest.raises(ValueError, match="beyond"):
        bsp.bsp_masked_adam_step_batched([bsp.AdamJob(W=z(2, 64, torch.float32), grad=z(2, 64, torch.float32), m=far, v=far, lr=0.1, m_scale=S, v_scale=S)],
                                         0.9, 0.999, 1e-8, 1)
    job = [bsp.AdamJob(W=z(2, 64, torch.float32), grad=z(2, 64, torch.float32), m=z(2, 64, torch.float32), v=z(2, 64, torch.float32), lr=0.1)]
    with pytest.raises(ValueError, match="beyond"):
        bsp.bsp_masked_adam_step_batched(job, 0.9, 0.999, 1e-8, 2 ** 32 + 1)
    torch.cuda.synchronize()
