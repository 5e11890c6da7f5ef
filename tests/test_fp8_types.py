"""Element types: a floating-point type of the right size but the wrong format is refused, not read as the right one."""
import pytest
import torch

import paper_2009_08065_b200 as bsp
from gpu_util import DEV


def adam_job(device="cpu", **change):
    z = lambda dtype, c=16: torch.zeros(4, c, dtype=dtype, device=device)  # noqa: E731
    return bsp.AdamJob(**{**dict(W=z(torch.float32), grad=z(torch.float32), m=z(torch.uint8), v=z(torch.uint8), lr=0.1, m_scale=z(torch.uint8, 1), v_scale=z(torch.uint8, 1)),
                          **{k: z(v, 1 if k.endswith("scale") else 16) for k, v in change.items()}})


WRONG = [dict(grad=torch.float16), dict(grad=torch.int32), dict(W=torch.int32), dict(W_bf16=torch.float16), dict(m=torch.float8_e5m2), dict(v=torch.float8_e4m3fn), dict(m=torch.float32),
         dict(v=torch.float32), dict(m=torch.bool), dict(m=torch.int32, v=torch.int32), dict(m_scale=torch.float8_e4m3fn), dict(v_scale=torch.bool)]
RIGHT = [dict(), dict(grad=torch.bfloat16), dict(grad=torch.int16, W_bf16=torch.uint16), dict(W_bf16=torch.bfloat16), dict(m=torch.float8_e4m3fn, v=torch.float8_e5m2),
         dict(m=torch.float32, v=torch.float32), dict(m_scale=torch.float8_e8m0fnu)]


@pytest.mark.parametrize("change", WRONG, ids=str)
def test_adam_refuses_types(change):
    with pytest.raises(ValueError, match="unexpected element type"):
        bsp.make_adam_job_array([adam_job(**change)])


@pytest.mark.gpu
@pytest.mark.parametrize("change", RIGHT, ids=str)
def test_adam_takes_types(change):
    bsp.bsp_masked_adam_step_batched([adam_job(DEV, **change)], 0.9, 0.999, 1e-8, 1)
    torch.cuda.synchronize()


@pytest.mark.gpu
def test_adam_refuses_types_of_scalars():
    job = [adam_job(DEV)]
    for kw in (dict(grad_scale=torch.ones(1, dtype=torch.int32, device=DEV)), dict(step_dev=torch.ones(1, dtype=torch.float32, device=DEV))):
        with pytest.raises(ValueError, match="expected elements of type"):
            bsp.bsp_masked_adam_step_batched(job, 0.9, 0.999, 1e-8, 1, **kw)


T, N, K = 9, 32, 64
BF16, U8 = torch.bfloat16, torch.uint8
E4, E5 = torch.float8_e4m3fn, torch.float8_e5m2


def z(rows, cols, dtype):
    return torch.zeros(rows, cols, dtype=dtype, device=DEV)


def calls():
    """name -> (call, arguments, {argument: wrong types}, {argument: types that are taken})"""
    bits = {torch.float16, torch.float32}
    ws = torch.empty(4096, dtype=U8, device=DEV)
    return {
        "quantize": (bsp.bsp_fp8_quantize, dict(X=z(T, K, BF16), fmt=0, Q=z(T, K, U8), S=z(T, 1, U8), Qc=z(T, K, U8), Sc=z(1, K, U8), col_sums=z(1, K, torch.float32)[0], ws=ws),
                     dict(X=bits, Q={E5, torch.bool}, Qc={E5}, S={E4}, Sc={E5}, col_sums={torch.int32}), dict(X={torch.int16, torch.uint16}, Q={E4}, Qc={E4}, S={torch.float8_e8m0fnu})),
        "quantize e5m2": (bsp.bsp_fp8_quantize, dict(X=z(T, K, BF16), fmt=1, Q=z(T, K, U8), S=z(T, 1, U8)), dict(Q={E4}), dict(Q={E5})),
        "weight": (bsp.bsp_fp8_quantize_weight, dict(W=z(N, K, BF16), Q=z(N, K, U8), S=z(1, 1, U8)), dict(W=bits, Q={E5}, S={E4}), dict(Q={E4})),
        "linear": (bsp.bsp_linear_fp8, dict(Wq=z(N, K, U8), WS=z(1, 1, U8), X=z(T, K, BF16), bias=z(1, N, BF16)[0], act=0, Y=z(T, N, BF16), ws=ws),
                   dict(Wq={E5}, WS={E4}, X=bits, bias=bits, Y=bits), dict(Wq={E4}, Y={torch.int16})),
        "quantized": (bsp.bsp_linear_fp8_quantized, dict(Wq=z(N, K, U8), WS=z(1, 1, U8), Xq=z(T, K, U8), XS=z(T, 1, U8), fmt=1, bias=z(1, N, BF16)[0], act=0, Y=z(T, N, BF16)),
                      dict(Wq={E5}, Xq={E4}, XS={E5}, bias=bits, Y=bits), dict(Xq={E5})),
        "dX": (bsp.bsp_linear_fp8_backward_input, dict(Wq=z(N, K, U8), WS=z(1, 1, U8), dYq=z(T, N, U8), dYS=z(T, 1, U8), fmt=0, dX=z(T, K, BF16)),
               dict(Wq={E5}, dYq={E5}, dX=bits), dict(dYq={E4})),
        "dW": (bsp.bsp_linear_fp8_backward_weight, dict(dYq=z(T, N, U8), dYS=z(1, N, U8), fmt_dy=1, Xq=z(T, K, U8), XS=z(1, K, U8), fmt_x=0, block=1, keep=z(N, K, U8), dW=z(N, K, BF16)),
               dict(dYq={E4}, Xq={E5}, keep={E4}, dW=bits), dict(dYq={E5}, Xq={E4}, keep={torch.bool})),
    }


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["quantize", "quantize e5m2", "weight", "linear", "quantized", "dX", "dW"])
def test_types_of_the_linear_layer(name):
    call, args, wrong, right = calls()[name]
    call(**args)
    for table, refused in ((wrong, True), (right, False)):
        for arg, types in table.items():
            for dtype in types:
                changed = {**args, arg: torch.zeros(args[arg].shape, dtype=dtype, device=DEV)}
                if refused:
                    with pytest.raises(ValueError, match="expected elements of type"):
                        call(**changed)
                else:
                    call(**changed)
    torch.cuda.synchronize()


def test_descriptors_hold_their_tensors(monkeypatch):
    """An array that is used again must not name memory that has been given back: a gradient that was converted in place of the argument
    lives as long as the array."""
    import weakref

    from paper_2009_08065_b200 import binding
    monkeypatch.setattr(binding, "_ptr", lambda t: None if t is None else t.data_ptr())
    job = adam_job(W_bf16=torch.bfloat16)
    job.keep = torch.ones(4, 16, dtype=U8)
    job.grad = torch.ones(4, 16).to(torch.bfloat16)
    fields = ("W", "grad", "m", "v", "m_scale", "v_scale", "keep", "W_bf16")
    refs = [weakref.ref(getattr(job, f)) for f in fields]
    arr = bsp.make_adam_job_array([job])
    addresses = [getattr(job, f).data_ptr() for f in fields]
    del job
    assert all(r() is not None for r in refs)
    assert [getattr(arr[0], f) for f in fields] == addresses
    del arr
    assert all(r() is None for r in refs)


@pytest.mark.gpu
def test_learning_rate_between_calls():
    job = adam_job(DEV)
    job.W.fill_(1.0)
    job.grad.fill_(1.0)
    arr = bsp.make_adam_job_array([job])
    arr[0].lr = 0.25
    bsp.bsp_masked_adam_step_batched(arr, 0.9, 0.999, 1e-8, 1)
    assert (job.W.cpu() - 0.75).abs().max() < 1e-6                      # (a first step of a constant gradient is lr)
