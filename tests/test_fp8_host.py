"""The 8-bit calls on the host: the oracle's formats against torch's, refused arguments, size queries (no device needed)."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2009_08065_b200 as bsp
from paper_2009_08065_b200 import binding
from oracle import fp8_oracle as F

P = ctypes.c_void_p(0x1000)                                        # never touched: every call below is refused on the host
ARG, SHAPE, WS, UNSUPPORTED = -1, -2, -3, -6


@pytest.mark.parametrize("fmt,dtype", [(F.E4M3, torch.float8_e4m3fn), (F.E5M2, torch.float8_e5m2)])
def test_oracle_formats_are_torchs(fmt, dtype):
    codes = torch.arange(256, dtype=torch.uint8)
    assert np.array_equal(F.code_values(fmt), codes.view(dtype).to(torch.float64).numpy(), equal_nan=True)
    x = np.concatenate([np.random.default_rng(1).normal(size=20000) * 2.0 ** np.random.default_rng(2).integers(-20, 7, 20000),
                        np.arange(-448, 449) / 16.0, (F.code_values(fmt)[:120] + F.code_values(fmt)[1:121]) / 2])
    x = x[np.abs(x) <= F.LARGEST[fmt]].astype(np.float32)
    assert np.array_equal(F.encode_nearest(x, fmt), torch.from_numpy(x).to(dtype).view(torch.uint8).numpy())


def test_oracle_scales_and_blocks():
    assert F.scale_byte(np.array([448.0, 448.1, 0.0, 1.75, 1.76, 2.0 ** -130]), F.E4M3).tolist() == [127, 128, 0, 119, 120, 0]
    assert F.scale_byte(np.array([57344.0, 57345.0]), F.E5M2).tolist() == [127, 128]
    x = np.ones((3, 130))
    x[1, 129] = np.inf
    q, s = F.quantize(x, 1, 128, F.E4M3)
    assert s.shape == (3, 2) and s[1, 1] == 127 and (q[1, 128:] == 0x7f).all() and (F.dequantize(q, s, 1, 128, F.E4M3)[0] == 1.0).all()


@pytest.mark.parametrize("fmt", [F.E4M3, F.E5M2])
def test_random_rounding_is_right_on_average(fmt):
    """20000 draws of each value: the mean is off by at most five standard deviations of a mean of as many draws of a step."""
    rng = np.random.default_rng(3)
    ym = rng.uniform(0.0, 1.0, 64).astype(np.float32) * np.float32(2.0) ** rng.integers(-12, 8, 64).astype(np.float32)
    r = np.stack([F.random_bits(5, step, 0, 1, 64)[0 if fmt == F.E4M3 else 1][0] for step in range(1, 20001)])
    v = F.code_values(fmt)
    got = v[F.encode_randomly(np.broadcast_to(ym, r.shape), r, fmt)].mean(0)
    lo = np.searchsorted(v[:120], ym, side="right") - 1
    step = v[lo + 1] - v[lo]
    assert (np.abs(got - ym) <= 5 * step / np.sqrt(20000) + step * 2.0 ** -16).all()


def test_size_query():
    assert bsp.bsp_linear_fp8_ws_bytes(1, 128) == 256 and bsp.bsp_linear_fp8_ws_bytes(3, 1000) >= 3 * (1008 + 8)
    for bad in ((0, 128), (1, 0), (-1, 5)):
        with pytest.raises(bsp.BspError) as e:
            bsp.bsp_linear_fp8_ws_bytes(*bad)
        assert e.value.status == ARG


def quantize(X=P, rows=4, cols=256, ldx=256, fmt=0, Q=P, ldq=256, S=P, lds=2, Qc=None, ldqc=0, Sc=None, ldsc=0, sums=None, ws=None, ws_bytes=0):
    return bsp.lib.bsp_fp8_quantize(X, rows, cols, ldx, fmt, Q, ldq, S, lds, Qc, ldqc, Sc, ldsc, sums, ws, ws_bytes, None)


@pytest.mark.parametrize("change,status", [
    (dict(X=None), ARG), (dict(rows=0), ARG), (dict(cols=-1), ARG), (dict(fmt=2), ARG), (dict(Q=None), ARG), (dict(S=None), ARG), (dict(Qc=P), ARG),
    (dict(Q=None, S=None), ARG), (dict(X=ctypes.c_void_p(0x1001)), ARG), (dict(ldx=255), SHAPE), (dict(ldq=255), SHAPE), (dict(lds=1), SHAPE),
    (dict(Qc=P, Sc=P, ldqc=256, ldsc=255), SHAPE), (dict(sums=P), ARG), (dict(sums=P, ws=P, ws_bytes=1023), WS), (dict(rows=65535 * 128 + 1), UNSUPPORTED)])
def test_quantize_refuses(change, status):
    assert quantize(**change) == status


MOST = 0x7FFFFE00                                                  # largest size


def test_sizes_beyond_the_kernels_counting():
    big = MOST + 1
    assert quantize(cols=big, ldx=big, ldq=big, lds=1 << 26) == UNSUPPORTED
    assert bsp.lib.bsp_fp8_quantize_weight(P, 1, big, big, P, big, P, 1 << 26, None) == UNSUPPORTED
    n = ctypes.c_size_t()
    assert bsp.lib.bsp_linear_fp8_ws_bytes(1, big, ctypes.byref(n)) == UNSUPPORTED and bsp.lib.bsp_linear_fp8_ws_bytes(big, 1, ctypes.byref(n)) == UNSUPPORTED
    f = bsp.lib.bsp_linear_fp8_quantized
    for n_out, k, t in ((big, 16, 1), (16, big, 1), (16, 16, big)):
        assert f(P, k, P, 1 << 26, n_out, k, P, k, P, 1 << 26, 0, t, None, 0, P, n_out, None) == UNSUPPORTED
        assert bsp.lib.bsp_linear_fp8_backward_input(P, k, P, 1 << 26, n_out, k, P, n_out, P, 1 << 26, 0, t, P, k, None) == UNSUPPORTED
        assert bsp.lib.bsp_linear_fp8_backward_weight(P, n_out, P, n_out, 0, P, k, P, k, 0, t, n_out, k, 1, None, P, k, None) == UNSUPPORTED
    assert adam(adam_job(rows=1, cols=big, ldw=big, ldg=big, ldm=big)) == UNSUPPORTED


def test_binding_refuses_what_is_not_on_a_device():
    x = torch.zeros(4, 16, dtype=torch.bfloat16)
    q, s = torch.zeros(4, 16, dtype=torch.uint8), torch.zeros(4, 1, dtype=torch.uint8)
    with pytest.raises((ValueError, RuntimeError)):
        bsp.bsp_fp8_quantize(x, bsp.FP8_E4M3, q, s)
    with pytest.raises(ValueError):
        bsp.make_adam_job_array([bsp.AdamJob(W=x.float(), grad=x, m=x.float(), v=x.float(), lr=1.0)])


def test_quantize_weight_refuses():
    f = bsp.lib.bsp_fp8_quantize_weight
    assert f(None, 128, 128, 128, P, 128, P, 1, None) == ARG and f(P, 128, 128, 128, P, 128, None, 1, None) == ARG
    assert f(P, 0, 128, 128, P, 128, P, 1, None) == ARG
    assert f(P, 128, 256, 255, P, 256, P, 2, None) == SHAPE and f(P, 128, 256, 256, P, 255, P, 2, None) == SHAPE
    assert f(P, 128, 256, 256, P, 256, P, 1, None) == SHAPE


def test_linear_refuses():
    f = bsp.lib.bsp_linear_fp8
    ok = dict(Wq=P, ldw=256, WS=P, ldws=2, n=64, k=256, X=P, t=4, ldx=256, bias=None, act=0, Y=P, ldy=64, ws=P, wsb=1 << 20)
    call = lambda **c: f(*{**ok, **c}.values(), None)  # noqa: E731
    for c in (dict(Wq=None), dict(WS=None), dict(n=0), dict(k=0), dict(X=None), dict(Y=None), dict(ws=None), dict(t=0), dict(act=2),
              dict(bias=ctypes.c_void_p(0x1001)), dict(ws=ctypes.c_void_p(0x1008))):
        assert call(**c) == ARG, c
    for c in (dict(ldw=255), dict(ldws=1), dict(ldx=255), dict(ldy=63)):
        assert call(**c) == SHAPE, c
    assert call(wsb=1000) == WS
    g = bsp.lib.bsp_linear_fp8_quantized
    ok = dict(Wq=P, ldw=256, WS=P, ldws=2, n=64, k=256, Xq=P, ldx=256, XS=P, ldxs=2, fmt=0, t=4, bias=None, act=0, Y=P, ldy=64)
    call = lambda **c: g(*{**ok, **c}.values(), None)  # noqa: E731
    for c in (dict(Xq=None), dict(XS=None), dict(fmt=2), dict(act=-1), dict(t=-3)):
        assert call(**c) == ARG, c
    for c in (dict(ldx=255), dict(ldxs=1), dict(ldy=63)):
        assert call(**c) == SHAPE, c


def test_backward_refuses():
    f = bsp.lib.bsp_linear_fp8_backward_input
    ok = dict(Wq=P, ldw=256, WS=P, ldws=2, n=300, k=256, dY=P, ldy=300, dYS=P, ldys=3, fmt=1, t=4, dX=P, ldx=256)
    call = lambda **c: f(*{**ok, **c}.values(), None)  # noqa: E731
    for c in (dict(Wq=None), dict(dY=None), dict(dYS=None), dict(fmt=-1), dict(t=0), dict(dX=None)):
        assert call(**c) == ARG, c
    for c in (dict(ldw=255), dict(ldws=1), dict(ldy=299), dict(ldys=2), dict(ldx=255)):
        assert call(**c) == SHAPE, c
    f = bsp.lib.bsp_linear_fp8_backward_weight
    ok = dict(dY=P, ldy=300, dYS=P, ldys=300, fy=1, X=P, ldx=256, XS=P, ldxs=256, fx=0, t=4, n=300, k=256, block=3, keep=None, dW=P, lddw=256)
    call = lambda **c: f(*{**ok, **c}.values(), None)  # noqa: E731
    for c in (dict(dY=None), dict(dYS=None), dict(X=None), dict(XS=None), dict(dW=None), dict(fy=2), dict(fx=2), dict(t=0), dict(block=0)):
        assert call(**c) == ARG, c
    for c in (dict(block=7), dict(ldy=299), dict(ldys=299), dict(ldx=255), dict(ldxs=255), dict(lddw=255)):
        assert call(**c) == SHAPE, c


def adam_job(**change):
    j = binding._AdamJob()
    for k, v in {**dict(W=0x1000, rows=4, cols=256, ldw=256, grad=0x1000, ldg=256, grad_type=0, m=0x1000, v=0x1000, ldm=256, state_bits=8, m_scale=0x1000,
                        v_scale=0x1000, keep=None, block=1, orient=0, lr=1e-3, weight_decay=0.0, W_bf16=None, ldb=0), **change}.items():
        setattr(j, k, v)
    return j


def adam(*jobs, n=None, beta1=0.9, beta2=0.999, eps=1e-8, step=1, scale=None, step_dev=None):
    arr = (binding._AdamJob * max(1, len(jobs)))(*jobs)
    return bsp.lib.bsp_masked_adam_step_batched(arr, len(jobs) if n is None else n, beta1, beta2, eps, step, 0, scale, step_dev, None)


@pytest.mark.parametrize("change,status", [
    (dict(W=None), ARG), (dict(grad=None), ARG), (dict(m=None), ARG), (dict(v=None), ARG), (dict(rows=0), ARG), (dict(state_bits=16), ARG),
    (dict(grad_type=2), ARG), (dict(m_scale=None), ARG), (dict(v_scale=None), ARG), (dict(lr=float("nan")), ARG), (dict(W=0x1002), ARG), (dict(grad=0x1002), ARG),
    (dict(state_bits=32, m=0x1002), ARG), (dict(W_bf16=0x1001, ldb=256), ARG), (dict(ldw=255), SHAPE), (dict(ldg=255), SHAPE), (dict(ldm=255), SHAPE),
    (dict(W_bf16=0x1000, ldb=255), SHAPE), (dict(keep=0x1000, block=3), SHAPE), (dict(keep=0x1000, block=0), ARG), (dict(keep=0x1000, orient=2), ARG),
    (dict(rows=2 ** 31 - 1, cols=2 ** 31 - 1, ldw=2 ** 31 - 1, ldg=2 ** 31 - 1, ldm=2 ** 31 - 1), UNSUPPORTED)])
def test_adam_refuses_a_job(change, status):
    assert adam(adam_job(**change)) == status
    assert adam(adam_job(state_bits=7), adam_job()) == ARG
    assert adam(adam_job(), adam_job(**change)) == status            # the last of several: nothing has been launched before it is looked at


def test_adam_refuses_a_call():
    assert adam(n=0) == ARG and bsp.lib.bsp_masked_adam_step_batched(None, 1, 0.9, 0.999, 1e-8, 1, 0, None, None, None) == ARG
    for c in (dict(beta1=1.0), dict(beta2=-0.1), dict(beta1=float("nan")), dict(eps=-1.0), dict(step=0), dict(scale=ctypes.c_void_p(0x1002)),
              dict(step_dev=ctypes.c_void_p(0x1002))):
        assert adam(adam_job(), **c) == ARG, c


def test_descriptors_of_another_kind_are_refused():
    with pytest.raises(ctypes.ArgumentError):
        bsp.bsp_masked_adam_step_batched((binding._LayerJob * 1)(), 0.9, 0.999, 1e-8, 1, stream=0)


@pytest.mark.parametrize("keep", [torch.ones(2, 16, dtype=torch.uint8), torch.ones(4, 15, dtype=torch.uint8), torch.ones(4, 32, dtype=torch.uint8)[:, ::2],
                                  torch.ones(4, 16, dtype=torch.int16)])
def test_flags_of_another_size_are_refused(keep):
    w = torch.zeros(8, 16)
    with pytest.raises(ValueError, match="keep is"):
        bsp.make_adam_job_array([bsp.AdamJob(W=w, grad=w, m=w, v=w, lr=1.0, keep=keep, block=2)])
