"""GPU parity of bsp_masked_adam_step_batched.

32-bit moments: bit for bit what bsp_masked_adam_step gives where that call takes the shape.  8-bit moments: the codes and scale bytes of the
oracle's float64 emulation of the float32 moments, bit for bit.  Weights: as derived in test_gpu_retrain.py, |W' - W'_ref| <= 2e-7 |W'_ref| + 5e-6 lr
for updates of order one.
"""
import numpy as np
import pytest
import torch

import paper_2009_08065_b200 as bsp
from oracle import bsp_oracle as O
from oracle import fp8_oracle as F
from gpu_util import DEV, bits_of

pytestmark = pytest.mark.gpu
LR, B1, B2, EPS = (float(np.float32(h)) for h in (3e-4, 0.9, 0.999, 1e-8))


def f32_to_bf16_rne(a):
    u = np.ascontiguousarray(a, dtype=np.float32).view(np.uint32).astype(np.uint64)
    return ((u + 0x7FFF + ((u >> 16) & 1)) >> 16).astype(np.uint16)


def padded(a, ld, fill=0):
    whole = torch.full((a.shape[0], ld), fill, dtype=torch.from_numpy(a[:0]).dtype, device=DEV)
    whole[:, :a.shape[1]] = torch.from_numpy(a).to(DEV)
    return whole[:, :a.shape[1]]


class Tensor:
    """One job with its state on the host."""

    def __init__(self, rows, cols, bits, grad16, orient=0, block=0, pad=0, seed=0, decay=0.0):
        rng = np.random.default_rng(seed + 31 * rows + cols)
        self.rows, self.cols, self.bits, self.grad16, self.decay, self.pad = rows, cols, bits, grad16, decay, pad
        self.rng = rng
        self.keep, self.mask = None, None
        if block:
            shape = (rows // block, cols) if orient == 0 else (rows, cols // block)
            self.keep = (rng.random(shape) < 0.5).astype(np.uint8)
            self.keep[0] = 0
            self.mask = np.repeat(self.keep, block, orient).astype(bool)
        w = (0.02 * rng.normal(size=(rows, cols))).astype(np.float32)
        self.W = padded(w if self.mask is None else (w * self.mask).astype(np.float32), cols + pad)
        self.Wb = padded(np.full((rows, cols), 0x7FC0, dtype=np.int16), cols + 2 * pad)
        self.keep_d = None if self.keep is None else torch.from_numpy(self.keep).to(DEV)
        self.G = padded(np.zeros((rows, cols), dtype=np.int16 if grad16 else np.float32), cols + pad)
        kb = (cols + 127) // 128
        if bits == 8:
            self.M, self.V = (padded(np.zeros((rows, cols), dtype=np.uint8), cols + pad) for _ in range(2))
            self.MS, self.VS = (torch.zeros((rows, kb), dtype=torch.uint8, device=DEV) for _ in range(2))
        else:
            self.M, self.V = (padded(np.zeros((rows, cols), dtype=np.float32), cols + pad) for _ in range(2))
            self.MS = self.VS = None
        self.job = bsp.AdamJob(W=self.W, grad=self.G, m=self.M, v=self.V, lr=LR, weight_decay=decay, m_scale=self.MS, v_scale=self.VS, keep=self.keep_d,
                               block=max(block, 1), orient=orient, W_bf16=self.Wb)

    def new_gradient(self, size=1e-2):
        g = (self.rng.normal(size=(self.rows, self.cols)) * size * np.exp(2 * self.rng.normal(size=(self.rows, 1)))).astype(np.float32)
        g[self.rng.random(g.shape) < 0.05] = 0.0
        if self.grad16:
            bits = f32_to_bf16_rne(g)
            self.G.copy_(torch.from_numpy(bits.view(np.int16)))
            return (bits.astype(np.uint32) << 16).view(np.float32)
        self.G.copy_(torch.from_numpy(g))
        return g

    def moments(self):
        if self.bits == 32:
            return self.M.cpu().numpy(), self.V.cpu().numpy()
        m = F.dequantize(self.M.cpu().numpy(), self.MS.cpu().numpy(), 1, 128, F.E4M3)
        v = F.dequantize(self.V.cpu().numpy(), self.VS.cpu().numpy(), 1, 128, F.E5M2)
        return m.astype(np.float32), v.astype(np.float32)

    def check(self, before, g, step, seed, job):
        w0, m0, v0 = before
        m, v = F.adam_moments(m0, v0, g, B1, B2)
        mh = m.astype(np.float64) / (1 - B1 ** step)
        vh = v.astype(np.float64) / (1 - B2 ** step)
        upd = mh / (np.sqrt(vh) + EPS)
        ref = w0.astype(np.float64) - LR * (upd + float(np.float32(self.decay)) * w0)
        if self.mask is not None:
            ref = ref * self.mask
        w = self.W.cpu().numpy()
        assert (np.abs(w - ref) <= 2e-7 * np.abs(ref) + 5e-6 * LR * np.maximum(1, np.abs(upd))).all()
        if self.mask is not None:
            assert not w.view(np.uint32)[~self.mask].any()
        assert np.array_equal(bits_of(self.Wb), f32_to_bf16_rne(w))
        if self.bits == 32:
            assert np.array_equal(self.M.cpu().numpy(), m) and np.array_equal(self.V.cpu().numpy(), v)
            return
        qm, sm, qv, sv = F.store_moments(m, v, seed, step, job)
        assert np.array_equal(self.MS.cpu().numpy(), sm) and np.array_equal(self.VS.cpu().numpy(), sv)
        assert np.array_equal(self.M.cpu().numpy(), qm) and np.array_equal(self.V.cpu().numpy(), qv)


SHAPES = [(1, 1, 0, 0, 0), (1, 768, 0, 0, 0), (3, 130, 0, 0, 1), (64, 128, 0, 16, 0), (96, 264, 0, 12, 8), (40, 200, 1, 5, 0), (33, 1000, 1, 8, 3), (130, 257, 0, 1, 0),
          (2, 4096, 0, 2, 16)]


def make(bits, grad16, shapes=SHAPES):
    return [Tensor(r, c, bits, grad16, orient, block, pad, seed=i, decay=0.01 if r > 1 else 0.0) for i, (r, c, orient, block, pad) in enumerate(shapes)]


def run(tensors, steps, seed, clip=None, **kw):
    arr = bsp.make_adam_job_array([t.job for t in tensors])
    scale = None if clip is None else torch.full((1,), clip, dtype=torch.float32, device=DEV)
    for step in steps:
        before = [(t.W.cpu().numpy(), *t.moments()) for t in tensors]
        grads = [t.new_gradient() for t in tensors]
        bsp.bsp_masked_adam_step_batched(arr, B1, B2, EPS, step, seed, scale, **kw)
        torch.cuda.synchronize()
        for i, (t, b, g) in enumerate(zip(tensors, before, grads)):
            t.check(b, g if clip is None else (g * np.float32(clip)).astype(np.float32), step, seed, i)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("grad16", [False, True])
def test_three_steps(bits, grad16):
    run(make(bits, grad16), (1, 2, 3), 12345)


# tensors without gaps: a part of a chunk, several rows in one, rows that end inside a block of 128, more chunks than run at once
STREAM = [(1, 8, 0, 0, 0), (3, 128, 0, 1, 0), (100, 8, 0, 4, 0), (16, 200, 0, 2, 0), (48, 920, 0, 12, 0), (7, 4096, 0, 0, 0), (1536, 1024, 0, 16, 0), (5, 136, 0, 5, 0)]


@pytest.mark.parametrize("grad16", [False, True])
def test_three_steps_without_gaps(grad16):
    run(make(8, grad16, STREAM), (1, 2, 3), 99, clip=0.5)


def test_views_that_begin_inside_an_arena():
    """8-bit moments that begin at multiples of 8 but not of 16 bytes, tensors right behind one another."""
    tensors = make(8, True, [(1, 8, 0, 0, 0), (3, 136, 0, 3, 0), (1, 24, 0, 0, 0), (40, 200, 0, 4, 0), (1, 920, 0, 0, 0)])
    total = sum(t.rows * t.cols for t in tensors)
    at = 0
    for name in ("W", "M", "V", "Wb", "G"):
        arena = torch.zeros(total, dtype=getattr(tensors[0], name).dtype, device=DEV)
        at = 0
        for t in tensors:
            view = arena[at:at + t.rows * t.cols].view(t.rows, t.cols)
            view.copy_(getattr(t, name))
            setattr(t, name, view)
            at += t.rows * t.cols
    for t in tensors:
        t.job.W, t.job.m, t.job.v, t.job.W_bf16, t.job.grad = t.W, t.M, t.V, t.Wb, t.G
    run(tensors, (1, 2), 4)


def test_clipped_and_late():
    run(make(8, True), (1, 1000, 2 ** 31 - 1), 2 ** 32 - 1, clip=0.37)


def test_mixed_jobs_in_one_call():
    tensors = make(8, True, SHAPES[:4]) + make(32, False, SHAPES[3:6]) + make(8, False, SHAPES[5:]) + make(32, True, SHAPES[:3])
    run(tensors, (1, 2), 7)


def test_more_tensors_than_one_launch_takes():
    run([Tensor(2 + i % 3, 100 + i, 8, i % 2 == 0, seed=i) for i in range(200)], (1, 2), 3)


@pytest.mark.parametrize("orient,block,shape", [(0, 16, (768, 768)), (0, 12, (96, 80)), (1, 5, (96, 80)), (0, 1, (7, 1028))])
def test_32_bits_are_the_single_call(orient, block, shape):
    t = Tensor(*shape, 32, False, orient, block, decay=0.01)
    W, M, V, Wb = (x.clone() for x in (t.W, t.M, t.V, t.Wb))
    for step in (1, 2, 3):
        t.new_gradient()
        bsp.bsp_masked_adam_step(W, t.G, M, V, t.keep_d, block, orient, LR, B1, B2, EPS, 0.01, step, Wb)
        bsp.bsp_masked_adam_step_batched([t.job], B1, B2, EPS, step)
    torch.cuda.synchronize()
    for a, b in ((W, t.W), (M, t.M), (V, t.V)):
        assert torch.equal(a.view(torch.int32), b.contiguous().view(torch.int32))
    assert torch.equal(Wb, t.Wb)


def test_step_on_the_device_and_replay():
    """A captured step whose number and gradient scale live on the device: each replay is the next step."""
    a, b = make(8, True), make(8, True)
    dev_step = torch.ones(1, dtype=torch.int32, device=DEV)
    scale = torch.full((1,), 0.5, dtype=torch.float32, device=DEV)
    grads = [[t.new_gradient() for t in a] for _ in range(3)]
    arr_a, arr_b = bsp.make_adam_job_array([t.job for t in a]), bsp.make_adam_job_array([t.job for t in b])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        bsp.bsp_masked_adam_step_batched(arr_a, B1, B2, EPS, 0, 9, scale, dev_step)
    for step in (1, 2, 3):
        for ta, tb, g in zip(a, b, grads[step - 1]):
            ta.G.copy_(torch.from_numpy(f32_to_bf16_rne(g).view(np.int16)))
            tb.G.copy_(ta.G)
        graph.replay()
        dev_step += 1
        bsp.bsp_masked_adam_step_batched(arr_b, B1, B2, EPS, step, 9, scale)
        torch.cuda.synchronize()
        for ta, tb in zip(a, b):
            assert torch.equal(ta.M, tb.M) and torch.equal(ta.V, tb.V) and torch.equal(ta.MS, tb.MS) and torch.equal(ta.VS, tb.VS)
            # (the device's bias corrections are float32: two roundings of about 1e-7 each on an update of order one or below)
            assert bool(((ta.W - tb.W).abs() <= 2e-7 * tb.W.abs() + 5e-6 * LR * 30).all())
    graph.reset()


def test_repeatable_and_seeded():
    def once(seed):
        ts = make(8, True)
        for t in ts:
            t.new_gradient()
        bsp.bsp_masked_adam_step_batched([t.job for t in ts], B1, B2, EPS, 1, seed)
        torch.cuda.synchronize()
        return [t.M.cpu().numpy() for t in ts]
    a, b, c = once(1), once(1), once(2)
    assert all(np.array_equal(x, y) for x, y in zip(a, b)) and any(not np.array_equal(x, y) for x, y in zip(a, c))


def test_a_constant_gradient_is_learned():
    """v decays and grows by a thousandth a step: rounded to nearest it would stay where it is.  With gradients of 1 for 3000 steps and
    then of 0.25, v has to end near 1/16: 512 weights of one block's size, mean within a tenth (3000 steps leave exp(-3) of the difference
    of 0.94, 0.047, and the mean of 512 values with a spread below one half of themselves is off by 0.03 of them)."""
    t = Tensor(4, 128, 8, False)
    arr = bsp.make_adam_job_array([t.job])
    for phase, g in enumerate((1.0, 0.25)):
        t.G.fill_(g)
        for step in range(1, 3001):
            bsp.bsp_masked_adam_step_batched(arr, B1, B2, EPS, phase * 3000 + step, 5)
    v = t.moments()[1]
    want = 0.0625 + (1 - np.exp(-3)) * np.exp(-3) - 0.0625 * np.exp(-3)
    assert abs(v.mean() / want - 1) < 0.1 and np.isfinite(t.W.cpu().numpy()).all()


def test_zero_and_tiny_moments():
    """All-zero gradients leave zero moments and the weights; a positive v never becomes zero beside a large one."""
    t = Tensor(2, 256, 8, False)
    w = t.W.clone()
    bsp.bsp_masked_adam_step_batched([t.job], B1, B2, EPS, 1, 0)
    assert torch.equal(t.W, w) and not t.M.any() and not t.V.any() and not t.MS.any()
    g = np.zeros((2, 256), dtype=np.float32)
    g[:, ::2] = 1e-12
    g[0, 5] = 1e3
    t.G.copy_(torch.from_numpy(g))
    bsp.bsp_masked_adam_step_batched([t.job], B1, B2, EPS, 2, 0)
    v = t.moments()[1]
    assert (v[:, ::2][v[:, ::2] > 0].size == 2 * 128) and v[0, 1] == 0 and np.isfinite(t.W.cpu().numpy()).all()


def test_gradients_that_are_not_finite():
    """An infinity reaches its weight and its block's moments, nothing else."""
    t, u = Tensor(3, 300, 8, False), Tensor(3, 300, 8, False)
    g = t.new_gradient()
    u.G.copy_(t.G)
    t.G[1, 140] = float("inf")
    bsp.bsp_masked_adam_step_batched([t.job], B1, B2, EPS, 1, 0)
    bsp.bsp_masked_adam_step_batched([u.job], B1, B2, EPS, 1, 0)
    m, v = t.moments()
    mu, vu = u.moments()
    assert np.isnan(m[1, 128:256]).all() and np.isnan(v[1, 128:256]).all()
    for a, b in ((m, mu), (v, vu)):
        a[1, 128:256] = b[1, 128:256] = 0
        assert np.array_equal(a, b)
    w, wu = t.W.cpu().numpy(), u.W.cpu().numpy()
    assert not np.isfinite(w[1, 140])
    w[1, 140] = wu[1, 140]
    assert np.array_equal(w, wu)
