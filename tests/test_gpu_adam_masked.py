"""The batched Adam step with 8-bit moments where gradients at pruned places are not finite: they are no part of the weights that are
kept, so nothing of them may reach the kept weights of the same block of 128, in this step or in later ones.  Where a moment there is not
finite, both begin again at zero; the rest is the oracle, bit for bit."""
import numpy as np
import pytest
import torch

import paper_2009_08065_b200 as bsp
from oracle import fp8_oracle as F
from gpu_util import DEV
from test_gpu_adam_batched import B1, B2, EPS, LR, Tensor

pytestmark = pytest.mark.gpu
ODD = [np.inf, -np.inf, np.nan, 3e38]                               # 3e38: v overflows, m does not


# without gaps (whole and ragged rows), with gaps, along rows, widths off 8
@pytest.mark.parametrize("rows,cols,orient,block,pad", [(32, 256, 0, 16, 0), (24, 200, 0, 4, 0), (32, 256, 0, 16, 8), (40, 200, 1, 5, 0), (13, 131, 0, 1, 0)])
@pytest.mark.parametrize("grad16", [False, True])
def test_pruned_places_keep_to_themselves(rows, cols, orient, block, pad, grad16):
    t = Tensor(rows, cols, 8, grad16, orient, block, pad)
    arr = bsp.make_adam_job_array([t.job])
    pruned = np.argwhere(~t.mask)
    rng = np.random.default_rng(rows)
    for step in (1, 2, 3):
        w0, m0, v0 = t.W.cpu().numpy(), *t.moments()
        assert np.isfinite(m0).all() and np.isfinite(v0).all()
        g = t.new_gradient()
        if step < 3:                                                # (the third: nothing is left behind)
            at = pruned[rng.choice(len(pruned), size=min(len(pruned), 60), replace=False)]
            for i, (r, c) in enumerate(at):
                t.G[int(r), int(c)] = (0x7F80, 0xFF80 - 65536, 0x7FC0, 0x7F61)[i % 4] if grad16 else float(ODD[i % 4])
                g[r, c] = np.float32(2.0 ** 127 * 1.7578125) if grad16 and i % 4 == 3 else np.float32(ODD[i % 4])
        bsp.bsp_masked_adam_step_batched(arr, B1, B2, EPS, step, 11)
        torch.cuda.synchronize()
        with np.errstate(all="ignore"):
            m, v = F.adam_moments(m0, v0, g, B1, B2)
        again = ~t.mask & ~(np.isfinite(m) & np.isfinite(v))
        m[again] = v[again] = 0.0
        qm, sm, qv, sv = F.store_moments(m, v, 11, step, 0)
        assert np.array_equal(t.MS.cpu().numpy(), sm) and np.array_equal(t.VS.cpu().numpy(), sv)
        assert np.array_equal(t.M.cpu().numpy(), qm) and np.array_equal(t.V.cpu().numpy(), qv)
        w = t.W.cpu().numpy()
        upd = m.astype(np.float64) / (1 - B1 ** step) / (np.sqrt(v.astype(np.float64) / (1 - B2 ** step)) + EPS)
        ref = (w0 - LR * (upd + float(np.float32(t.decay)) * w0)) * t.mask
        assert (np.abs(w - ref) <= 2e-7 * np.abs(ref) + 5e-6 * LR * np.maximum(1, np.abs(upd))).all()
        assert not w.view(np.uint32)[~t.mask].any()


def test_kept_places_still_mark_their_block():
    """An infinity at a kept place and one at a pruned place of the same block: the block is NaN throughout, as without the second."""
    t = Tensor(2, 256, 8, False, 0, 1)
    t.new_gradient()
    row = 1
    kept, pruned = np.flatnonzero(t.mask[row, :128]), np.flatnonzero(~t.mask[row, :128])
    t.G[row, int(kept[0])] = float("inf")
    t.G[row, int(pruned[0])] = float("nan")
    bsp.bsp_masked_adam_step_batched([t.job], B1, B2, EPS, 1, 0)
    m, v = t.moments()
    assert np.isnan(m[row, :128]).all() and np.isnan(v[row, :128]).all()
    assert np.isfinite(m[row, 128:]).all() and np.isfinite(m[0]).all()
    w = t.W.cpu().numpy()
    assert not np.isfinite(w[row, kept[0]]) and np.isfinite(np.delete(w[row], kept[0])).all()
