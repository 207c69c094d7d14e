"""AdamW with 8-bit states and scaled gradients: the product is formed in 64 bits like all that decides the states, which are equal to the
oracle's.  Tolerance of the parameters as in test_gpu_adamw.py."""
import numpy as np
import pytest

from oracle import attn_decoder_oracle as orc
from paper_1909_09577_amd import binding as nm
from test_gpu_adamw import HYPER, SIZES, U24, dev, draw8

pytestmark = pytest.mark.gpu


def step(host, scale):
    import torch
    t = [[dev(a) for a in h] for h in host]
    plan = nm.nm_adamw_plan([x[0] for x in t], [x[1] for x in t], [x[2] for x in t], [x[4] for x in t], m_scales=[x[3] for x in t],
                            v_scales=[x[5] for x in t], weight_decay=0.02)
    nm.nm_adamw_step(plan, step=3, seed=77, grad_scale=torch.tensor([scale], device="cuda"), **HYPER)
    torch.cuda.synchronize()
    return [[x.cpu().numpy() for x in d] for d in t]


@pytest.mark.parametrize("scale", [1 / 3, 0.0, 1e-6])
def test_states_are_those_of_the_scaled_gradients(scale):
    host = [draw8(n, n) for n in SIZES]
    scale, block = float(np.float32(scale)), 0
    for (p, g, mc, ms, rc, rs), got in zip(host, step(host, scale)):
        rp, rmc, rms, rrc, rrs = orc.adamw8(p, g, mc, ms, rc, rs, block, 77, 3, weight_decay=0.02, grad_scale=scale, **HYPER)
        block += len(ms)
        assert (got[3] == rms.astype(np.float32)).all() and (got[5] == rrs.astype(np.float32)).all()
        assert (got[2] & 127 == rmc & 127).all() and ((got[2] == rmc) | (rmc & 127 == 0)).all() and (got[4] == rrc).all()
        m, r = np.abs(orc.e4m3_values()[mc]) * np.repeat(ms, 256)[:len(p)].astype(np.float64), orc.e4m3_values()[rc] * np.repeat(rs, 256)[:len(p)].astype(np.float64)
        gs = g.astype(np.float64) * scale
        root = np.sqrt((0.98 * r * r + 0.02 * gs ** 2) / (1 - 0.98 ** 3))
        update = HYPER["lr"] / (1 - 0.9 ** 3) * (m + np.abs(gs)) / (root + 1e-8)
        assert (np.abs(got[0] - rp) <= 24 * U24 * (np.abs(p) + update) + 1e-44).all()


def test_a_product_beyond_float():
    """Gradients and a scale whose product no float holds are no infinities."""
    host = [draw8(600, 5)]
    host[0][1][:300] = 1e30
    got = step(host, 1e9)[0]
    assert np.isfinite(got[3]).all() and np.isfinite(got[5]).all()
    assert not (got[2] & 127 == 127).any() and not (got[4] == 127).any() and (got[4][:300] > 0).all()


def test_moments_that_no_scale_reaches():
    """They are stored as NaN, each by itself: the rest of their block keeps its values."""
    host = [draw8(600, 5)]
    p, g, mc, ms, rc, rs = (a.copy() for a in host[0])
    g *= 1e-20
    g[[7, 300]] = 1e30, -1e35
    scale = float(np.float32(1e20))
    got = step([(p, g, mc, ms, rc, rs)], scale)[0]
    assert np.flatnonzero(got[2] & 127 == 127).tolist() == [7, 300] == np.flatnonzero(got[4] == 127).tolist()
    rest = np.ones(600, bool)
    rest[[7, 300]] = False
    h = g.copy()
    h[~rest], mc[~rest], rc[~rest] = 0, 0, 0  # the oracle without them
    _, rmc, rms, rrc, rrs = orc.adamw8(p, h, mc, ms, rc, rs, 0, 77, 3, weight_decay=0.02, grad_scale=scale, **HYPER)
    assert (got[3] == rms.astype(np.float32)).all() and (got[5] == rrs.astype(np.float32)).all()
    assert (got[2] & 127 == rmc & 127)[rest].all() and (got[4] == rrc)[rest].all()
    assert np.isfinite(got[0][rest]).all()
