"""The AdamW step on the GPU against the float64 oracle: many tensors of any size and alignment, states in 32 and in 8 bits.

Tolerances (derived): a float state is two products and a sum (3 * 2^-24 of its terms), the update a quotient of some ten
operations (16 * 2^-24 of it, and that much of the parameter); 8-bit codes and scales are decided in 64 bits on both sides and are
equal; the bfloat16 copy is the parameter rounded once."""
import numpy as np
import pytest

from oracle import attn_decoder_oracle as orc
from paper_1909_09577_amd import binding as nm

pytestmark = pytest.mark.gpu
U24 = 2.0 ** -24
HYPER = dict(lr=2e-3, beta1=0.9, beta2=0.98, eps=1e-8)
SIZES = [1, 3, 255, 256, 257, 1000, 4096, 4097, 9000]


def dev(a, offset=0):
    """Device copy that begins `offset` elements behind an aligned address."""
    import torch
    t = torch.empty(len(a) + offset, dtype={np.dtype("float32"): torch.float32, np.dtype("uint8"): torch.uint8}[a.dtype], device="cuda")
    t[offset:].copy_(torch.from_numpy(a))
    return t[offset:]


def draw(n, seed):
    r = np.random.default_rng(seed)
    f = lambda s: (s * r.standard_normal(n)).astype(np.float32)  # noqa: E731
    return f(0.05), f(1e-3), f(1e-3), (f(1e-3) ** 2).astype(np.float32)


@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("step", [1, 1000])
def test_float_states(offset, step):
    import torch
    host = [draw(n, n) for n in SIZES]
    t = [[dev(a, offset) for a in h] for h in host]
    copies = [torch.zeros(n + offset, dtype=torch.bfloat16, device="cuda")[offset:] if i % 3 else None for i, n in enumerate(SIZES)]
    decay = [0.1 * (i % 2) for i in range(len(SIZES))]
    scale = torch.tensor([0.25], device="cuda")
    plan = nm.nm_adamw_plan([x[0] for x in t], [x[1] for x in t], [x[2] for x in t], [x[3] for x in t], copies=copies, weight_decay=decay)
    nm.nm_adamw_step(plan, step=step, grad_scale=scale, **HYPER)
    torch.cuda.synchronize()
    for (p, g, m, v), (dp, dg, dm, dv), c, wd in zip(host, t, copies, decay):
        rp, rm, rv = orc.adamw(p, g, m, v, step, weight_decay=wd, grad_scale=0.25, **HYPER)
        gs = np.abs(g.astype(np.float64)) * 0.25
        got = [x.double().cpu().numpy() for x in (dp, dm, dv)]
        assert (np.abs(got[1] - rm) <= 4 * U24 * (np.abs(m) + gs) + 1e-44).all()
        assert (np.abs(got[2] - rv) <= 6 * U24 * (v + gs * gs) + 1e-44).all()
        update = HYPER["lr"] / (1 - 0.9 ** step) * (np.abs(m) + gs) / (np.sqrt(rv / (1 - 0.98 ** step)) + 1e-8)
        assert (np.abs(got[0] - rp) <= 20 * U24 * (np.abs(p) + update)).all()
        assert (dg.cpu().numpy() == g).all()
        if c is not None:
            assert torch.equal(c, dp.to(torch.bfloat16))


def draw8(n, seed):
    r = np.random.default_rng(seed)
    p, g, _, _ = draw(n, seed)
    g *= np.exp(3 * r.standard_normal(n)).astype(np.float32)  # blocks of very different elements
    blocks = (n + 255) // 256
    mc = r.integers(0, 256, n).astype(np.uint8)
    mc[mc & 127 == 127] = 0
    rc = r.integers(0, 127, n).astype(np.uint8)
    ms, rs = (np.exp(r.standard_normal(blocks)) * 1e-5).astype(np.float32), (np.exp(r.standard_normal(blocks)) * 1e-5).astype(np.float32)
    return p, g, mc, ms, rc, rs


@pytest.mark.parametrize("offset", [0, 1])
def test_states_in_8_bits(offset):
    import torch
    host = [draw8(n, n) for n in SIZES]
    for h in host[3:5]:  # a block of zeros; one of values below the smallest normal float
        h[1][:256], h[2][:256], h[4][:256] = 0, 0, 0
    host[4][1][:256] = 1e-41
    t = [[dev(a, offset) for a in h] for h in host]
    copies = [torch.zeros(n + offset, dtype=torch.bfloat16, device="cuda")[offset:] for n in SIZES]
    plan = nm.nm_adamw_plan([x[0] for x in t], [x[1] for x in t], [x[2] for x in t], [x[4] for x in t], m_scales=[x[3] for x in t],
                            v_scales=[x[5] for x in t], copies=copies, weight_decay=0.02)
    for step, seed in ((7, 1234567), (8, 0xFFFFFFFF)):
        nm.nm_adamw_step(plan, step=step, seed=seed, **HYPER)
        torch.cuda.synchronize()
        block, after = 0, []
        for (p, g, mc, ms, rc, rs), d, c in zip(host, t, copies):
            rp, rmc, rms, rrc, rrs = orc.adamw8(p, g, mc, ms, rc, rs, block, seed, step, weight_decay=0.02, **HYPER)
            block += len(ms)
            got = [x.cpu().numpy() for x in d]
            assert (got[3] == rms.astype(np.float32)).all() and (got[5] == rrs.astype(np.float32)).all()
            assert (got[2] & 127 == rmc & 127).all() and ((got[2] == rmc) | (rmc & 127 == 0)).all() and (got[4] == rrc).all()
            m, r = np.abs(orc.e4m3_values()[mc]) * np.repeat(ms, 256)[:len(p)].astype(np.float64), orc.e4m3_values()[rc] * np.repeat(rs, 256)[:len(p)].astype(np.float64)
            root = np.sqrt((0.98 * r * r + 0.02 * g.astype(np.float64) ** 2) / (1 - 0.98 ** step))
            update = HYPER["lr"] / (1 - 0.9 ** step) * (m + np.abs(g)) / (root + 1e-8)
            assert (np.abs(got[0] - rp) <= 24 * U24 * (np.abs(p) + update) + 1e-44).all()
            assert torch.equal(c, d[0].to(torch.bfloat16))
            after.append((got[0], g, got[2], got[3], got[4], got[5]))
        host = after


def test_rounding_of_8_bit_states_keeps_the_mean():
    """A moment that changes by far less than a step: over many elements and steps the mean follows the true one."""
    import torch
    n, steps = 1 << 16, 40
    p, g = torch.zeros(n, device="cuda"), torch.full((n,), 1e-3, device="cuda")
    m, r = torch.zeros(n, dtype=torch.uint8, device="cuda"), torch.zeros(n, dtype=torch.uint8, device="cuda")
    g[::256] = 1.0  # a large neighbour in every block: the others' steps are coarse
    ms, rs = torch.ones(n // 256, device="cuda"), torch.ones(n // 256, device="cuda")
    plan = nm.nm_adamw_plan([p], [g], [m], [r], m_scales=[ms], v_scales=[rs])
    for s in range(1, steps + 1):
        nm.nm_adamw_step(plan, lr=1e-3, beta1=0.99, beta2=0.999, step=s, seed=s * 7919)
    torch.cuda.synchronize()
    val = torch.tensor(orc.e4m3_values(), device="cuda")
    mean = (val[m.long()] * ms.repeat_interleave(256)).view(-1, 256)[:, 1:].mean().item()
    true = 1e-3 * (1 - 0.99 ** steps)
    # an element's error is a sum of steps' roundings, each below a step (at most 1/8 of the value, 2^-9 of the scale), over n elements
    assert abs(mean - true) < 6 * steps ** 0.5 * max(true / 8, 2 ** -9 * ms.max().item()) / n ** 0.5
    assert torch.isfinite(p).all()


def test_infinite_and_nan_gradients_stay_where_they_are():
    import torch
    n = 600
    for bits in (32, 8):
        p, g, mc, ms, rc, rs = (dev(a) for a in draw8(n, 5))
        g[10], g[300] = float("inf"), float("nan")
        if bits == 8:
            plan = nm.nm_adamw_plan([p], [g], [mc], [rc], m_scales=[ms], v_scales=[rs])
        else:
            m, v = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
            plan = nm.nm_adamw_plan([p], [g], [m], [v])
        nm.nm_adamw_step(plan, step=2, seed=3, **HYPER)
        torch.cuda.synchronize()
        bad = ~torch.isfinite(p)
        assert bad.nonzero().flatten().tolist() == [10, 300]
        if bits == 8:
            assert (mc == 127).nonzero().flatten().tolist() == [10, 300] == (rc == 127).nonzero().flatten().tolist()
            assert torch.isfinite(ms).all() and torch.isfinite(rs).all()
