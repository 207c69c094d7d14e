"""Token scores at the ends of their type's range: places filled with its lowest value, largest values, and scores so large that a float32
log-sum-exp holds little of the logarithm of the sum.

Reference: float64, from the definitions, with the largest score and the logarithm of the sum apart (their sum holds nothing of the latter beyond 2^53).

Tolerances (derived, per element; u = 2^-24), as those of the tests of ordinary scores but for these: the largest score is subtracted first, so
that what is left is off by u of itself, and a log-probability does not see the log-sum-exp's magnitude; the log-sum-exp is rounded once.  The gradient goes
by the rounded log-sum-exp of the forward pass: up to a magnitude of 4096 a probability is off by that rounding, beyond by a sum over the
classes like the forward pass's (d = V/4 + 64 roundings in each)."""
import numpy as np
import pytest

from paper_1909_09577_amd import binding as nm
from test_gpu_cross_attn import STEP, check, host, to
from test_gpu_head_norm import ints

pytestmark = pytest.mark.gpu
u_ = 2.0 ** -24
LOWEST = {"bf16": -(2.0 - 2.0 ** -7) * 2.0 ** 127, "f32": -(2.0 - 2.0 ** -23) * 2.0 ** 127}


def run_and_check(z, dtype, *, top=3, lengths=None, grad=None, seed=0):
    import torch
    r = np.random.default_rng(seed)
    B, V, U = z.shape
    dev = to(z, dtype)
    z = host(dev)
    print(f"case {z.shape} {dtype} top {top} {lengths}", flush=True)
    t, top = r.integers(0, V, (B, U)), min(top, V)
    ok = np.ones((B, U), bool) if lengths is None else np.arange(U)[None] < np.asarray(lengths)[:, None]
    best = z.max(1)
    with np.errstate(invalid="ignore"):
        x = np.where(z > -np.inf, z - best[:, None], -np.inf)
    e = np.exp(x)
    log_s = np.log(e.sum(1))
    logq = x - log_s[:, None]
    q, safe = np.exp(logq), np.where(np.isfinite(logq), logq, 0)
    H = -(q * safe).sum(1)
    at = lambda a: np.take_along_axis(a, t[:, None], 1)[:, 0]  # noqa: E731
    dt = torch.from_numpy(t).cuda()
    got = nm.nm_token_scores_fwd(dev, dt, top=top, lengths=ints(lengths))
    h = {k: host(v) for k, v in got.items()}
    d, terms = (V / 4 + 64) * u_, H + np.log(V) + 4

    def near(name, ref, tol):
        valid = ok if ref.ndim == 2 else np.broadcast_to(ok[:, None], ref.shape)
        # a difference of two scores may be as low as -2^129; from -2^128 + 2^103 down float32 has no finite number that is nearest
        with np.errstate(over="ignore"):
            inf = np.isneginf(ref.astype(np.float32)) & valid
        assert np.array_equal(np.isneginf(h[name]), inf), name
        check(np.where(inf, 0, h[name]), np.where(valid & ~inf, ref, 0), np.where(valid & ~inf, tol, 0), name)

    finite = lambda a: np.where(np.isfinite(a), np.abs(a), 0)  # noqa: E731
    near("lse", best + log_s, d + terms * 4 * u_ + np.abs(best + log_s) * 2 * u_)
    near("entropy", H, 3 * (d + 8 * u_) * terms)
    near("logp", at(logq), d + terms * 4 * u_ + finite(at(logq)) * 2 * u_)
    order = np.argsort(-z, axis=1, kind="stable")[:, :top]
    assert np.array_equal(h["top_ids"], np.where(ok[:, None], order, -1))
    near("top_logp", np.take_along_axis(logq, order, 1), d + terms[:, None] * 4 * u_ + finite(np.take_along_axis(logq, order, 1)) * 2 * u_)

    dl, dh = (r.standard_normal((B, U)).astype(np.float32) for _ in range(2))
    gdt = None if grad is None else torch.bfloat16 if grad == "bf16" else torch.float32
    f = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    g = nm.nm_token_scores_bwd(dev, dt, got["lse"], got["entropy"], f(dl), f(dh), lengths=ints(lengths), dtype=gdt)
    hot = np.arange(V)[None, :, None] == t[:, None]
    ref = dl[:, None] * (hot - q) - dh[:, None] * q * (safe + H[:, None])
    large = np.abs(best + log_s)[:, None]
    rel = np.where(large > 4000, 2 * d, 2 * large * u_) + (np.abs(safe) + H[:, None] + 8) * 4 * u_ + 2 * d
    mag = np.abs(dl)[:, None] * (hot + q) + np.abs(dh)[:, None] * q * (np.abs(safe) + H[:, None] + 1)
    least = 2.0 ** -126 * (np.abs(dl)[:, None] + np.abs(dh)[:, None] * (np.abs(safe) + H[:, None]))
    tol = STEP[grad or dtype] * np.abs(ref) + 2 * np.minimum(rel, 1) * mag + 2 * least
    check(host(g), np.where(ok[:, None], ref, 0), np.where(ok[:, None], tol, 0), "dscores")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V, U", [(1, 1), (29, 1), (5000, 1), (29, 5), (700, 7), (29, 8), (700, 9), (5000, 40), (60, 2100)])
def test_places_of_the_lowest_value(V, U, dtype):
    """What a mask leaves that fills with the type's lowest value and bars every class: all are equally likely."""
    run_and_check(np.full((2, V, U), LOWEST[dtype]), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V, U", [(40, 1), (3000, 2), (300, 33)])
def test_some_places_and_classes_of_the_lowest_value(V, U, dtype):
    r = np.random.default_rng(1)
    z = 3 * r.standard_normal((3, V, U))
    z[:, ::3] = LOWEST[dtype]
    z[:, 1::3] = -np.inf
    z[0, 2::3] = LOWEST[dtype]  # (nothing else is left there)
    run_and_check(z, dtype, lengths=[U, max(U - 1, 1), U])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V, U", [(17, 1), (3000, 3), (500, 20)])
def test_largest_values(V, U, dtype):
    r = np.random.default_rng(2)
    z = 3 * r.standard_normal((4, V, U))
    z[0, 5] = 3e38
    z[1, [2, V - 1]] = 3e38
    z[1, 3] = LOWEST[dtype]
    z[2, 1] = -LOWEST[dtype]
    z[2, 7::2] = LOWEST[dtype]
    z[3] = -LOWEST[dtype]
    run_and_check(z, dtype)


@pytest.mark.parametrize("big", [2e3, 1e4, 3e5, 1e9, 1e30])
@pytest.mark.parametrize("V, U", [(30, 1), (900, 6), (900, 8), (2000, 50)])
def test_large_scores_close_together(V, U, big):
    """The classes that count differ by little, the log-sum-exp holds little of the logarithm of their number."""
    r = np.random.default_rng(3)
    z = np.float32(big) + np.float32(np.spacing(np.float32(big))) * r.integers(-2, 3, (2, V, U)) + np.where(big < 1e5, r.standard_normal((2, V, U)), 0)
    run_and_check(z, "f32")
    run_and_check(-z, "f32", grad="bf16", lengths=[U, max(U - 2, 1)])


def test_a_gradient_of_large_scores_replayed():
    """The sums over the classes are made within the call."""
    import torch
    z = torch.full((2, 300, 12), LOWEST["f32"], device="cuda")
    z[1] = torch.randn(300, 12, device="cuda")
    t = torch.zeros(2, 12, dtype=torch.int64, device="cuda")
    of = nm.nm_token_scores_fwd(z, t)
    dl = torch.ones(2, 12, device="cuda")
    want = nm.nm_token_scores_bwd(z, t, of["lse"], None, dl)
    out = torch.empty_like(want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        nm.nm_token_scores_bwd(z, t, of["lse"], None, dl, dscores=out)
    for _ in range(3):
        out.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
