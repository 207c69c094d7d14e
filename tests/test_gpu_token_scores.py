"""Token scores on the GPU against the float64 oracle.

Tolerances (derived, per element; u = 2^-24).  A lane adds at most V/4 exponentials in a row and joins some dozens of sums: d = V/4 + 64
roundings.  An exponential is off by 2u of its argument's magnitude in powers of two and two units, and the arguments' mean magnitude is at most
the entropy and the logarithm of the sum.  So the log-sum-exp is off by d*u + (entropy + log V + 4)*4u and by 4u of itself, an entropy by
three times that in its terms (their magnitudes are at most entropy + log V + 1).  A gradient's probability is off by 4u of its
logarithm's and the log-sum-exp's magnitudes; results are rounded once to the type of the gradient.  Below 2^-126 float32 has no
full digits and the exponential gives zero: a probability is off by that much too, a gradient by that times what multiplies it."""
import numpy as np
import pytest

from oracle import token_oracle as orc
from paper_1909_09577_amd import binding as nm
from test_gpu_cross_attn import STEP, check, host, to
from test_gpu_head_norm import ints

pytestmark = pytest.mark.gpu
u_ = 2.0 ** -24


def both(got, ref, tol, what):
    """Infinities in the same places, the rest within tol."""
    inf = np.isinf(ref)
    assert np.array_equal(np.where(inf, got, 0), np.where(inf, ref, 0)), what
    check(np.where(inf, 0, got), np.where(inf, 0, ref), np.where(inf, 1, tol), what)


def run_and_check(B, V, U, dtype, *, top=0, lengths=None, barred=0.0, grad=None, wide=True, seed=0, big=3.0, ties=False, targets=True, entropy=True):
    import torch
    r = np.random.default_rng(seed)
    z = big * r.standard_normal((B, V, U))
    if ties:
        z = np.round(z)
    z[r.random((B, V, U)) < barred] = -np.inf
    z = host(to(z, dtype))
    t = r.integers(-1, V + 1, (B, U)) if targets else None
    dev = to(z, dtype)
    if lengths is not None:
        for b, n in enumerate(lengths):
            dev[b, :, max(n, 0):] = float("nan")
    tt = None if t is None else torch.from_numpy(t).cuda().to(torch.int64 if wide else torch.int32)
    print(f"case {B} {V} {U} {dtype} top {top} {lengths} {barred}", flush=True)
    got = nm.nm_token_scores_fwd(dev, tt, top=top, lengths=ints(lengths))
    ref = orc.token_scores(z, t, top, lengths)
    assert set(got) == {"entropy", "lse"} | ({"logp"} if targets else set()) | ({"top_ids", "top_logp"} if top else set())
    h = {k: host(v) for k, v in got.items()}
    finite = lambda a: np.where(np.isfinite(a), np.abs(a), 0)  # noqa: E731
    terms = ref["entropy"] + np.log(V) + 4
    off = (V / 4 + 64) * u_ + terms * 4 * u_ + finite(ref["lse"]) * 4 * u_
    both(h["lse"], ref["lse"], off, "lse")
    both(h["entropy"], ref["entropy"], 3 * ((V / 4 + 64) * u_ + 8 * u_) * terms, "entropy")
    if targets:
        both(h["logp"], ref["logp"], off + finite(ref["logp"]) * 2 * u_, "logp")
    if top:
        assert np.array_equal(h["top_ids"], ref["top_ids"])
        both(h["top_logp"], ref["top_logp"], off[:, None] + finite(ref["top_logp"]) * 2 * u_, "top_logp")
    if not targets and not entropy:
        return
    dl = r.standard_normal((B, U)).astype(np.float32) if targets else None
    dh = r.standard_normal((B, U)).astype(np.float32) if entropy else None
    f32 = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a, np.float32)).cuda()  # noqa: E731
    gdt = None if grad is None else torch.bfloat16 if grad == "bf16" else torch.float32
    g = nm.nm_token_scores_bwd(dev, tt, f32(ref["lse"]), f32(ref["entropy"]) if entropy else None, f32(dl), f32(dh), lengths=ints(lengths), dtype=gdt)
    rg, mag, logs = orc.token_scores_bwd(z, t, dl, dh, lengths)
    rel = (np.abs(logs) + finite(ref["lse"])[:, None] + finite(ref["entropy"])[:, None] + 8) * 4 * u_
    least = 2.0 ** -126 * ((0 if dl is None else np.abs(dl)[:, None]) + (0 if dh is None else np.abs(dh)[:, None] * (np.abs(logs) + ref["entropy"][:, None])))
    check(host(g), rg, STEP[grad or dtype] * np.abs(rg) + 2 * rel * mag + 2 * least + (np.abs(dh)[:, None] * np.exp(logs) * rel * 2 if entropy else 0), "dscores")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("U", [1, 2, 3, 5, 7, 8, 9, 13, 33, 64, 65, 100])
def test_places(U, dtype):
    run_and_check(2, 29, U, dtype, top=5)
    run_and_check(1, 700, U, dtype, top=1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [1, 2, 15, 16, 17, 64, 1000, 9001])
def test_vocabularies(V, dtype):
    run_and_check(3, V, 1, dtype, top=min(V, 16))
    run_and_check(2, V, 11, dtype, top=min(V, 8), wide=False)


@pytest.mark.parametrize("top", [0, 1, 2, 3, 4, 5, 8, 9, 16])
@pytest.mark.parametrize("ties", [False, True])
def test_alternatives(top, ties):
    """Of equal scores the lower class comes first."""
    run_and_check(2, 500, 1, "bf16", top=top, ties=ties)
    run_and_check(2, 500, 40, "f32", top=top, ties=ties)
    run_and_check(1, 6000, 2, "f32", top=top, ties=ties)


@pytest.mark.parametrize("barred", [0.3, 0.97, 1.0])
def test_barred_classes(barred):
    run_and_check(3, 40, 5, "f32", top=16, barred=barred)
    run_and_check(2, 300, 50, "bf16", top=4, barred=barred)
    run_and_check(2, 5000, 1, "f32", top=8, barred=barred)


@pytest.mark.parametrize("lengths", [[20, 0, 1], [100, -1, 9]], ids=str)
def test_lengths(lengths):
    for U in (1, 6, 20, 70):
        run_and_check(3, 60, U, "bf16", top=3, lengths=lengths)
    run_and_check(3, 4000, 20, "f32", top=3, lengths=lengths)


@pytest.mark.parametrize("U", [1, 6, 30])
def test_parts(U):
    run_and_check(2, 90, U, "bf16", grad="f32")
    run_and_check(2, 90, U, "f32", grad="bf16", entropy=False)
    run_and_check(2, 90, U, "f32", targets=False)
    run_and_check(2, 90, U, "f32", targets=False, entropy=False, top=2)


def test_wide_rows():
    run_and_check(1, 3, 2200, "f32", top=2)
    run_and_check(1, 2, 4100, "bf16")


def test_large_scores():
    run_and_check(2, 400, 9, "f32", top=4, big=300.0)


def test_what_is_not_a_number():
    """A NaN makes its place's results NaN and is behind all others in order; +infinity gives NaN."""
    import torch
    z = torch.randn(1, 50, 10, device="cuda")
    z[0, 7, 3] = float("nan")
    z[0, 9, 4] = float("inf")
    got = nm.nm_token_scores_fwd(z, torch.zeros(1, 10, dtype=torch.int64, device="cuda"), top=2)
    bad = torch.zeros(10, dtype=torch.bool, device="cuda")
    bad[3] = bad[4] = True
    for name in ("lse", "entropy", "logp"):
        assert torch.equal(got[name][0].isfinite(), ~bad), name
    assert got["top_ids"][0, 0, 4] == 9 and 7 not in got["top_ids"][0, :, 3].tolist()
    z[:] = float("nan")
    assert nm.nm_token_scores_fwd(z, top=2)["top_ids"][0, :, 0].tolist() == [0, 1]


def test_gradients_are_the_differences():
    import torch
    B, V, U = 1, 12, 9
    g = torch.Generator(device="cuda").manual_seed(0)
    z, dl, dh = torch.randn(B, V, U, device="cuda", generator=g), torch.randn(B, U, device="cuda", generator=g), torch.randn(B, U, device="cuda", generator=g)
    t = torch.randint(0, V, (B, U), device="cuda", generator=g)
    f = nm.nm_token_scores_fwd(z, t)
    grad = nm.nm_token_scores_bwd(z, t, f["lse"], f["entropy"], dl, dh)

    def total(z):
        got = nm.nm_token_scores_fwd(z, t)
        return (got["logp"].double() * dl + got["entropy"].double() * dh).sum().item()

    eps = 2.0 ** -7  # error eps^2 times third derivatives of order one; 18 float32 results of order two, off by 2^-22 each, over eps: 6e-4
    for v, u in ((0, 0), (5, 3), (11, 8), (3, 4)):
        e = torch.zeros_like(z)
        e[0, v, u] = eps
        assert abs((total(z + e) - total(z - e)) / (2 * eps) - grad[0, v, u].item()) < 2e-3
