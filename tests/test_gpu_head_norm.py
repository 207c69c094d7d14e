"""Norms and rotation of queries and keys on the GPU against the float64 oracle.

Tolerances (derived, per element).  The mean of D squares is off by (D+2)*2^-24 of itself, so 1/rms by half of that and three roundings; a
normalised value has three more, the angle's fraction is rounded to 2^-25 of half a turn (less than 2^-23 in the result) and its
cosine and sine by two units: (D+16)*2^-24 of the magnitudes that a turned value adds.  A gradient sees 1/rms three times, the mean of D
products and again two turned terms: (3D+48)*2^-24.  A sum over n tokens and heads has n more roundings.  Results are rounded once to the storage type."""
import numpy as np
import pytest

from oracle import token_oracle as orc
from paper_1909_09577_amd import binding as nm
from test_gpu_cross_attn import STEP, check, host, to

pytestmark = pytest.mark.gpu


def ints(a):
    import torch
    return None if a is None else torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


def setup(H, Hkv, D, rot, norm, weights, seed):
    import torch
    r = np.random.default_rng(seed)
    w = [1 + 0.3 * r.standard_normal(D).astype(np.float32) if weights and n else None for n in (H, Hkv)]
    freqs = 10000.0 ** (-np.arange(0, rot, 2) / max(rot, 1))
    dev = dict(heads=H, kv_heads=Hkv, norm=norm, q_weight=None if w[0] is None else torch.from_numpy(w[0]).cuda(),
               k_weight=None if w[1] is None else torch.from_numpy(w[1]).cuda(), freqs=torch.from_numpy(freqs).cuda() if rot else None)
    return r, dict(norm=norm, qw=w[0], kw=w[1], freqs=freqs), dev


def run_and_check(B, H, Hkv, D, U, dtype, *, rot=None, norm=True, weights=True, pairs=False, positions=None, lengths=None, seed=0, apart=False):
    import torch
    rot = D if rot is None else rot
    r, ref_kw, dev = setup(H, Hkv, D, rot, norm, weights and norm, seed)
    C = (H + Hkv) * D
    x, dout = (host(to(r.standard_normal((B, C, U)) * s, dtype)) for s in (2.0, 1.0))
    if positions == "far":
        positions = r.integers(0, 10 ** 6, (B, U))
    ref_kw.update(pairs=pairs, positions=positions, lengths=lengths)
    dev.update(pairs=pairs, positions=ints(positions), lengths=ints(lengths))
    print(f"case {B} {H} {Hkv} {D} {U} {dtype} {rot} {norm} {pairs} {lengths}", flush=True)

    def place(a):  # items apart: the first part of a larger projection
        if not apart:
            return to(a, dtype)
        big = torch.full((B, C + 3 * D, U), float("nan"), device="cuda", dtype=torch.bfloat16 if dtype == "bf16" else torch.float32)
        big[:, :C] = to(a, dtype)
        return big[:, :C]

    dx_in, g_in = place(x), place(dout)
    if lengths is not None:
        for b, n in enumerate(lengths):
            dx_in[b, :, max(n, 0):] = float("nan")
            g_in[b, :, max(n, 0):] = float("nan")
    out = nm.nm_head_norm_fwd(dx_in, **dev)
    ref, mag = orc.head_norm_fwd(x, H, Hkv, **ref_kw)
    check(host(out), ref, STEP[dtype] * np.abs(ref) + (D + 16) * 2.0 ** -24 * mag, "out")
    to_dx = place(np.zeros_like(x)) if apart else None
    dx, dqw, dkw = nm.nm_head_norm_bwd(g_in, dx_in, dx=to_dx, **dev)
    rx, rq, rk, m = orc.head_norm_bwd(dout, x, H, Hkv, **ref_kw)
    check(host(dx), rx, STEP[dtype] * np.abs(rx) + (3 * D + 48) * 2.0 ** -24 * m["dx"], "dx")
    if dev["q_weight"] is not None:
        check(host(dqw), rq, (D + 32 + B * U * H) * 2.0 ** -24 * m["dqw"], "dq_weight")
    else:
        assert dqw is None
    if dev["k_weight"] is not None:
        check(host(dkw), rk, (D + 32 + B * U * Hkv) * 2.0 ** -24 * m["dkw"], "dk_weight")
    else:
        assert dkw is None


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("U", [1, 7, 8, 9, 31, 32, 33, 70])
def test_lengths_of_rows(U, dtype):
    run_and_check(2, 3, 1, 64, U, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,rot", [(2, 2), (16, 8), (32, 32), (64, 0), (80, 80), (96, 48), (98, 30), (128, 128), (128, 2)])
@pytest.mark.parametrize("pairs", [False, True])
def test_widths(D, rot, pairs, dtype):
    for U in (3, 41):
        run_and_check(2, 5, 2, D, U, dtype, rot=rot, pairs=pairs, positions="far" if U == 41 else None)


@pytest.mark.parametrize("U", [5, 45])
def test_parts(U):
    run_and_check(2, 2, 0, 64, U, "bf16")                       # queries alone
    run_and_check(2, 2, 1, 64, U, "bf16", norm=False)            # rotation alone
    run_and_check(2, 2, 1, 64, U, "f32", norm=False, pairs=True)
    run_and_check(2, 2, 1, 64, U, "bf16", weights=False)         # a norm without weights
    run_and_check(2, 9, 6, 48, U, "bf16", apart=True)
    run_and_check(1, 1, 1, 64, U, "bf16", norm=False, rot=0)


@pytest.mark.parametrize("lengths", [[45, 0, 1], [100, -1, 33], [20, 32, 44]], ids=str)
def test_ragged(lengths):
    run_and_check(3, 2, 1, 64, 45, "bf16", lengths=lengths)
    run_and_check(3, 2, 1, 64, 6, "bf16", lengths=lengths)
    run_and_check(3, 2, 1, 64, 20, "f32", lengths=lengths)


def test_more_tiles_than_workgroups_side_by_side():
    run_and_check(7, 1, 1, 16, 32 * 150 + 5, "bf16")


def test_gradients_are_the_differences():
    """The float32 gradient of a sum against central differences of the forward call."""
    import torch
    H, Hkv, D, U = 1, 1, 16, 9
    _, _, dev = setup(H, Hkv, D, 12, True, True, 3)
    g = torch.Generator(device="cuda").manual_seed(0)
    x, d = (torch.randn(1, 2 * D, U, device="cuda", generator=g) for _ in range(2))
    dx, dqw, _ = nm.nm_head_norm_bwd(d, x, **dev)
    f = lambda x, **kw: (nm.nm_head_norm_fwd(x, **dict(dev, **kw)).double() * d.double()).sum().item()  # noqa: E731
    eps = 2.0 ** -7  # error eps^2 times third derivatives of order one, and 2^-24 * 3 * sqrt(2*D*U) / eps = 4e-4 of float32
    for i, u in ((0, 0), (5, 3), (13, 8), (20, 4), (31, 7)):
        e = torch.zeros_like(x)
        e[0, i, u] = eps
        assert abs((f(x + e) - f(x - e)) / (2 * eps) - dx[0, i, u].item()) < 3e-3
    for i in (0, 11, 15):
        e = torch.zeros(D, device="cuda")
        e[i] = eps
        assert abs((f(x, q_weight=dev["q_weight"] + e) - f(x, q_weight=dev["q_weight"] - e)) / (2 * eps) - dqw[i].item()) < 3e-3


def cache_case(B, H, Hkv, D, U, dtype, page, lengths, *, q_lengths=None, rot=None, norm=True, pairs=False, table=None, spare=2, seed=0):
    import torch
    rot = D if rot is None else rot
    r, ref_kw, dev = setup(H, Hkv, D, rot, norm, norm, seed)
    n = max(1, -(-max(max(lengths), 1) // page))
    if table is None:
        table = r.permutation(B * n + spare)[:B * n].reshape(B, n)
    pages = B * n + spare
    x, k, v = (host(to(r.standard_normal(s), dtype)) for s in ((B, (H + 2 * Hkv) * D, U), (pages, Hkv, page, D), (pages, Hkv, D, page)))
    print(f"case {B} {H} {Hkv} {D} {U} {dtype} page {page} {lengths} {q_lengths}", flush=True)
    (rq, rk, rv), (mq, mk, mv) = orc.head_norm_cache(x, k, v, table, lengths, H, Hkv, q_lengths=q_lengths, pairs=pairs, **ref_kw)
    dk, dv = to(k, dtype), to(v, dtype)
    q = nm.nm_head_norm_cache(to(x, dtype), dk, dv, ints(table), ints(lengths), q_lengths=ints(q_lengths), pairs=pairs, **dev)
    tol = lambda ref, mag: np.where(mag > 0, STEP[dtype] * np.abs(ref), 0) + (D + 16) * 2.0 ** -24 * mag  # noqa: E731  (untouched: the same)
    check(host(q), rq, tol(rq, mq), "q")
    check(host(dk), rk, tol(rk, mk), "k_cache")
    assert np.array_equal(host(dv), rv), "v_cache"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("U", [1, 5, 40])
def test_cache(U, page, dtype):
    cache_case(3, 4, 2, 64, U, dtype, page, [U, U + page - 1, 2 * page + 3 + U])


def test_cache_of_ragged_chunks_and_other_widths():
    cache_case(3, 4, 1, 80, 20, "bf16", 16, [33, 20, 1], q_lengths=[20, 0, 1], rot=40, pairs=True)
    cache_case(2, 2, 2, 18, 9, "f32", 32, [100, 9], q_lengths=[30, -2], norm=False)
    cache_case(1, 3, 3, 128, 1, "bf16", 64, [100000 % 7000], norm=False, rot=0)


@pytest.mark.parametrize("table,lengths", [([[0, -1], [1, 2]], [40, 20]), ([[0, 99], [1, 2]], [40, 20]), ([[0, 3], [1, 2]], [5, -7]),
                                           ([[0, 3], [1, 2]], [500, 2 ** 31 - 1]), ([[0, 3], [1, 2]], [34, -2 ** 31])], ids=str)
def test_tokens_without_a_place_are_not_written(table, lengths):
    import torch
    if max(lengths) < 64:
        cache_case(2, 2, 1, 32, 8, "bf16", 16, lengths, table=np.array(table), spare=4)
    x = torch.randn(2, 4 * 32, 8, device="cuda").bfloat16()
    k, v = torch.zeros(8, 1, 16, 32, device="cuda").bfloat16(), torch.zeros(8, 1, 32, 16, device="cuda").bfloat16()
    nm.nm_head_norm_cache(x, k, v, ints(table), ints(lengths), heads=2, kv_heads=1)
    (_, rk, rv), _ = orc.head_norm_cache(host(x), host(k) * 0, host(v) * 0, np.array(table), [min(n, 10 ** 6) for n in lengths], 2, 1, norm=True)
    assert ((host(k) != 0) == (rk != 0)).all() and np.array_equal(host(v), rv)
