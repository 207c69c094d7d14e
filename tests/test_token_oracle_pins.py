"""The float64 oracle of the operators on tokens against differences and simple facts (CPU)."""
import numpy as np
import pytest

from oracle import token_oracle as orc
from test_attn_decoder_oracle_pins import differences


def test_embedding():
    r = np.random.default_rng(0)
    ids, table = np.array([[2, 0, 2], [5, -1, 1]]), r.standard_normal((4, 3))
    out = orc.embedding_fwd(ids, table, 2.0, [3, 2])
    assert np.allclose(out[0], 2 * table[[2, 0, 2]].T) and (out[1] == 0).all()
    dout = r.standard_normal((2, 3, 3))
    got, mag, count = orc.embedding_bwd(dout, ids, 4, 2.0, [3, 2])
    ref = differences(lambda t: (orc.embedding_fwd(ids, t, 2.0, [3, 2]) * dout).sum(), table)
    assert np.abs(got - ref).max() < 1e-8 and list(count) == [1, 0, 2, 0] and (mag >= np.abs(got) - 1e-12).all()


@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("rot", [0, 2, 6])
@pytest.mark.parametrize("norm", [False, True])
def test_head_norm(norm, rot, pairs):
    B, H, Hkv, D, U = 2, 2, 1, 6, 3
    r = np.random.default_rng(1)
    x, dout = (r.standard_normal((B, (H + Hkv) * D, U)) for _ in range(2))
    qw, kw = (r.standard_normal(D), r.standard_normal(D)) if norm else (None, None)
    kws = dict(norm=norm, qw=qw, kw=kw, freqs=100.0 ** -np.arange(rot // 2), pairs=pairs, positions=r.integers(0, 50, (B, U)), lengths=[3, 2])
    f = lambda **k: (orc.head_norm_fwd(k.pop("x", x), H, Hkv, **dict(kws, **k))[0] * dout).sum()  # noqa: E731
    dx, dqw, dkw, _ = orc.head_norm_bwd(dout, x, H, Hkv, **kws)
    assert np.abs(dx - differences(lambda t: f(x=t), x)).max() < 1e-8
    if norm:
        assert np.abs(dqw - differences(lambda t: f(qw=t), qw)).max() < 1e-8 and np.abs(dkw - differences(lambda t: f(kw=t), kw)).max() < 1e-8
    else:
        out, _ = orc.head_norm_fwd(x, H, Hkv, **kws)  # turning changes no length
        assert np.allclose((out ** 2).sum(1)[0], (x ** 2).sum(1)[0])


def test_turning_depends_on_distance_alone():
    r = np.random.default_rng(2)
    q, k, freqs = r.standard_normal(8), r.standard_normal(8), [1.0, 0.3, 0.01, 0.002]
    dots = [orc.turned(q, p + 5, freqs, pairs)[0] @ orc.turned(k, p, freqs, pairs)[0] for p in (0, 7, 1000) for pairs in (False,)]
    assert np.ptp(dots) < 1e-10


def test_cache_and_attention():
    B, H, Hkv, D, U, page = 2, 4, 2, 16, 3, 4
    r = np.random.default_rng(3)
    table = np.array([[2, 0, -1], [1, 9, 3]])
    k, v = r.standard_normal((5, Hkv, page, D)), r.standard_normal((5, Hkv, D, page))
    x = r.standard_normal((B, (H + 2 * Hkv) * D, U))
    (q, k2, v2), (_, mk, _) = orc.head_norm_cache(x, k, v, table, [7, 4], H, Hkv, norm=False, q_lengths=[3, 2])
    assert np.allclose(k2[0, :, 0:3], x[0, H * D:(H + Hkv) * D].reshape(Hkv, D, 3).transpose(0, 2, 1))  # places 4..6: page 0
    assert np.allclose(v2[1, :, :, 2:4], x[1, (H + Hkv) * D:, :2].reshape(Hkv, D, 2))               # places 2, 3: page 1
    touched = np.zeros(5, bool)
    touched[[0, 1]] = True
    assert ((k2 != k).any((1, 2, 3)) == touched).all() and (mk[~touched] == 0).all() and (q[1, :, 2] == 0).all()
    o, lse, _, _ = orc.paged_attn(q, k2, v2, table, [7, 4], H, Hkv, 0.25, q_lengths=[3, 2])
    assert np.isneginf(lse[1, :, 2]).all() and (o[1, :, 2] == 0).all() and np.isfinite(lse[0]).all()
    one, _, _, _ = orc.paged_attn(q, k2, v2, table, [7, 4], H, Hkv, 0.25, q_lengths=[3, 2], window=1)  # itself alone: its value
    assert np.allclose(one[0, :, 1].reshape(H, D), np.repeat(v2[0, :, :, 1], 2, 0))
    # a place on a page that is none of the cache's is as if it were not there
    far, _, _, _ = orc.paged_attn(q, k2, v2, table, [7, 6], H, Hkv, 0.25, q_lengths=[3, 1])
    near, _, _, _ = orc.paged_attn(q, k2, v2, table, [7, 4], H, Hkv, 0.25, q_lengths=[3, 1])
    assert np.allclose(far[1], near[1])


def test_token_scores():
    r = np.random.default_rng(4)
    B, V, U = 2, 5, 3
    z, targets = r.standard_normal((B, V, U)), r.integers(0, V, (B, U))
    z[0, 1, 0] = -np.inf
    targets[1, 1] = -1
    targets[0, 0] = 2
    got = orc.token_scores(z, targets, 3, [3, 2])
    assert np.isclose(got["logp"][0, 0], z[0, 2, 0] - got["lse"][0, 0]) and got["logp"][1, 1] == 0 and got["lse"][1, 2] == 0
    assert got["top_ids"][1, 0, 2] == -1 and got["top_ids"][0, 0, 1] == z[0, :, 1].argmax()
    dl, dh = r.standard_normal((B, U)), r.standard_normal((B, U))

    def total(z):
        g = orc.token_scores(z, targets, 0, [3, 2])
        return (g["logp"] * dl + np.where(np.arange(U) < np.array([[3], [2]]), g["entropy"], 0) * dh).sum()

    grad, mag, _ = orc.token_scores_bwd(z, targets, dl, dh, [3, 2])
    z[0, 1, 0] = 0  # (differences at -infinity are none)
    grad, _, _ = orc.token_scores_bwd(z, targets, dl, dh, [3, 2])
    assert np.abs(grad - differences(total, z)).max() < 1e-8
    z[1, :, 0] = -np.inf
    got = orc.token_scores(z, targets, 2, None)
    assert np.isneginf(got["lse"][1, 0]) and got["entropy"][1, 0] == 0 and list(got["top_ids"][1, :, 0]) == [0, 1]
