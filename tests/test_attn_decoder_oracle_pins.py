"""The float64 oracle of the attention decoder's operators against differences and simple facts (CPU)."""
import numpy as np
import pytest

from oracle import attn_decoder_oracle as orc

EPS = 1e-5  # of central differences: error of order EPS^2 times third derivatives, and 1e-16/EPS


def differences(fn, x):
    g = np.zeros(x.shape)
    for i in np.ndindex(x.shape):
        d = np.zeros(x.shape)
        d[i] = EPS
        g[i] = (fn(x + d) - fn(x - d)) / (2 * EPS)
    return g


@pytest.mark.parametrize("H,Hkv,windows", [(2, 2, False), (4, 2, True), (3, 1, False)])
def test_attention_gradients_are_the_differences(H, Hkv, windows):
    B, D, U, T, sc = 2, 3, 4, 5, 0.7
    r = np.random.default_rng(0)
    q, k, v, do = (r.standard_normal(s) for s in ((B, H * D, U), (B, Hkv * D, T), (B, Hkv * D, T), (B, H * D, U)))
    w = np.stack([r.integers(0, 3, (B, U)), r.integers(2, T + 2, (B, U))], 2) if windows else None
    ok = orc.allowed(B, U, T, [T, 3], [U, 2], w)
    loss = lambda q, k, v: (orc.attn_fwd(q, k, v, H, Hkv, sc, ok)[0] * do).sum()  # noqa: E731
    o, _, p, _ = orc.attn_fwd(q, k, v, H, Hkv, sc, ok)
    dq, dk, dv, _ = orc.attn_bwd(do, q, k, v, o, p, H, Hkv, sc)
    for got, ref in ((dq, differences(lambda x: loss(x, k, v), q)), (dk, differences(lambda x: loss(q, x, v), k)), (dv, differences(lambda x: loss(q, k, x), v))):
        assert np.abs(got - ref).max() < 1e-8


def test_attention_facts():
    B, H, D, U, T = 1, 2, 4, 3, 6
    r = np.random.default_rng(1)
    q, k = r.standard_normal((B, H * D, U)), r.standard_normal((B, H * D, T))
    ok = orc.allowed(B, U, T, [4], [2])
    o, lse, p, _ = orc.attn_fwd(q, k, np.ones((B, H * D, T)), H, H, 1.0, ok)
    assert np.allclose(o[:, :, :2], 1) and (o[:, :, 2] == 0).all() and np.isneginf(lse[:, :, 2]).all()
    assert np.allclose(p[:, :, :2].sum(3), 1) and (p[..., 4:] == 0).all()
    one = orc.allowed(B, U, T, [1])
    assert np.allclose(orc.attn_fwd(q, k, k, H, H, 1.0, one)[0], k[:, :, :1])  # one state: its value


@pytest.mark.parametrize("layer", [False, True])
@pytest.mark.parametrize("gate", [None, "item", "element"])
def test_norm_gradients_are_the_differences(layer, gate):
    B, C, T = 2, 5, 3
    r = np.random.default_rng(2)
    x, f, dy, dn = (r.standard_normal((B, C, T)) for _ in range(4))
    par = {n: r.standard_normal(C) for n in ("rscale", "post_weight", "next_weight")}
    par["post_bias"], par["next_bias"] = (r.standard_normal(C), r.standard_normal(C)) if layer else (None, None)
    par["gate"] = None if gate is None else r.random((B, C) if gate == "item" else (B, C, T))
    lengths = [T, 2]

    def loss(x, f, **kw):
        y, n = orc.norm_fwd(x, f, post=True, layer=layer, lengths=lengths, **dict(par, **kw))
        return sum((y[b, :, :t] * dy[b, :, :t] + n[b, :, :t] * dn[b, :, :t]).sum() for b, t in enumerate(lengths))

    y, _ = orc.norm_fwd(x, f, post=True, layer=layer, lengths=lengths, **par)
    got = orc.norm_bwd(dy, dn, y, f, post=True, layer=layer, lengths=lengths, **{k: v for k, v in par.items() if k != "next_bias"})
    assert np.abs(got["dx"] - differences(lambda a: loss(a, f), x)).max() < 1e-7
    assert np.abs(got["df"] - differences(lambda a: loss(x, a), f)).max() < 1e-7
    for n, v in par.items():
        if v is not None:
            name = "d" + n if n != "gate" else "dgate_" + gate
            assert np.abs(got[name] - differences(lambda a: loss(x, f, **{n: a}), v)).max() < 1e-7, n  # noqa: B023


def test_adamw_facts():
    """Without momentum and decay the first step is lr times the gradient's sign; weight decay alone shrinks."""
    g = np.array([3.0, -0.2, 1e-4])
    p, m, v = orc.adamw(np.ones(3), g, np.zeros(3), np.zeros(3), 1, 0.1, 0.0, 0.9, 1e-12, 0.0)
    assert np.allclose(p, 1 - 0.1 * np.sign(g)) and np.allclose(m, g) and np.allclose(v, 0.1 * g * g)
    p, _, _ = orc.adamw(np.ones(3), np.zeros(3), np.zeros(3), np.zeros(3), 5, 0.1, 0.9, 0.9, 1e-8, 0.5)
    assert np.allclose(p, 0.95)


def test_codes_are_those_of_torch_and_rounding_is_unbiased():
    torch = pytest.importorskip("torch")
    val = orc.e4m3_values()
    ref = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert ((val == ref) | (np.isnan(val) & np.isnan(ref))).all()
    for z in (0.3, 5.1, 447.0, 2.0 ** -8.5, 1e-4):
        got = np.mean([val[orc._encode(z, 1.0, u, False)] for u in range(0, 65536, 16)])
        assert abs(got - z) < max(z / 8, 2 ** -9) / 1000
    assert orc._encode(1e-4, 1.0, 0, True) == 1 and orc._encode(0.0, 1.0, 65535, True) == 0 and orc._encode(-448.0, 1.0, 65535, False) == 254
    bits = np.array([orc.mixed(e, 5) for e in range(20000)])
    assert abs((bits & 0xFFFF).mean() / 65536 - 0.5) < 0.01 and abs((bits >> 16).mean() / 65536 - 0.5) < 0.01
    assert abs(np.corrcoef(bits & 0xFFFF, bits >> 16)[0, 1]) < 0.03
