"""The norms around a block on the GPU against the float64 oracle: storage types, gates, norms present and absent, padded batches,
channel counts and lengths that fill no group.

Tolerances (derived): outputs are rounded once to the storage type (2^-8 or 2^-24 of the value); the float32 arithmetic before it,
sums over C channels among it, is off by a few C * 2^-24 of the magnitudes involved, which near C = 1000 stays below 2e-4 of the rms
of a row for any order of the sum and is taken as (C + 64) * 2^-24 * rms here; sums over n positions by n * 2^-24 of the sum of
their terms' magnitudes on top."""
import numpy as np
import pytest

from oracle import attn_decoder_oracle as orc
from paper_1909_09577_amd import binding as nm

pytestmark = pytest.mark.gpu
STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


def to(a, dtype):
    import torch
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a, np.float32)).cuda().to(torch.bfloat16 if dtype == "bf16" else torch.float32)


def host(t):
    import torch
    torch.cuda.synchronize()
    return t.double().cpu().numpy()


def check(got, ref, tol, what):
    off = np.abs(got - ref) - tol
    assert np.isfinite(got).all() and (off <= 0).all(), f"{what}: off by {np.abs(got - ref).max():.3e}, at {np.unravel_index(np.nanargmax(off), off.shape)}"


def arrays(B, C, T, dtype, gate, layer, seed=0):
    r = np.random.default_rng(seed)
    act = lambda: host(to(r.standard_normal((B, C, T)) + 0.5, dtype))  # noqa: E731
    vec = lambda mid: host(to(mid + 0.3 * r.standard_normal(C), "f32"))  # noqa: E731
    a = {n: act() for n in ("x", "f", "y", "dy", "dn")}
    a["gate"] = None if gate is None else host(to(r.random((B, C)), "f32")) if gate == "item" else host(to(r.random((B, C, T)), dtype))
    a["rscale"], a["post_weight"], a["next_weight"] = vec(0.5), vec(1.0), vec(1.0)
    a["post_bias"], a["next_bias"] = (vec(0.0), vec(0.0)) if layer else (None, None)
    return a


def on_device(a, dtype):
    return {n: to(x, dtype if n in ("x", "f", "y", "dy", "dn") or (n == "gate" and x is not None and x.ndim == 3) else "f32") for n, x in a.items()}


def poison(dev, lengths):
    for n in ("x", "f", "y", "dy", "dn", "gate"):
        if dev[n] is not None and dev[n].dim() == 3:
            for b, length in enumerate(lengths):
                dev[n][b, :, max(0, length):] = float("nan") if b % 2 else float("inf")


SHAPES = [(2, 256, 40), (1, 512, 77), (2, 768, 33), (1, 1024, 64), (1, 1000, 9), (3, 384, 8), (2, 640, 1), (1, 256, 5), (1, 7, 30), (1, 1, 1), (1, 1100, 21),
          (1, 896, 130), (2, 100, 3), (1, 130, 65)]


@pytest.mark.parametrize("layer", [False, True])
@pytest.mark.parametrize("gate", [None, "item", "element"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_both_passes(shape, dtype, gate, layer):
    import torch
    B, C, T = shape
    for lengths in (None, [T // 2 + 1] + [0] * (B > 1) + [T + 3] * (B > 2)):
        a = arrays(B, C, T, dtype, gate, layer)
        dev = on_device(a, dtype)
        kw = dict(layer=layer, lengths=None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda"))
        if lengths is not None:
            poison(dev, lengths)
        names = ("gate", "rscale", "post_weight", "post_bias", "next_weight", "next_bias")
        y, n = nm.nm_residual_norm_fwd(dev["x"], dev["f"], **{k: dev[k] for k in names}, **kw)
        store = lambda v: host(to(v, dtype))  # noqa: E731
        ref = {k: a[k] for k in names}
        ry, _ = orc.norm_fwd(a["x"], a["f"], post=True, layer=layer, lengths=lengths, **ref)
        slack = (C + 64) * 2.0 ** -24
        size = 1 + np.abs(ry).max()
        y = host(y)
        check(y, ry, STEP[dtype] * np.abs(ry) + slack * size, "y")
        _, rn = orc.norm_fwd(y, layer=layer, lengths=lengths, next_weight=a["next_weight"], next_bias=a["next_bias"])  # of the y that was stored
        check(host(n), rn, STEP[dtype] * np.abs(rn) + slack * (4 + np.abs(rn).max()) * (1 if C > 1 else 50), "n")
        assert store(y).shape == y.shape

        got = nm.nm_residual_norm_bwd(dev["dy"], dev["dn"], dev["y"], dev["f"], **{k: dev[k] for k in names}, **kw)
        ref.pop("next_bias")
        r = orc.norm_bwd(a["dy"], a["dn"], a["y"], a["f"], post=True, layer=layer, lengths=lengths, **ref)
        worst = slack * 30 * (1 if C > 6 else 1000)  # (a row of one channel is a constant: its norm's gradient is nothing but rounding)
        for name in ("dx", "df"):
            check(host(got[name]), r[name], STEP[dtype] * np.abs(r[name]) + worst * (1 + np.abs(r[name]).max()), name)
        if gate == "element":
            check(host(got["dgate"]), r["dgate_element"], STEP[dtype] * np.abs(r["dgate_element"]) + worst * (1 + np.abs(r["dgate_element"]).max()), "dgate")
        elif gate == "item":
            check(host(got["dgate"]), r["dgate_item"], (worst + (T + 8) * 2.0 ** -24) * (1 + r["abs_dgate_item"]), "dgate")
        else:
            assert got["dgate"] is None
        for name in ("drscale", "dpost_weight", "dpost_bias", "dnext_weight", "dnext_bias"):
            if name.endswith("bias") and not layer:
                assert got[name] is None
                continue
            check(host(got[name]), r[name], (worst + (B * T + 8) * 2.0 ** -24) * (1 + r["abs_" + name]), name)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", [(2, 256, 40), (1, 512, 3), (1, 1100, 9)], ids=str)
def test_parts_of_it(shape, dtype):
    """The norm in front of the first block; a block without a norm behind it; no weights; no next norm; no gradient of y."""
    B, C, T = shape
    a = arrays(B, C, T, dtype, None, False)
    d = on_device(a, dtype)
    slack = (C + 64) * 2.0 ** -24
    x, n = nm.nm_residual_norm_fwd(d["x"])
    _, rn = orc.norm_fwd(a["x"])
    assert x is d["x"]
    check(host(n), rn, STEP[dtype] * np.abs(rn) + slack * 8, "n")
    y, n = nm.nm_residual_norm_fwd(d["x"], d["f"], next_norm=False)
    assert n is None
    ry = a["x"] + a["f"]
    check(host(y), ry, STEP[dtype] * np.abs(ry) + slack * 8, "y")
    y, n = nm.nm_residual_norm_fwd(d["x"], d["f"], post_norm=True, layer=True)
    ry, _ = orc.norm_fwd(a["x"], a["f"], post=True, layer=True)
    check(host(y), ry, STEP[dtype] * np.abs(ry) + slack * 8, "y")
    got = nm.nm_residual_norm_bwd(None, d["dn"], d["y"])
    r = orc.norm_bwd(None, a["dn"], a["y"])
    check(host(got["dx"]), r["dx"], STEP[dtype] * np.abs(r["dx"]) + 30 * slack, "dx")
    assert got["df"] is None and got["dnext_weight"] is None
    got = nm.nm_residual_norm_bwd(d["dy"], None, None, d["f"], rscale=d["rscale"])
    r = orc.norm_bwd(a["dy"], None, None, a["f"], rscale=a["rscale"])
    assert (host(got["dx"]) == a["dy"]).all()
    check(host(got["df"]), r["df"], STEP[dtype] * np.abs(r["df"]) + slack, "df")
    check(host(got["drscale"]), r["drscale"], (slack + (B * T + 8) * 2.0 ** -24) * (1 + r["abs_drscale"]), "drscale")


def test_the_same_bits_every_time_and_in_a_graph():
    import torch
    a = arrays(4, 768, 203, "bf16", "item", True)
    d = on_device(a, "bf16")
    names = ("gate", "rscale", "post_weight", "post_bias", "next_weight", "next_bias")
    kw = {k: d[k] for k in names}
    run = lambda: nm.nm_residual_norm_bwd(d["dy"], d["dn"], d["y"], d["f"], layer=True, **kw)  # noqa: E731
    one = run()
    two = run()
    assert all(torch.equal(one[k], two[k]) for k in one)
    ws = torch.empty(nm.nm_residual_norm_bwd_workspace_bytes(4, 768, 203), dtype=torch.uint8, device="cuda")
    out = {k: torch.empty_like(v) for k, v in one.items()}
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        nm.nm_residual_norm_bwd(d["dy"], d["dn"], d["y"], d["f"], layer=True, out=out, workspace=ws, **kw)
    for _ in range(3):
        for v in out.values():
            v.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(one[k], out[k]) for k in one)
