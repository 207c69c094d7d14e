"""The norms around a block on padded batches of rows that end in part of a group: every item's length lies within the last groups of
the row, so that the last group, which is read from where the row's last whole group begins, holds valid positions of the tile
before beside padding.  Tolerances are those of test_gpu_residual_norm.py."""
import numpy as np
import pytest

from oracle import attn_decoder_oracle as orc
from paper_1909_09577_amd import binding as nm
from test_gpu_residual_norm import STEP, arrays, check, host, on_device, poison

pytestmark = pytest.mark.gpu
VECTORS = ("rscale", "post_weight", "post_bias", "next_weight", "next_bias")
# channels, time, items, whether the whole rows are compared (else their ends); the last: several rounds of workgroups
CASES = [(256, 33, 10, True), (256, 65, 10, True), (768, 100, 10, True), (768, 129, 10, True), (300, 385, 10, False), (256, 801, 70, False)]


def make(C, T, B, dtype, gate, layer):
    import torch
    lengths = [T - 9 + b % 10 for b in range(B)]
    a = arrays(B, C, T, dtype, gate, layer)
    dev = on_device(a, dtype)
    poison(dev, lengths)
    return a, dev, lengths, torch.tensor(lengths, dtype=torch.int32, device="cuda")


def ends(a, lengths, T, whole):
    """(first position compared, the oracle's arguments from there on, the lengths there)."""
    at = 0 if whole else T - 40
    cut = {n: x[:, :, at:] if x is not None and x.ndim == 3 else x for n, x in a.items()}
    return at, cut, [n - at for n in lengths]


@pytest.mark.parametrize("gate,layer", [(None, False), ("element", True)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_forward(case, dtype, gate, layer):
    C, T, B, whole = case
    a, dev, lengths, ln = make(C, T, B, dtype, gate, layer)
    kw = {k: dev[k] for k in VECTORS + ("gate",)}
    at, cut, left = ends(a, lengths, T, whole)
    ry, _ = orc.norm_fwd(cut["x"], cut["f"], post=True, layer=layer, lengths=left, **{k: cut[k] for k in VECTORS + ("gate",)})
    slack, size = (C + 64) * 2.0 ** -24, 1 + np.abs(ry).max()
    for _ in range(3):
        y, n = nm.nm_residual_norm_fwd(dev["x"], dev["f"], layer=layer, lengths=ln, **kw)
        y = host(y)[:, :, at:]
        check(y, ry, STEP[dtype] * np.abs(ry) + slack * size, "y")
        _, rn = orc.norm_fwd(y, layer=layer, lengths=left, next_weight=a["next_weight"], next_bias=a["next_bias"])
        check(host(n)[:, :, at:], rn, STEP[dtype] * np.abs(rn) + slack * (4 + np.abs(rn).max()), "n")


@pytest.mark.parametrize("gate,layer", [(None, False), ("element", True), ("item", False)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_backward(case, dtype, gate, layer):
    C, T, B, whole = case
    a, dev, lengths, ln = make(C, T, B, dtype, gate, layer)
    kw = {k: dev[k] for k in VECTORS + ("gate",)}
    at, cut, left = ends(a, lengths, T, whole)
    names = ("rscale", "post_weight", "post_bias", "next_weight", "gate")
    r = orc.norm_bwd(cut["dy"], cut["dn"], cut["y"], cut["f"], post=True, layer=layer, lengths=left, **{k: cut[k] for k in names})
    worst = (C + 64) * 2.0 ** -24 * 30
    for _ in range(3):
        got = nm.nm_residual_norm_bwd(dev["dy"], dev["dn"], dev["y"], dev["f"], layer=layer, lengths=ln, **kw)
        for name, of in (("dx", "dx"), ("df", "df")) + ((("dgate", "dgate_element"),) if gate == "element" else ()):
            check(host(got[name])[:, :, at:], r[of], STEP[dtype] * np.abs(r[of]) + worst * (1 + np.abs(r[of]).max()), name)
        if not whole:
            continue
        if gate == "item":
            check(host(got["dgate"]), r["dgate_item"], (worst + (T + 8) * 2.0 ** -24) * (1 + r["abs_dgate_item"]), "dgate")
        for name in ("drscale", "dpost_weight", "dnext_weight") + (("dpost_bias", "dnext_bias") if layer else ()):
            check(host(got[name]), r[name], (worst + (B * T + 8) * 2.0 ** -24) * (1 + r["abs_" + name]), name)
