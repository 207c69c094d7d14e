"""The norms' backward pass without an eps: what is not part of the sums (padding, a norm that is not there) is no zero times infinity.
Tolerances are those of test_gpu_residual_norm.py."""
import numpy as np
import pytest

from oracle import attn_decoder_oracle as orc
from paper_1909_09577_amd import binding as nm
from test_gpu_residual_norm import STEP, arrays, check, host, on_device, poison

pytestmark = pytest.mark.gpu
SHAPES = [(2, 256, 40), (2, 768, 33), (1, 384, 100), (1, 1100, 9)]


def compare(got, r, dtype, B, C, T, vectors):
    worst = (C + 64) * 2.0 ** -24 * 30
    for name in ("dx", "df"):
        check(host(got[name]), r[name], STEP[dtype] * np.abs(r[name]) + worst * (1 + np.abs(r[name]).max()), name)
    for name in vectors:
        check(host(got[name]), r[name], (worst + (B * T + 8) * 2.0 ** -24) * (1 + r["abs_" + name]), name)


@pytest.mark.parametrize("layer", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_padding(shape, dtype, layer):
    import torch
    B, C, T = shape
    lengths = [T // 2 + 1, T - 3][:B]
    a = arrays(B, C, T, dtype, "element", layer)
    dev = on_device(a, dtype)
    poison(dev, lengths)
    names = ("gate", "rscale", "post_weight", "post_bias", "next_weight")
    got = nm.nm_residual_norm_bwd(dev["dy"], dev["dn"], dev["y"], dev["f"], layer=layer, eps=0.0, next_bias=dev["next_bias"],
                                  lengths=torch.tensor(lengths, dtype=torch.int32, device="cuda"), **{k: dev[k] for k in names})
    r = orc.norm_bwd(a["dy"], a["dn"], a["y"], a["f"], post=True, layer=layer, eps=0.0, lengths=lengths, **{k: a[k] for k in names})
    compare(got, r, dtype, B, C, T, ("drscale", "dpost_weight", "dnext_weight") + (("dpost_bias", "dnext_bias") if layer else ()))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_no_next_norm(shape, dtype):
    B, C, T = shape
    a = arrays(B, C, T, dtype, None, False)
    dev = on_device(a, dtype)
    got = nm.nm_residual_norm_bwd(dev["dy"], None, None, dev["f"], rscale=dev["rscale"], post_weight=dev["post_weight"], eps=0.0)
    r = orc.norm_bwd(a["dy"], None, None, a["f"], rscale=a["rscale"], post=True, post_weight=a["post_weight"], eps=0.0)
    assert (host(got["dx"]) == a["dy"]).all()
    compare(got, r, dtype, B, C, T, ("drscale", "dpost_weight"))
    got = nm.nm_residual_norm_bwd(dev["dy"], None, None, dev["f"], rscale=dev["rscale"], eps=0.0)
    r = orc.norm_bwd(a["dy"], None, None, a["f"], rscale=a["rscale"], eps=0.0)
    compare(got, r, dtype, B, C, T, ("drscale",))
