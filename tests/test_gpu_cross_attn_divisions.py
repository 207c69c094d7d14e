"""Cross attention where the work is divided otherwise: more tiles of tokens than the backward pass keeps windows of, and an item whose
positions and tokens several workgroups share when it comes alone, but not in a large batch.  Tolerances are those of
test_gpu_cross_attn.py; two results of one item differ by at most two of them."""
import numpy as np
import pytest

from oracle import attn_decoder_oracle as orc
from paper_1909_09577_amd import binding as nm
from test_gpu_cross_attn import STEP, check, float_error, host, make, run_and_check, to

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape,dtype", [((1, 1, 1, 64, 16500, 150), "bf16"), ((1, 1, 1, 128, 8300, 140), "bf16"), ((1, 1, 1, 32, 8300, 260), "f32"),
                                         ((1, 2, 1, 16, 16450, 40), "bf16")], ids=str)
def test_windows_of_many_tokens(shape, dtype):
    _, _, _, _, U, T = shape
    at = np.arange(U) * (T / U)
    w = np.stack([at - 9, at + 9], 1).round().astype(np.int64)[None]
    w[:, U - 100:U - 50] = [[3, 3]]       # nothing, in the last tiles
    w[:, U - 50:U - 40] = [[0, T]]
    run_and_check(*shape, dtype, windows=w)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,H,Hkv,D,U,T", [(100, 8, 8, 64, 40, 700), (150, 8, 4, 64, 3, 4000), (60, 4, 2, 128, 70, 500)], ids=str)
def test_an_item_alone_and_in_a_large_batch(B, H, Hkv, D, U, T, dtype):
    import torch
    code = nm.NM_BF16 if dtype == "bf16" else nm.NM_F32
    dims = (H, Hkv, D, U, T, code)
    for op in (nm.NM_OP_ATTN_FWD, nm.NM_OP_ATTN_BWD):  # (what shares take of the workspace does not grow with the batch)
        assert nm.nm_cross_attn_workspace_bytes(op, B, *dims) < B * nm.nm_cross_attn_workspace_bytes(op, 1, *dims)
    a = make(1, H, Hkv, D, U, T, dtype)
    g = torch.Generator(device="cuda").manual_seed(1)
    one = {n: to(x, dtype) for n, x in a.items()}
    many = {n: torch.cat([torch.randn(B - 1, *t.shape[1:], device="cuda", generator=g).to(t.dtype), t]) for n, t in one.items()}
    kw, got = dict(heads=H, kv_heads=Hkv), []
    for x in (one, many):
        o, lse = nm.nm_cross_attn_fwd(x["q"], x["k"], x["v"], want_lse=True, **kw)
        if x is many:  # the backward passes of the same saved outputs
            o2, lse2 = o.clone(), lse.clone()
            o2[-1], lse2[-1] = got[0][0][0], got[0][1][0]
        else:
            o2, lse2 = o, lse
        got.append([t[-1:] for t in (o, lse, *nm.nm_cross_attn_bwd(x["do"], x["q"], x["k"], x["v"], o2, lse2, **kw))])
    alone, inside = ([host(t) for t in ts] for ts in got)
    sc = D ** -0.5
    ro, rlse, p, mag = orc.attn_fwd(a["q"], a["k"], a["v"], H, Hkv, sc, orc.allowed(1, U, T))
    prob, per = float_error(a, p, sc, H, Hkv)
    storage, rounded = STEP[dtype], STEP["bf16"] if dtype == "bf16" else 0.0
    rq, rk, rv, m = orc.attn_bwd(a["do"], a["q"], a["k"], a["v"], alone[0], p, H, Hkv, sc)
    f, sums, n_u = prob + 2.0 ** -23 * np.abs(rlse).max() + prob + (T + 8) * per + 2.0 ** -22, (D + 8) * per, U * (H // Hkv)
    tol = [(rounded * (1 + storage) + prob + (T + 8) * per) * mag * (1 + storage) + storage * np.abs(ro) + 1e-37,
           prob + (T + 8) * per + 2.0 ** -22 * np.abs(rlse) + 2.0 ** -22,
           (rounded * m["dq"] + (f + sums + (T + 8) * per) * m["dq_parts"]) * (1 + 2 * storage) + storage * np.abs(rq) + 1e-37,
           (rounded * m["dk"] + (f + sums + (n_u + 8) * per) * m["dk_parts"]) * (1 + 2 * storage) + storage * np.abs(rk) + 1e-37,
           (rounded + f + (n_u + 8) * per) * m["dv"] * (1 + storage) + storage * np.abs(rv) + 1e-37]
    for what, x, y, t, ref in zip(("o", "lse", "dq", "dk", "dv"), alone, inside, tol, (ro, rlse, rq, rk, rv)):
        check(x, ref, t, what + " alone")
        check(y, ref, t, what + " in a batch")
        check(x, y, 2 * t, what)
