"""Attention over a paged cache in bfloat16: as exact for many columns (new tokens times the heads that share keys) as for few, and the same
bits every time.

Tolerances (derived, per element): those of the tests of its sizes, with probabilities that enter the second product in two bfloat16 terms whatever
the number of columns: the first is off by half a step (2^-8), the second by half a step of that, 2^-16 of the probability in all.  The result
is rounded once."""
import numpy as np
import pytest

from oracle import token_oracle as orc
from paper_1909_09577_amd import binding as nm
from test_gpu_cross_attn import STEP, check, host, to
from test_gpu_head_norm import ints

pytestmark = pytest.mark.gpu


def inputs(B, H, Hkv, D, U, page, lengths, seed=0):
    r = np.random.default_rng(seed)
    most = -(-max(lengths) // page)
    table = r.permutation(B * most)[:B * most].reshape(B, most)
    q, k, v = (host(to(r.standard_normal(s), "bf16")) for s in ((B, H * D, U), (B * most, Hkv, page, D), (B * most, Hkv, D, page)))
    return q, k, v, table


@pytest.mark.parametrize("D", [16, 48, 64, 112, 128])
@pytest.mark.parametrize("heads, U, lengths, window", [((4, 1), 9, [300, 41], 0), ((2, 2), 33, [33, 400], 0), ((4, 2), 150, [150, 161], 0),
                                                     ((4, 2), 70, [200, 70], 50), ((8, 1), 40, [1900, 900], 0)], ids=str)
def test_many_columns(heads, U, lengths, window, D):
    q, k, v, table = inputs(2, *heads, D, U, 64, lengths)
    print(f"case {heads} {D} {U} {lengths} window {window}", flush=True)
    o, lse, mag, terms = orc.paged_attn(q, k, v, table, lengths, *heads, D ** -0.5, window=window)
    got, got_lse = nm.nm_paged_attn_fwd(*(to(x, "bf16") for x in (q, k, v)), ints(table), ints(lengths), heads=heads[0], kv_heads=heads[1], window=window,
                                        want_lse=True)
    score, n = terms * (D + 4) * 2.0 ** -24 + terms * 2.0 ** -23, max(lengths)
    p_off = 2 * score + 8 * 2.0 ** -24 + 2.0 ** -16
    check(host(got), o, STEP["bf16"] * np.abs(o) + (p_off[:, :, None].repeat(D, 2).reshape(o.shape) + n * 2.0 ** -24) * mag, "o")
    check(host(got_lse), lse, score + (n + 8) * 2.0 ** -24 + np.abs(lse) * 2.0 ** -22, "lse")


def test_the_same_bits_every_time():
    import torch
    lengths = [700, 40, 233]
    q, k, v, table = inputs(3, 8, 2, 128, 40, 64, lengths, seed=1)
    args = [to(x, "bf16") for x in (q, k, v)] + [ints(table), ints(lengths)]
    calls = [nm.nm_paged_attn_fwd(*args, heads=8, kv_heads=2, want_lse=True) for _ in range(4)]
    torch.cuda.synchronize()
    assert all(torch.equal(calls[0][i], c[i]) for c in calls for i in (0, 1))
