"""Embedding lookup and its gradient on the GPU against the float64 oracle.

Tolerances (derived, per element).  A looked-up value is a product rounded to float32 and to the storage type.  A gradient is a sum of n
float32 terms that the library adds in any grouping, times the scale: n + 2 roundings of 2^-24 of the sum of their magnitudes."""
import numpy as np
import pytest

from oracle import token_oracle as orc
from paper_1909_09577_amd import binding as nm
from test_gpu_cross_attn import STEP, check, host, to

pytestmark = pytest.mark.gpu


def lengths_on(device, lengths):
    import torch
    return None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device=device)


def run_and_check(B, V, C, U, dtype, *, lengths=None, wide=True, tokens="any", scale=1.7, seed=0, accumulate=False):
    import torch
    r = np.random.default_rng(seed)
    ids = {"any": lambda: r.integers(0, V, (B, U)), "one": lambda: np.full((B, U), V - 1),
           "outside": lambda: r.integers(-2, V + 2, (B, U)), "few": lambda: r.integers(0, max(1, V // 50), (B, U)) * 7 % V, "low": lambda: r.integers(0, 3, (B, U))}[tokens]()
    table, dout = (host(to(r.standard_normal(s), dtype)) for s in ((V, C), (B, C, U)))
    dev_ids = torch.from_numpy(ids).cuda().to(torch.int64 if wide else torch.int32)
    ln = lengths_on("cuda", lengths)
    print(f"case {B} {V} {C} {U} {dtype} {tokens} {lengths}", flush=True)
    got = nm.nm_embedding_fwd(dev_ids, to(table, dtype), scale=scale, lengths=ln)
    ref = orc.embedding_fwd(ids, table, scale, lengths)
    check(host(got), ref, (STEP[dtype] + 2.0 ** -23) * np.abs(ref), "out")

    g = to(dout, dtype)
    if lengths is not None:  # what lies in the padding must not matter
        for b, n in enumerate(lengths):
            g[b, :, max(0, n):] = float("nan")
    old = r.standard_normal((V, C)).astype(np.float32)
    dtable = torch.from_numpy(old).cuda() if accumulate else torch.full((V, C), float("nan"), device="cuda")
    got = nm.nm_embedding_bwd(g, dev_ids, V, scale=scale, lengths=ln, dtable=dtable, accumulate=accumulate)
    assert got is dtable
    ref, mag, count = orc.embedding_bwd(dout, ids, V, scale, lengths)
    tol = (count + 2)[:, None] * 2.0 ** -24 * mag
    if accumulate:
        ref = ref + old
        tol = tol + 2.0 ** -24 * np.abs(ref)
        assert np.array_equal(host(got)[count == 0], old.astype(np.float64)[count == 0])
    check(host(got), ref, tol, "dtable")
    again = nm.nm_embedding_bwd(g, dev_ids, V, scale=scale, lengths=ln)
    assert accumulate or torch.equal(again, got)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", [(1, 1, 1, 1), (3, 29, 256, 1), (2, 29, 100, 5), (2, 300, 65, 15), (2, 40, 64, 16), (3, 700, 130, 77), (1, 9000, 24, 200),
                                   (2, 50, 513, 70), (1, 7, 3, 129), (5, 33, 8, 3)], ids=str)
def test_shapes(shape, dtype):
    run_and_check(*shape, dtype)


@pytest.mark.parametrize("tokens", ["one", "outside", "few"])
@pytest.mark.parametrize("wide", [True, False])
def test_tokens(tokens, wide):
    run_and_check(3, 400, 96, 90, "bf16", tokens=tokens, wide=wide)
    run_and_check(4, 57, 40, 2, "f32", tokens=tokens, wide=wide)


@pytest.mark.parametrize("lengths", [[90, 0, 1], [200, -3, 64], [65, 63, 90]], ids=str)
def test_lengths(lengths):
    run_and_check(3, 60, 72, 90, "bf16", lengths=lengths)
    run_and_check(3, 60, 72, 7, "bf16", lengths=lengths)


@pytest.mark.parametrize("tokens", ["any", "one", "few"])
def test_accumulation(tokens):
    run_and_check(2, 200, 520, 100, "bf16", tokens=tokens, accumulate=True)


@pytest.mark.parametrize("tokens", ["any", "one", "few"])
def test_more_places_than_a_sorting_workgroup_has_at_a_time(tokens):
    run_and_check(3, 5000, 8, 8100, "bf16", tokens=tokens, lengths=[8100, 8000, 4097])


@pytest.mark.parametrize("V", [600, 20000])
def test_more_places_of_some_tokens_than_a_list_holds(V):
    run_and_check(3, V, 8, 5000, "bf16", tokens="low", lengths=[5000, 4999, 3])


def test_infinities_and_nan_stay_with_their_token():
    import torch
    ids = torch.tensor([[0, 1, 2, 1]], device="cuda")
    table = torch.tensor([[1.0] * 8, [float("inf")] * 8, [float("nan")] * 8], device="cuda")
    out = nm.nm_embedding_fwd(ids, table)
    assert torch.equal(out[0, :, 0], table[0]) and torch.equal(out[0, :, 3], table[1]) and out[0, :, 2].isnan().all()
    dout = out.clone()
    got = nm.nm_embedding_bwd(dout, ids, 4)
    assert (got[0] == 1).all() and (got[1] == float("inf")).all() and got[2].isnan().all() and (got[3] == 0).all()
