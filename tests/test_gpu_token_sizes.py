"""The calls on tokens at sizes whose offsets and launches do not fit 32 bits, against torch in float64 (of the largest ones on parts)."""
import math

import pytest

from paper_1909_09577_amd import binding as nm

pytestmark = pytest.mark.gpu
u_ = 2.0 ** -24


@pytest.mark.parametrize("top", [0, 1, 3])
def test_scores_of_as_many_classes_as_there_may_be(top):
    """All but the last ones are barred: the sum is their number, which float32 holds exactly, so what is left are the roundings of a logarithm
    and of the result (2 units of a number below 16 each)."""
    import torch
    V, n = 2 ** 31 - 2 ** 16 - 1, 8_000_000
    z = torch.full((1, V, 1), -math.inf, device="cuda", dtype=torch.bfloat16)
    z[0, V - n:] = 0.0
    target = torch.tensor([[V - 5]], device="cuda")
    of = nm.nm_token_scores_fwd(z, target, top=top)
    tol = 4 * 16 * u_
    for name, want in (("lse", math.log(n)), ("entropy", math.log(n)), ("logp", -math.log(n))):
        assert abs(of[name].item() - want) <= tol, name
    if top:
        assert of["top_ids"].flatten().tolist() == list(range(V - n, V - n + top))
        assert (of["top_logp"] + math.log(n)).abs().max().item() <= tol
        return
    g = nm.nm_token_scores_bwd(z, target, of["lse"], None, torch.ones(1, 1, device="cuda"))
    assert abs(g[0, V - 5, 0].item() - 1) <= 2.0 ** -8 and not g[0, :V - n].any()
    g[0, V - 5] = -1 / n
    assert (g[0, V - n:].float() * n + 1).abs().max().item() <= 2.0 ** -8 + 20 * u_


def test_scores_of_rows_whose_offsets_pass_32_bits():
    """Sixteen rows of 67 million places are more than 2^32 bytes.  Tolerance: 32 terms, exponents of at most 20 in powers of two, two units of each."""
    import torch
    V, U = 32, 67108832
    z = torch.randn(1, V, U, device="cuda")
    of = nm.nm_token_scores_fwd(z)
    for u0 in range(0, U, 1 << 22):
        part = z[0, :, u0:u0 + (1 << 22)].double()
        lse = torch.logsumexp(part, 0)
        assert (of["lse"][0, u0:u0 + (1 << 22)] - lse).abs().max().item() <= (V + 64) * u_ + 16 * 4 * u_, u0
        x = part - lse
        entropy = -(x.exp() * x).sum(0)
        assert (of["entropy"][0, u0:u0 + (1 << 22)] - entropy).abs().max().item() <= 3 * (V + 72) * u_ * 10, u0


def test_alternatives_of_more_places_than_a_launch_has_wavefronts():
    """72 million places: each place's join is a wavefront's."""
    import torch
    B, V, U, top = 1024, 29, 70000, 4
    z = torch.randn(B, V, U, device="cuda", dtype=torch.bfloat16)
    of = nm.nm_token_scores_fwd(z, top=top, out={"top_ids": torch.full((B, top, U), -7, dtype=torch.int32, device="cuda")})
    assert of["top_ids"].min().item() >= 0
    for b in (0, 500, 958, 959, B - 1):
        best, ids = z[b].float().sort(dim=0, descending=True, stable=True)
        lse = torch.logsumexp(z[b].double(), 0)
        assert torch.equal(of["top_ids"][b].long(), ids[:top]), b
        assert (of["lse"][b] - lse).abs().max().item() <= (V + 64) * u_ + 16 * 4 * u_, b
        assert (of["top_logp"][b] - (best[:top].double() - lse)).abs().max().item() <= (V + 64) * u_ + 16 * 8 * u_, b


def gradient_of(dout, ids, V):
    """The table's gradient from the places that have a token, in float64, and the sums of the terms' magnitudes and how often tokens occur."""
    import torch
    B, C, U = dout.shape
    b, u = (ids >= 0).nonzero(as_tuple=True)
    rows, to = dout.permute(0, 2, 1)[b, u].double(), ids[b, u]
    zeros = lambda: torch.zeros(V, C, dtype=torch.float64, device="cuda")  # noqa: E731
    return zeros().index_add_(0, to, rows), zeros().index_add_(0, to, rows.abs()), torch.bincount(to, minlength=V)


@pytest.mark.parametrize("dtype, B, U, C, V, share", [("bf16", 1024, 65600, 16, 29, 1e-4), ("f32", 65535, 2, 8192, 1000, 0.2)], ids=["runs", "tiles"])
def test_an_embedding_gradient_of_more_workgroups_than_a_launch_may_have(dtype, B, U, C, V, share):
    """More than 2^26 places' joins; more tiles to turn, ranges and rows to fill than 2^23.  A share of the places has a token.  Tolerance: a
    rounding for each term and the result."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(1)
    dout = torch.randn(B, C, U, device="cuda", generator=g, dtype=torch.bfloat16 if dtype == "bf16" else torch.float32)
    ids = torch.randint(0, V, (B, U), device="cuda", generator=g)
    ids[torch.rand(B, U, device="cuda", generator=g) > share] = -1
    ids[-1, -1], ids[0, 0], ids[-1, 0] = V - 1, 0, 3
    ids[B // 2] = torch.where(torch.arange(U, device="cuda") < 100, 7, ids[B // 2])
    got = nm.nm_embedding_bwd(dout, ids, V)
    ref, mag, count = gradient_of(dout, ids, V)
    assert ((got - ref).abs() <= (count + 2)[:, None] * u_ * mag).all()


def test_a_large_accumulated_embedding_gradient_keeps_the_other_rows():
    import torch
    B, U, C, V = 65535, 2, 8192, 400
    dout = torch.ones(B, C, U, device="cuda")
    ids = torch.full((B, U), -1, device="cuda")
    ids[5, 1], ids[-1, 0] = 17, 399
    dtable = torch.randn(V, C, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    want = dtable.clone()
    want[17] += 1
    want[399] += 1
    assert torch.equal(nm.nm_embedding_bwd(dout, ids, V, dtable=dtable, accumulate=True), want)
