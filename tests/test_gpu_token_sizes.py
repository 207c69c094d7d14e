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
