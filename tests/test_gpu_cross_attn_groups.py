"""Cross attention where a workgroup's wavefronts take the same tokens of several heads, and where several workgroups share the positions
that a workgroup's tokens look at.  Tolerances are those of test_gpu_cross_attn.py."""
import numpy as np
import pytest

from test_gpu_cross_attn import run_and_check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", [(2, 4, 1, 64, 24, 70), (1, 8, 2, 128, 33, 65), (2, 4, 2, 80, 65, 40), (1, 6, 1, 64, 50, 100), (1, 3, 1, 64, 90, 33),
                                   (1, 8, 1, 96, 31, 130), (1, 16, 1, 32, 130, 9), (1, 4, 1, 64, 260, 5)], ids=str)
def test_heads_side_by_side(shape, dtype):
    B, _, _, _, U, T = shape
    run_and_check(*shape, dtype)
    run_and_check(*shape, dtype, lengths=[T // 2 + 1] * B, q_lengths=[U // 2 + 1] * B, poison=True)
    run_and_check(*shape, dtype, apart=True, seed=1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", [(1, 4, 1, 64, 40, 1500), (1, 2, 1, 128, 70, 1100), (1, 2, 2, 64, 150, 900), (1, 1, 1, 64, 3, 4000)], ids=str)
def test_windows_and_shared_positions(shape, dtype):
    B, _, _, _, U, T = shape
    at = np.arange(U) * (T / U)
    w = np.stack([at - T / 9, at + T / 9], 1).round().astype(np.int64)[None].repeat(B, 0)  # some begin below 0, some end behind T
    run_and_check(*shape, dtype, windows=w)
    w[:, U // 3:U // 2] = [[T, 0]]          # nothing, and the wrong way round
    run_and_check(*shape, dtype, windows=w, lengths=[T - T // 5], q_lengths=[U - U // 4])
    narrow = np.stack([at, at + 1], 1).astype(np.int64)[None].repeat(B, 0)  # one frame each
    run_and_check(*shape, dtype, windows=narrow)


def test_same_bits_every_time():
    """Sums of shared positions and tokens are joined in one order."""
    import torch
    from paper_1909_09577_amd import binding as nm
    g = torch.Generator(device="cuda").manual_seed(0)
    r = lambda *s: torch.randn(*s, device="cuda", generator=g).bfloat16()  # noqa: E731
    q, k, v, do = r(1, 8 * 64, 70), r(1, 2 * 64, 3001), r(1, 2 * 64, 3001), r(1, 8 * 64, 70)
    at = (torch.arange(70, device="cuda") * 42).int()
    kw = dict(heads=8, kv_heads=2, windows=torch.stack([at, at + 400], 1)[None].contiguous())
    first = None
    for _ in range(3):
        o, lse = nm.nm_cross_attn_fwd(q, k, v, want_lse=True, **kw)
        got = (o, lse, *nm.nm_cross_attn_bwd(do, q, k, v, o, lse, **kw))
        torch.cuda.synchronize()
        first = first or got
        assert all(torch.equal(a, b) for a, b in zip(got, first))
