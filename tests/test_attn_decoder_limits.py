"""CPU-only: calls that would need more work items than a launch may have (2^32) are refused before any device call."""
import ctypes

import pytest

from paper_1909_09577_amd import binding as nm
from test_attn_decoder_boundary import A, BAD, UNS, WS, attn_bwd, attn_fwd, norm_fwd, tensor


@pytest.mark.parametrize("dtype", [nm.NM_BF16, nm.NM_F32])
def test_attention(dtype):
    many = dict(B=1 << 19, H=16, Hkv=16, D=1, U=1, T=1)
    assert attn_fwd(dtype=dtype, **many) == UNS and attn_bwd(dtype=dtype, **many) == UNS
    for op in (nm.NM_OP_ATTN_FWD, nm.NM_OP_ATTN_BWD):
        assert nm.nm_cross_attn_workspace_bytes(op, *many.values(), dtype) == 0
    for fewer in (dict(many, B=(1 << 19) - 1), dict(many, Hkv=8)):  # (the workspace is what is missing)
        assert attn_bwd(dtype=dtype, ws=None, **fewer) == WS
        assert attn_fwd(dtype=dtype, o=A[0], **fewer) == BAD


def test_norms():
    for kw in (dict(B=2, C=1, T=1 << 29), dict(B=1, C=7, T=(1 << 28) + 1), dict(B=2, C=15, T=(1 << 26) + 1, dtype=nm.NM_F32),
               dict(B=1, C=1, T=1 << 30, dtype=nm.NM_F32)):
        assert norm_fwd(y=A[0], **kw) == UNS, kw
    for kw in (dict(B=1, C=7, T=(1 << 28) - 512), dict(B=2, C=15, T=(1 << 26) - 256, dtype=nm.NM_F32),
               dict(B=1, C=15, T=(1 << 27) + 1, dtype=nm.NM_F32), dict(B=60000, C=1000, T=33)):
        assert norm_fwd(y=A[0], **kw) == BAD, kw  # (y over x)


def test_adamw():
    def plan_bytes(count, n):
        table = (nm.AdamWTensor * count)(*(tensor(n=n) for _ in range(count)))
        return nm.lib().nm_adamw_plan_bytes(ctypes.byref(table[0]), count, 32)

    n = (1 << 31) - 4096  # 2^19 - 1 runs
    assert plan_bytes(32, n) > 0 and plan_bytes(33, n) == 0
