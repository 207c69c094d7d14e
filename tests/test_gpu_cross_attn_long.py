"""Cross attention over so many states that byte offsets pass 32 bits, from one item to the next and within a tensor.

Tolerances (derived): p and the result are rounded once to bfloat16 (2^-8 each).  A sum over T states goes over at most 64 workgroups of
eight wavefronts with a matrix instruction per 16 states, so fewer than T/8192 + 600 additions follow one another; scores are sums of 128 terms
in float32 (132 * 2^-24 of the sum of their magnitudes, below 2^-13 here)."""
import pytest

pytestmark = pytest.mark.gpu


def test_offsets_beyond_32_bits():
    import torch
    from paper_1909_09577_amd import binding as nm
    B, H, Hkv, D, U, T = 2, 2, 2, 128, 3, (1 << 22) + 37
    g = torch.Generator(device="cuda").manual_seed(0)
    kv = torch.empty(B, 2 * Hkv * D, T, dtype=torch.bfloat16, device="cuda")
    for b in range(B):
        for c in range(0, 2 * Hkv * D, 64):
            kv[b, c:c + 64] = torch.randn(64, T, device="cuda", generator=g)
    k, v = kv[:, :Hkv * D], kv[:, Hkv * D:]
    assert kv.stride(0) * 2 > 1 << 32 and Hkv * D * T < 1 << 31
    q, do = (torch.randn(B, H * D, U, device="cuda", generator=g).bfloat16() for _ in range(2))
    lengths = torch.tensor([T, T - 5], dtype=torch.int32, device="cuda")
    kw = dict(heads=H, kv_heads=Hkv, lengths=lengths)
    o, lse = nm.nm_cross_attn_fwd(q, k, v, want_lse=True, **kw)
    dq, dk, dv = nm.nm_cross_attn_bwd(do, q, k, v, o, lse, **kw)
    torch.cuda.synchronize()
    adds = (T / 8192 + 600) * 2.0 ** -24 + 2.0 ** -12
    r = 2.0 ** -8
    for b in range(B):
        n = int(lengths[b])
        assert not dk[b, :, n:].any() and not dv[b, :, n:].any()
        for h in range(H):
            rows = slice(h * D, (h + 1) * D)
            kh, vh = k[b, rows, :n].float(), v[b, rows, :n].float()
            for u in range(U):
                s = (kh * q[b, rows, u].float()[:, None]).sum(0).double() * D ** -0.5
                ref = torch.logsumexp(s, 0)
                assert abs(lse[b, h, u] - ref) <= 2.0 ** -12 + 2.0 ** -22 * abs(ref)
                p = torch.exp(s - ref)
                want = torch.stack([(vh[d].double() * p).sum() for d in range(D)])
                size = torch.stack([(vh[d].abs().double() * p).sum() for d in range(D)])
                assert ((o[b, rows, u].double() - want).abs() <= (r + adds) * size * (1 + r) + r * want.abs()).all()
                if u == 0:
                    dp = (vh * do[b, rows, 0].float()[:, None]).sum(0).double()
                    ds = p * (dp - (o[b, rows, 0].double() * do[b, rows, 0].double()).sum())
                    want = torch.stack([(kh[d].double() * ds).sum() for d in range(D)]) * D ** -0.5
                    size = torch.stack([(kh[d].abs().double() * ds.abs()).sum() for d in range(D)]) * D ** -0.5
                    assert ((dq[b, rows, 0].double() - want).abs() <= adds * 4 * size + r * want.abs()).all()
            # the last frames' gradients: sums over three tokens
            end = slice(n - 64, n)
            ke, ve = k[b, rows, end].double(), v[b, rows, end].double()
            qh, doh, oh = (x[b, rows].double() for x in (q, do, o))
            p = torch.exp((qh.T.contiguous() @ ke) * D ** -0.5 - lse[b, h].double()[:, None])
            ds = p * (doh.T.contiguous() @ ve - (doh * oh).sum(0)[:, None])
            want_v, size_v = doh @ p, doh.abs() @ p
            want_k, size_k = qh @ ds * D ** -0.5, qh.abs() @ (p * (doh.abs().T.contiguous() @ ve.abs() + (doh * oh).abs().sum(0)[:, None])) * D ** -0.5
            assert ((dv[b, rows, end].double() - want_v).abs() <= (r + adds) * size_v * (1 + r) + r * want_v.abs() + 1e-37).all()
            assert ((dk[b, rows, end].double() - want_k).abs() <= adds * 4 * size_k * (1 + r) + r * want_k.abs() + 1e-37).all()
