"""Heads' norms over more tiles of tokens than there are workgroups side by side in the backward pass, with heads that two to four wavefronts share:
what they exchange for one tile must not meet the next one's.  Reference: torch in float64; tolerances as those of the tests of its sizes, a
sum over n tokens and heads with n more roundings."""
import pytest

from paper_1909_09577_amd import binding as nm
from test_gpu_cross_attn import STEP

pytestmark = pytest.mark.gpu


def turn(x, angle):
    import torch
    h = angle.shape[-2]
    a, b, rest = x[:, :, :h], x[:, :, h:2 * h], x[:, :, 2 * h:]
    return torch.cat([a * angle.cos() - b * angle.sin(), b * angle.cos() + a * angle.sin(), rest], 2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D, H, Hkv", [(64, 3, 2), (80, 2, 1), (128, 5, 1)])
def test_more_tiles_than_workgroups(D, H, Hkv, dtype):
    import torch
    B, U, rot, eps = 7, 32 * 300 + 5, D - 16, 1e-5
    g = torch.Generator(device="cuda").manual_seed(D)
    make = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    x, dout = (2 * make(B, (H + Hkv) * D, U)).to(dt), make(B, (H + Hkv) * D, U).to(dt)
    qw, kw = 1 + 0.3 * make(D), 1 + 0.3 * make(D)
    freqs = 10000.0 ** (-torch.arange(0, rot, 2, device="cuda", dtype=torch.float64) / rot)
    lengths = torch.tensor([U, U - 40, 0, 1, U, U - 9001, 333], dtype=torch.int32, device="cuda")
    kwargs = dict(heads=H, kv_heads=Hkv, q_weight=qw, k_weight=kw, freqs=freqs, lengths=lengths, eps=eps)
    out = nm.nm_head_norm_fwd(x, **kwargs)
    dx, dqw, dkw = nm.nm_head_norm_bwd(dout, x, **kwargs)
    assert all(torch.equal(a, b) for a, b in zip((dx, dqw, dkw), nm.nm_head_norm_bwd(dout, x, **kwargs)))

    w = torch.cat([qw.expand(H, D), kw.expand(Hkv, D)]).double()[None, :, :, None]
    angle = freqs[:, None] * torch.arange(U, device="cuda", dtype=torch.float64)
    dws, mags = torch.zeros(H + Hkv, D, dtype=torch.float64, device="cuda"), torch.zeros(H + Hkv, D, dtype=torch.float64, device="cuda")
    u, size = 2.0 ** -24, STEP[dtype]
    for b in range(B):
        ok = torch.arange(U, device="cuda") < lengths[b]
        z, d = (t[b:b + 1].double().view(1, H + Hkv, D, U) * ok for t in (x, dout))
        r = 1 / (z.square().mean(2, keepdim=True) + eps).sqrt()
        n = z * r
        m = torch.cat([(n * w)[:, :, :rot // 2].abs() + (n * w)[:, :, rot // 2:rot].abs()] * 2 + [(n * w)[:, :, rot:].abs()], 2)
        y = turn(n * w, angle)
        assert ((out[b].double().view_as(y[0]) - y[0]).abs() <= size * y[0].abs() + (D + 16) * u * m[0]).all(), b
        dn = turn(d, -angle)
        md = torch.cat([d[:, :, :rot // 2].abs() + d[:, :, rot // 2:rot].abs()] * 2 + [d[:, :, rot:].abs()], 2)
        ref = r * (w * dn - n * (w * dn * n).mean(2, keepdim=True)) * ok
        mag = r * (w.abs() * md + n.abs() * (w.abs() * md * n.abs()).mean(2, keepdim=True))
        assert ((dx[b].double().view_as(ref[0]) - ref[0]).abs() <= size * ref[0].abs() + (3 * D + 48) * u * mag[0]).all(), b
        dws += (dn * n).sum((0, 3))
        mags += (md * n.abs()).sum((0, 3))
    for got, heads in ((dqw, slice(0, H)), (dkw, slice(H, H + Hkv))):
        count = (heads.stop - heads.start) * B * U
        assert ((got - dws[heads].sum(0)).abs() <= (D + 32 + count) * u * mags[heads].sum(0)).all()
