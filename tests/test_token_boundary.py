"""CPU-only: the operators on tokens report every argument error before any device call."""
import ctypes
import types

import pytest

from paper_1909_09577_amd import binding as nm
from test_attn_decoder_boundary import A, BAD, UNS, WS

INF, NAN = float("inf"), float("nan")


def at(i, offset=0):
    return ctypes.c_void_p(A[i].value + offset)


def embed_fwd(B=2, V=50, C=64, U=9, ids=A[0], id_bytes=8, table=A[1], scale=1.0, len=None, out=A[2], dtype=0):
    return nm.lib().nm_embedding_fwd(B, V, C, U, ids, id_bytes, table, scale, len, out, dtype, None)


def embed_bwd(B=2, V=50, C=64, U=9, dout=A[0], ids=A[1], id_bytes=8, scale=1.0, len=None, dtable=A[2], flags=0, dtype=0, ws=None, ws_bytes=1 << 40):
    return nm.lib().nm_embedding_bwd(B, V, C, U, dout, ids, id_bytes, scale, len, dtable, flags, dtype, ws, ws_bytes, None)


@pytest.mark.parametrize("call", [embed_fwd, embed_bwd])
def test_embedding_geometry(call):
    for bad in (dict(B=0), dict(V=0), dict(C=0), dict(U=0), dict(U=-1), dict(id_bytes=2), dict(scale=NAN), dict(scale=INF), dict(dtype=2)):
        assert call(**bad) == BAD, bad
    for big in (dict(B=1 << 16, U=1 << 10, C=64), dict(V=1 << 26), dict(B=70000, U=1), dict(B=1, C=1, U=(1 << 31) - 5), dict(B=65535, C=64 * 129, U=2)):
        assert call(**big) == UNS, big


def test_embedding_pointers():
    for bad in (dict(ids=None), dict(table=None), dict(out=None), dict(out=A[1]), dict(out=A[0]), dict(out=at(1, 50 * 64 * 2 - 1)), dict(len=A[2])):
        assert embed_fwd(**bad) == BAD, bad
    for bad in (dict(ids=None), dict(dout=None), dict(dtable=None), dict(dtable=A[0]), dict(dtable=A[1]), dict(flags=1), dict(flags=8), dict(len=A[2])):
        assert embed_bwd(**bad) == BAD, bad
    need = nm.nm_embedding_bwd_workspace_bytes(2, 50, 64, 9)
    assert need >= 2 * 9 * 64 * 2 and need % 256 == 0 and nm.nm_embedding_bwd_workspace_bytes(0, 50, 64, 9) == 0
    for bad in (dict(), dict(ws=A[3], ws_bytes=need - 1), dict(ws=at(3, 64))):
        assert embed_bwd(**bad) == WS, bad


HEADS = dict(B=2, H=4, Hkv=2, D=64, U=9)


def heads_fwd(x=A[0], xs=None, qw=None, kw=None, eps=1e-5, freqs=A[1], rot=64, pos=None, len=None, out=A[2], os=None, flags=1, dtype=0, **dims):
    d = dict(HEADS, **dims)
    item = (d["H"] + d["Hkv"]) * d["D"] * d["U"]
    return nm.lib().nm_head_norm_fwd(*d.values(), x, item if xs is None else xs, qw, kw, eps, freqs, rot, pos, len, out, item if os is None else os,
                                     flags, dtype, None)


def heads_bwd(dout=A[3], ds=None, x=A[0], xs=None, qw=None, kw=None, eps=1e-5, freqs=A[1], rot=64, pos=None, len=None, dx=A[2], dxs=None, dqw=None,
              dkw=None, flags=1, dtype=0, ws=None, ws_bytes=1 << 40, **dims):
    d = dict(HEADS, **dims)
    item = (d["H"] + d["Hkv"]) * d["D"] * d["U"]
    s = [item if v is None else v for v in (ds, xs, dxs)]
    return nm.lib().nm_head_norm_bwd(*d.values(), dout, s[0], x, s[1], qw, kw, eps, freqs, rot, pos, len, dx, s[2], dqw, dkw, flags, dtype, ws, ws_bytes, None)


def heads_cache(x=A[0], xs=None, qw=None, kw=None, eps=1e-5, freqs=A[1], rot=64, pages=10, page=16, table=A[4], most=5, len=A[5], q_len=None, k=A[6],
                v=A[7], q=A[2], qs=None, flags=1, dtype=0, **dims):
    d = dict(HEADS, **dims)
    item, q_item = (d["H"] + 2 * d["Hkv"]) * d["D"] * d["U"], d["H"] * d["D"] * d["U"]
    return nm.lib().nm_head_norm_cache(*d.values(), x, item if xs is None else xs, qw, kw, eps, freqs, rot, pages, page, table, most, len, q_len, k, v, q,
                                       q_item if qs is None else qs, flags, dtype, None)


@pytest.mark.parametrize("call", [heads_fwd, heads_bwd, heads_cache])
def test_heads_geometry(call):
    for bad in (dict(B=0), dict(H=0), dict(Hkv=-1), dict(D=0), dict(U=0), dict(rot=66), dict(rot=3), dict(rot=-2), dict(rot=0), dict(freqs=None),
                dict(dtype=2), dict(flags=4), dict(eps=-1.0), dict(eps=NAN), dict(eps=INF), dict(flags=0, qw=A[8]), dict(flags=0, kw=A[8]), dict(xs=100),
                dict(xs=1 << 41), dict(x=None)):
        assert call(**bad) == BAD, bad
    for big in (dict(D=63, rot=2), dict(D=130), dict(U=1 << 26), dict(B=1 << 24, U=7), dict(B=1 << 26, U=16), dict(H=1 << 17, D=2, rot=2, U=1)):
        assert call(**big) == UNS, big


def test_heads_pointers():
    for bad in (dict(out=None), dict(out=A[0]), dict(out=at(0, 64)), dict(os=10), dict(Hkv=0, kw=A[8]), dict(out=A[8], qw=A[8]), dict(len=A[2]), dict(pos=A[2])):
        assert heads_fwd(**bad) == BAD, bad
    for bad in (dict(dx=None), dict(dout=None), dict(dx=A[3]), dict(dx=A[0]), dict(dxs=10), dict(ds=10), dict(dqw=A[8]), dict(dkw=A[8]),
                dict(qw=A[8], dqw=A[8]), dict(qw=A[8], dqw=A[2]), dict(qw=A[8], kw=A[9], dqw=A[10], dkw=A[10])):
        assert heads_bwd(**bad) == BAD, bad
    need = nm.nm_head_norm_bwd_workspace_bytes(*HEADS.values())
    assert need > 0 and need % 256 == 0 and nm.nm_head_norm_bwd_workspace_bytes(0, 4, 2, 64, 9) == 0
    for bad in (dict(), dict(ws=A[11], ws_bytes=need - 1), dict(ws=at(11, 16))):
        assert heads_bwd(qw=A[8], dqw=A[9], **bad) == WS, bad
    for bad in (dict(q=None), dict(k=None), dict(v=None), dict(table=None), dict(len=None), dict(pages=0), dict(most=0), dict(Hkv=0), dict(k=A[7]), dict(q=A[6]),
                dict(q=A[0]), dict(k=A[0]), dict(v=A[0]), dict(k=A[4]), dict(qs=10)):
        assert heads_cache(**bad) == BAD, bad
    for other in (dict(page=8), dict(page=48), dict(page=512), dict(page=0), dict(most=(1 << 30)), dict(pages=(1 << 31) - 1, page=256)):
        assert heads_cache(**other) == UNS, other


PAGED = dict(B=2, H=4, Hkv=2, D=64, U=9)


def paged(q=A[0], qs=None, k=A[1], v=A[2], pages=10, page=16, table=A[3], most=5, len=A[4], q_len=None, window=0, scale=0.125, o=A[5], os=None, lse=None,
          dtype=0, ws=A[6], ws_bytes=None, **dims):
    d = dict(PAGED, **dims)
    item = d["H"] * d["D"] * d["U"]
    need = nm.nm_paged_attn_workspace_bytes(*d.values(), page, most, dtype)
    return nm.lib().nm_paged_attn_fwd(*d.values(), q, item if qs is None else qs, k, v, pages, page, table, most, len, q_len, window, scale, o,
                                      item if os is None else os, lse, dtype, ws, need if ws_bytes is None else ws_bytes, None)


def test_paged_attention():
    for bad in (dict(B=0), dict(H=0), dict(Hkv=0), dict(H=3), dict(D=0), dict(U=0), dict(dtype=2), dict(page=0), dict(most=0), dict(pages=0), dict(window=-1),
                dict(scale=NAN), dict(scale=INF), dict(q=None), dict(k=None), dict(v=None), dict(table=None), dict(len=None), dict(o=None), dict(qs=10),
                dict(os=10), dict(os=1 << 41), dict(o=A[0]), dict(o=A[1]), dict(o=A[3]), dict(lse=A[5]), dict(lse=A[2]), dict(k=at(1, 8)), dict(v=at(2, 4))):
        assert paged(**bad) == BAD, bad
    for other in (dict(D=72), dict(D=144), dict(page=8), dict(page=48), dict(page=512), dict(most=1 << 28), dict(U=1 << 26), dict(B=1 << 25, U=1),
                  dict(pages=(1 << 31) - 1, page=256), dict(B=1 << 20, H=64, Hkv=8, U=8)):
        assert paged(**other) == UNS, other
    many = dict(B=1, H=1, Hkv=1, U=1, most=1000)
    need = nm.nm_paged_attn_workspace_bytes(1, 1, 1, 64, 1, 16, 1000)
    assert need > 0 and need % 256 == 0
    for bad in (dict(ws=None), dict(ws_bytes=need - 1), dict(ws=at(6, 32))):
        assert paged(**many, **bad) == WS, bad


def scores_fwd(B=2, V=50, U=9, scores=A[0], targets=A[1], size=8, len=None, top=3, logp=A[2], entropy=A[3], lse=A[4], ids=A[5], top_logp=A[6], dtype=0,
               ws=None, ws_bytes=0):
    return nm.lib().nm_token_scores_fwd(B, V, U, scores, targets, size, len, top, logp, entropy, lse, ids, top_logp, dtype, ws, ws_bytes, None)


def scores_bwd(B=2, V=50, U=9, scores=A[0], targets=A[1], size=8, len=None, lse=A[2], entropy=A[3], dlogp=A[4], dentropy=A[5], out=A[6], dtype=0, grad=0):
    return nm.lib().nm_token_scores_bwd(B, V, U, scores, targets, size, len, lse, entropy, dlogp, dentropy, out, dtype, grad, None)


@pytest.mark.parametrize("call", [scores_fwd, scores_bwd])
def test_scores_geometry(call):
    for bad in (dict(B=0), dict(V=0), dict(U=0), dict(dtype=2), dict(size=2), dict(scores=None), dict(targets=None)):
        assert call(**bad) == BAD, bad
    for big in (dict(V=1 << 27), dict(B=1 << 23, U=2, V=2), dict(B=1, U=1, V=(1 << 31) - 2), dict(B=1 << 24, U=1, V=20)):
        assert call(**big) == UNS, big


def test_scores_pointers():
    for bad in (dict(logp=None), dict(ids=None), dict(top_logp=None), dict(top=0), dict(top=-1), dict(top=51), dict(logp=A[0]), dict(lse=A[1]), dict(lse=A[3]),
                dict(ids=A[6]), dict(targets=None, logp=None, top=0, ids=None, top_logp=None, entropy=None, lse=None), dict(len=A[2])):
        assert scores_fwd(**bad) == BAD, bad
    assert scores_fwd(top=17) == UNS
    long = dict(B=1, V=100000, U=1)
    need = nm.nm_token_scores_workspace_bytes(1, 100000, 1, 3)
    assert need > 0 and need % 256 == 0 and nm.nm_token_scores_workspace_bytes(1, 100000, 1, 17) == 0
    for bad in (dict(), dict(ws=A[7], ws_bytes=need - 1), dict(ws=at(7, 16), ws_bytes=need)):
        assert scores_fwd(**long, **bad) == WS, bad
    for bad in (dict(lse=None), dict(out=None), dict(entropy=None), dict(dlogp=None), dict(targets=None, dlogp=None, dentropy=None), dict(grad=2), dict(out=A[0]),
                dict(out=A[2]), dict(out=A[4])):
        assert scores_bwd(**bad) == BAD, bad


def test_binding_refuses_what_it_can_see():
    torch = pytest.importorskip("torch")
    x, ids = torch.zeros(2, 8, 4), torch.zeros(2, 4, dtype=torch.int64)
    cache, table, n = torch.zeros(3, 1, 16, 2), torch.zeros(2, 1, dtype=torch.int32), torch.ones(2, dtype=torch.int32)
    for call in (lambda: nm.nm_embedding_fwd(ids, x[0]), lambda: nm.nm_embedding_bwd(x, ids, 5), lambda: nm.nm_head_norm_fwd(x, heads=3, kv_heads=1),
                 lambda: nm.nm_head_norm_bwd(x, x, heads=3, kv_heads=1), lambda: nm.nm_head_norm_cache(x, cache, cache, table, n, heads=2, kv_heads=1),
                 lambda: nm.nm_paged_attn_fwd(x, cache, cache, table, n, heads=4, kv_heads=1), lambda: nm.nm_token_scores_fwd(x, ids),
                 lambda: nm.nm_token_scores_bwd(x, ids, x, None, x)):
        with pytest.raises(ValueError, match="device tensor"):
            call()


def on(device):
    return types.SimpleNamespace(is_cuda=True, get_device=lambda: device, dim=lambda: 3)


def test_a_tensor_of_another_device_is_refused(monkeypatch):
    torch = pytest.importorskip("torch")
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    with pytest.raises(ValueError, match="current device"):
        nm.nm_token_scores_fwd(on(1))
    with pytest.raises(ValueError, match="current device"):
        nm.nm_paged_attn_fwd(on(1), None, None, None, None, heads=1, kv_heads=1)
