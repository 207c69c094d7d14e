"""CPU-only: cross attention, the norms around a block and the AdamW step report every argument error before any device call."""
import ctypes

import pytest

from paper_1909_09577_amd import binding as nm

A = [ctypes.c_void_p(0x700000000000 + i * 0x1000000000) for i in range(12)]  # never dereferenced
BAD, UNS, WS = nm.NM_ERR_BAD_ARG, nm.NM_ERR_UNSUPPORTED, nm.NM_ERR_WORKSPACE
DIMS = dict(B=2, H=4, Hkv=2, D=64, U=8, T=100)


def attn_fwd(q=A[0], k=A[1], v=A[2], o=A[3], lse=None, scale=0.125, dtype=0, ws=A[4], ws_bytes=None, strides=None, **dims):
    d = dict(DIMS, **dims)
    qi, ki = d["H"] * d["D"] * d["U"], d["Hkv"] * d["D"] * d["T"]
    sq, sk, sv, so = strides or (qi, ki, ki, qi)
    need = nm.nm_cross_attn_workspace_bytes(nm.NM_OP_ATTN_FWD, *d.values(), dtype)
    return nm.lib().nm_cross_attn_fwd(*d.values(), q, sq, k, sk, v, sv, None, None, None, scale, o, so, lse, dtype, ws,
                                      need if ws_bytes is None else ws_bytes, None)


def attn_bwd(ptrs=None, lse=A[8], scale=0.125, dtype=0, ws=A[9], ws_bytes=None, strides=None, **dims):
    d = dict(DIMS, **dims)
    qi, ki = d["H"] * d["D"] * d["U"], d["Hkv"] * d["D"] * d["T"]
    items = [qi, qi, ki, ki, qi, qi, ki, ki]  # dout q k v o dq dk dv
    p = dict(zip("gqkvo", A), dq=A[5], dk=A[6], dv=A[7])
    p.update(ptrs or {})
    s = dict(zip(p, items))
    s.update(strides or {})
    need = nm.nm_cross_attn_workspace_bytes(nm.NM_OP_ATTN_BWD, *d.values(), dtype)
    ins = [x for n in "gqkvo" for x in (p[n], s[n])]
    outs = [x for n in ("dq", "dk", "dv") for x in (p[n], s[n])]
    return nm.lib().nm_cross_attn_bwd(*d.values(), *ins, lse, None, None, None, scale, *outs, dtype, ws,
                                      need if ws_bytes is None else ws_bytes, None)


@pytest.mark.parametrize("call", [attn_fwd, attn_bwd])
def test_attention_geometry(call):
    for bad in (dict(B=0), dict(H=0), dict(Hkv=0), dict(D=0), dict(U=0), dict(T=0), dict(T=-1), dict(H=3), dict(Hkv=3)):
        assert call(**bad) == BAD, bad
    assert call(dtype=2) == BAD and call(dtype=-1) == BAD
    assert call(D=129) == UNS and call(T=1 << 30) == UNS and call(U=1 << 30) == UNS and call(B=1 << 30) == UNS
    assert call(scale=float("nan")) == BAD and call(scale=float("inf")) == BAD


def test_attention_pointers_strides_and_overlap():
    for n in ("q", "k", "v", "o"):
        assert attn_fwd(**{n: None}) == BAD, n
    for n in ("g", "q", "k", "v", "o", "dq", "dk", "dv"):
        assert attn_bwd({n: None}) == BAD, n
    assert attn_bwd(lse=None) == BAD
    qi, ki = 4 * 64 * 8, 2 * 64 * 100
    assert attn_fwd(strides=(qi - 1, ki, ki, qi)) == BAD and attn_fwd(strides=(qi, ki, ki - 1, qi)) == BAD
    assert attn_fwd(strides=(qi, 1 << 41, ki, qi)) == BAD
    assert attn_bwd(strides={"dk": ki - 1}) == BAD
    assert attn_fwd(o=A[0]) == BAD and attn_fwd(o=ctypes.c_void_p(A[1].value + 8)) == BAD and attn_fwd(lse=A[2]) == BAD
    assert attn_fwd(lse=A[3]) == BAD
    assert attn_bwd({"dq": A[1]}) == BAD and attn_bwd({"dk": A[6], "dv": A[6]}) == BAD and attn_bwd({"dv": A[8]}) == BAD
    # halves of one tensor: the items lie between each other's and do not overlap (the workspace is what is missing)
    half = ctypes.c_void_p(A[6].value + ki * 2)
    assert attn_bwd({"dv": half}, strides={"dk": 2 * ki, "dv": 2 * ki}, ws=None) == WS
    less = ctypes.c_void_p(A[6].value + ki * 2 - 2)
    assert attn_bwd({"dv": less}, strides={"dk": 2 * ki, "dv": 2 * ki}, ws=None) == BAD


def test_attention_workspace():
    need = nm.nm_cross_attn_workspace_bytes(nm.NM_OP_ATTN_BWD, *DIMS.values(), 0)
    assert need >= 2 * 4 * 8 * 4 and need % 256 == 0
    assert attn_bwd(ws=None) == WS and attn_bwd(ws_bytes=need - 1) == WS and attn_bwd(ws=ctypes.c_void_p(A[9].value + 16)) == WS
    long = dict(B=1, H=1, Hkv=1, T=10000)  # positions shared among workgroups
    need = nm.nm_cross_attn_workspace_bytes(nm.NM_OP_ATTN_FWD, *dict(DIMS, **long).values(), 0)
    assert need > 0 and need % 256 == 0
    assert attn_fwd(ws=None, **long) == WS and attn_fwd(ws_bytes=need - 1, **long) == WS
    assert nm.nm_cross_attn_workspace_bytes(99, *DIMS.values(), 0) == 0
    assert nm.nm_cross_attn_workspace_bytes(nm.NM_OP_ATTN_FWD, *dict(DIMS, D=0).values(), 0) == 0


POST, NEXT, LAYER = nm.NM_NORM_POST, nm.NM_NORM_NEXT, nm.NM_NORM_LAYER


def norm_fwd(B=2, C=64, T=16, x=A[0], f=A[1], gate=None, kind=0, rscale=None, pw=None, pb=None, nw=None, nb=None, eps=1e-5, y=A[2], n=A[3],
             flags=POST | NEXT, dtype=0):
    return nm.lib().nm_residual_norm_fwd(B, C, T, x, f, gate, kind, rscale, pw, pb, nw, nb, eps, None, y, n, flags, dtype, None)


def norm_bwd(B=2, C=64, T=16, dy=A[0], dn=A[1], y=A[2], f=A[3], gate=None, kind=0, rscale=None, pw=None, pb=None, nw=None, eps=1e-5, dx=A[4],
             df=A[5], dgate=None, drs=None, dpw=None, dpb=None, dnw=None, dnb=None, flags=POST | NEXT, dtype=0, ws=None, ws_bytes=0):
    return nm.lib().nm_residual_norm_bwd(B, C, T, dy, dn, y, f, gate, kind, rscale, pw, pb, nw, eps, None, dx, df, dgate, drs, dpw, dpb, dnw,
                                         dnb, flags, dtype, ws, ws_bytes, None)


@pytest.mark.parametrize("call", [norm_fwd, norm_bwd])
def test_norm_arguments(call):
    for bad in (dict(B=0), dict(C=0), dict(T=0), dict(C=-4), dict(dtype=3), dict(flags=8), dict(eps=-1.0), dict(eps=float("nan")),
                dict(eps=float("inf")), dict(kind=3), dict(kind=-1), dict(kind=1), dict(kind=2), dict(gate=A[6], kind=0)):
        assert call(**bad) == BAD, bad
    assert call(C=8193) == UNS and call(B=65001) == UNS and call(B=60000, C=8000, T=1000) == UNS
    assert call(pb=A[6]) == BAD                                                # a bias without LAYER
    assert call(flags=NEXT, pw=A[6]) == BAD                                     # a weight of a norm that is not there


def test_norm_pointers():
    for bad in (dict(x=None), dict(f=None), dict(y=None), dict(n=None), dict(flags=POST), dict(nb=A[6]), dict(y=A[0]), dict(y=A[1]), dict(n=A[0]),
                dict(n=A[2]), dict(f=None, y=None, flags=0, n=None), dict(f=None, y=None, flags=NEXT, rscale=A[6]),
                dict(gate=A[2], kind=2), dict(flags=POST, n=None, nw=A[6])):
        assert norm_fwd(**bad) == BAD, bad
    for bad in (dict(dx=None), dict(df=None), dict(f=None), dict(dn=None), dict(y=None), dict(dy=None, dn=None, flags=POST), dict(dx=A[0]), dict(df=A[4]),
                dict(dgate=A[6]), dict(dnb=A[6]), dict(dpb=A[6]), dict(flags=POST, dn=None, dnw=A[6]), dict(f=None, df=None, flags=NEXT, drs=A[6]),
                dict(gate=A[6], kind=2, dgate=A[6])):
        assert norm_bwd(**bad) == BAD, bad
    need = nm.nm_residual_norm_bwd_workspace_bytes(2, 64, 16)
    assert need > 0 and need % 256 == 0 and nm.nm_residual_norm_bwd_workspace_bytes(0, 64, 16) == 0
    for bad in (dict(ws=None), dict(ws=A[7], ws_bytes=need - 1), dict(ws=ctypes.c_void_p(A[7].value + 64), ws_bytes=need)):
        assert norm_bwd(dnw=A[6], **bad) == WS, bad


def tensor(**kw):
    t = dict(param=A[0].value, grad=A[1].value, m=A[2].value, v=A[3].value, m_scale=None, v_scale=None, copy=A[4].value, n=1000, weight_decay=0.1)
    t.update(kw)
    return nm.AdamWTensor(**t)


def plan_bytes(t, bits=32, count=1):
    return nm.lib().nm_adamw_plan_bytes(ctypes.byref(t) if t is not None else None, count, bits)


def test_adamw_plan_arguments():
    L = nm.lib()
    need = plan_bytes(tensor())
    assert need > 0 and need % 256 == 0 and plan_bytes(tensor(copy=None)) == need
    for bad in (dict(param=None), dict(grad=None), dict(m=None), dict(v=None), dict(n=0), dict(n=1 << 31), dict(weight_decay=-1.0),
                dict(weight_decay=float("nan")), dict(weight_decay=float("inf")), dict(m_scale=A[5].value, v_scale=A[6].value), dict(v=A[2].value),
                dict(param=A[1].value), dict(param=A[0].value + 2), dict(copy=A[4].value + 1), dict(m=A[2].value + 1)):
        assert plan_bytes(tensor(**bad)) == 0, bad
        assert L.nm_adamw_plan(ctypes.byref(tensor(**bad)), 1, 32, ctypes.create_string_buffer(4096), 4096) == BAD
    assert plan_bytes(None) == 0 and plan_bytes(tensor(), count=0) == 0 and plan_bytes(tensor(), bits=16) == 0
    assert plan_bytes(tensor(), bits=8) == 0
    eight = tensor(m_scale=A[5].value, v_scale=A[6].value, m=A[2].value + 1)
    assert plan_bytes(eight, bits=8) == need
    assert plan_bytes(tensor(m_scale=A[5].value, v_scale=A[5].value), bits=8) == 0
    buf = (ctypes.c_uint64 * 1024)()
    assert L.nm_adamw_plan(ctypes.byref(tensor()), 1, 32, ctypes.byref(buf), need - 1) == WS
    assert L.nm_adamw_plan(ctypes.byref(tensor()), 1, 32, None, need) == BAD


def test_adamw_step_arguments():
    L = nm.lib()
    t = tensor()
    need = plan_bytes(t)
    buf = (ctypes.c_uint64 * (need // 8))()
    assert L.nm_adamw_plan(ctypes.byref(t), 1, 32, ctypes.byref(buf), need) == nm.NM_OK

    def step(host=ctypes.byref(buf), device=A[5], size=need, lr=1e-3, b1=0.9, b2=0.99, eps=1e-8, n=1):
        return L.nm_adamw_step(host, device, size, lr, b1, b2, eps, n, None, 0, None)

    inf, nan = float("inf"), float("nan")
    for bad in (dict(host=None), dict(device=None), dict(device=ctypes.c_void_p(A[5].value + 64)), dict(size=need - 1), dict(size=16), dict(lr=inf),
                dict(lr=nan), dict(b1=1.0), dict(b1=-0.1), dict(b1=nan), dict(b2=1.0), dict(eps=0.0), dict(eps=nan), dict(eps=inf), dict(n=0)):
        assert step(**bad) == BAD, bad
    other = (ctypes.c_uint64 * (need // 8))()  # not a plan
    assert step(host=ctypes.byref(other)) == BAD


def test_binding_refuses_what_it_can_see():
    torch = pytest.importorskip("torch")
    x = torch.zeros(2, 4, 8)
    with pytest.raises(ValueError):
        nm.nm_residual_norm_fwd(x)
    with pytest.raises(ValueError):
        nm.nm_cross_attn_fwd(x, x, x, heads=2)
    with pytest.raises(nm.NmError):
        nm.nm_cross_attn_fwd(x, x, x, heads=3)
    with pytest.raises(ValueError):
        nm.nm_adamw_plan([x], [x], [x], [x], weight_decay=[0.0, 0.0])
