"""Cross attention on the GPU against the float64 oracle, over head layouts, lengths from one on, odd sizes, padded batches, windows
that leave a token nothing, and tensors whose items are apart.

Tolerances (derived, per element).  In bfloat16 mode p and ds are rounded once as operands and the result once (2^-8 each); the
rest is float32: a score is off by at most (D+4)*2^-24 of the sum of its terms' magnitudes, a probability by twice that (its own
score and the log-sum-exp) and a sum over n terms by n*2^-24 of their magnitudes."""
import numpy as np
import pytest

from oracle import attn_decoder_oracle as orc
from paper_1909_09577_amd import binding as nm

pytestmark = pytest.mark.gpu
STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


def to(a, dtype):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a, np.float32)).cuda().to(torch.bfloat16 if dtype == "bf16" else torch.float32)


def host(t):
    import torch
    torch.cuda.synchronize()
    return t.double().cpu().numpy()


def make(B, H, Hkv, D, U, T, dtype, seed=0, big=1.0):
    """float64 arrays of storable values."""
    r = np.random.default_rng(seed)
    arrays = {"q": big * r.standard_normal((B, H * D, U)), "k": r.standard_normal((B, Hkv * D, T)), "v": r.standard_normal((B, Hkv * D, T)),
              "do": r.standard_normal((B, H * D, U))}
    return {n: host(to(a, dtype)) for n, a in arrays.items()}


def float_error(a, p, scale, heads, kv_heads):
    """Relative error of a probability from float32 arithmetic, and of a sum over the states."""
    B, HD, U = a["q"].shape
    D, T = HD // heads, a["k"].shape[2]
    q = np.abs(a["q"]).reshape(B, heads, D, U)
    k = np.repeat(np.abs(np.where(np.isfinite(a["k"]), a["k"], 0)).reshape(B, kv_heads, D, T), heads // kv_heads, 1)
    score = np.where(p > 0, np.einsum("bhdu,bhdt->bhut", q, k), 0).max() * abs(scale) * (D + 4) * 2.0 ** -24
    return 2 * score + 8 * 2.0 ** -24, 2.0 ** -24


def check(got, ref, tol, what):
    got = np.asarray(got)
    assert np.isfinite(got).all(), f"{what}: not finite"
    off = np.abs(got - ref) - tol
    assert (off <= 0).all(), f"{what}: off by {np.abs(got - ref).max():.3e}, at most {tol.flat[off.argmax()]:.3e} there, at {np.unravel_index(off.argmax(), off.shape)}"


def run_and_check(B, H, Hkv, D, U, T, dtype, *, scale=None, lengths=None, q_lengths=None, windows=None, seed=0, big=1.0, poison=False, apart=False,
                  bwd=True):
    import torch
    a = make(B, H, Hkv, D, U, T, dtype, seed, big)
    sc = D ** -0.5 if scale is None else scale
    ok = orc.allowed(B, U, T, lengths, q_lengths, windows)
    dev = {n: to(x, dtype) for n, x in a.items()}
    if poison:  # what lies in the padding must not matter
        for b in range(B):
            if lengths is not None:
                dev["k"][b, :, max(0, lengths[b]):] = float("nan")
                dev["v"][b, :, max(0, lengths[b]):] = float("inf")
            if q_lengths is not None:
                for n in ("q", "do"):
                    dev[n][b, :, max(0, q_lengths[b]):] = float("nan")
    if apart:  # keys and values as halves of one tensor, queries and gradients as parts of wider ones
        kv = torch.cat([dev["k"], dev["v"]], 1)
        dev["k"], dev["v"] = kv[:, :Hkv * D], kv[:, Hkv * D:]
        wide = torch.cat([dev["q"], dev["do"], dev["do"]], 1)
        dev["q"], dev["do"] = wide[:, :H * D], wide[:, H * D:2 * H * D]
    as_int = lambda x: None if x is None else torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")  # noqa: E731
    kw = dict(heads=H, kv_heads=Hkv, scale=scale, lengths=as_int(lengths), q_lengths=as_int(q_lengths), windows=as_int(windows))
    o, lse = nm.nm_cross_attn_fwd(dev["q"], dev["k"], dev["v"], want_lse=True, **kw)
    ro, rlse, p, mag = orc.attn_fwd(a["q"], a["k"], a["v"], H, Hkv, sc, ok)
    prob, per = float_error(a, p, sc, H, Hkv)
    storage = STEP[dtype]
    rounded = STEP["bf16"] if dtype == "bf16" else 0.0
    check(host(o), ro, (rounded * (1 + storage) + prob + (T + 8) * per) * mag * (1 + storage) + storage * np.abs(ro) + 1e-37, "o")
    live = ok.any(2)[:, None].repeat(H, 1)
    got = host(lse)
    assert (got[~live] == -np.inf).all()
    check(got[live], rlse[live], (prob + (T + 8) * per + 2.0 ** -22 * np.abs(rlse) + 2.0 ** -22)[live], "lse")
    if not bwd:
        return
    saved = host(to(ro, dtype))
    lse_in = to(np.where(live, rlse, -np.inf), "f32")
    o_in = to(ro, dtype)
    if poison and q_lengths is not None:
        for b in range(B):
            o_in[b, :, max(0, q_lengths[b]):] = float("nan")
    dq, dk, dv = nm.nm_cross_attn_bwd(dev["do"], dev["q"], dev["k"], dev["v"], o_in, lse_in, **kw)
    rq, rk, rv, m = orc.attn_bwd(a["do"], a["q"], a["k"], a["v"], saved, p, H, Hkv, sc)
    n_u = U * (H // Hkv)
    lse_err = 2.0 ** -23 * (np.abs(rlse[live]).max() if live.any() else 0)
    f = prob + lse_err
    sums = (D + 8) * per
    check(host(dv), rv, (rounded + f + (n_u + 8) * per) * m["dv"] * (1 + storage) + storage * np.abs(rv) + 1e-37, "dv")
    check(host(dk), rk, (rounded * m["dk"] + (f + sums + (n_u + 8) * per) * m["dk_parts"]) * (1 + 2 * storage) + storage * np.abs(rk) + 1e-37, "dk")
    check(host(dq), rq, (rounded * m["dq"] + (f + sums + (T + 8) * per) * m["dq_parts"]) * (1 + 2 * storage) + storage * np.abs(rq) + 1e-37, "dq")


SHAPES = [  # B, H, Hkv, D, U, T
    (1, 1, 1, 64, 1, 1), (1, 2, 2, 64, 1, 5), (2, 4, 4, 64, 1, 64), (1, 4, 2, 64, 1, 600), (2, 8, 2, 64, 1, 333), (2, 4, 1, 128, 2, 97),
    (1, 2, 2, 32, 7, 31), (2, 2, 2, 64, 33, 65), (1, 2, 1, 64, 40, 130), (1, 1, 1, 96, 31, 200), (2, 3, 3, 80, 17, 77), (1, 2, 2, 128, 64, 129),
    (1, 2, 2, 64, 130, 70), (1, 1, 1, 64, 300, 40), (1, 1, 1, 128, 140, 100), (1, 2, 1, 48, 5, 8), (1, 1, 1, 1, 3, 9), (2, 2, 1, 5, 6, 2), (1, 1, 1, 100, 34, 7),
    (3, 2, 2, 16, 1, 3), (1, 2, 2, 24, 257, 4),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_whole_batches(shape, dtype):
    run_and_check(*shape, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape,lengths,q_lengths", [
    ((5, 2, 2, 64, 9, 70), [70, 0, 1, 33, 65], [9, 9, 1, 0, 5]),
    ((4, 4, 2, 64, 40, 131), [131, 128, 2, -3], [40, 33, 1, 400]),
    ((3, 2, 1, 128, 1, 100), [100, 64, 500], [1, 0, 1]),
    ((2, 1, 1, 40, 150, 37), [0, 36], [150, 129]),
    ((2, 8, 8, 80, 3, 1000), [999, 513], None),
], ids=str)
def test_padding_is_not_read(shape, lengths, q_lengths, dtype):
    run_and_check(*shape, dtype, lengths=lengths, q_lengths=q_lengths, poison=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", [(2, 2, 2, 64, 40, 150), (1, 4, 1, 128, 9, 333), (2, 2, 1, 96, 3, 70), (1, 1, 1, 64, 140, 200)], ids=str)
def test_windows_some_of_them_empty(shape, dtype):
    B, _, _, _, U, T = shape
    r = np.random.default_rng(3)
    lo = r.integers(-5, T, (B, U))
    w = np.stack([lo, lo + r.integers(-3, 40, (B, U))], 2)
    w[:, ::3] = [[T // 2, T // 2]]      # nothing
    w[0, 1] = [0, 2 ** 31 - 1]
    w[0, U - 1] = [-2 ** 31, T + 7]
    run_and_check(*shape, dtype, windows=w)
    run_and_check(*shape, dtype, windows=w, lengths=[T // 2 + 1] * B, q_lengths=[U - 1] * B, poison=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", [(3, 4, 2, 64, 11, 77), (2, 2, 2, 128, 50, 129), (2, 2, 2, 24, 1, 7)], ids=str)
def test_items_that_are_apart(shape, dtype):
    run_and_check(*shape, dtype, apart=True)


@pytest.mark.parametrize("scale", [0.0, -0.3, 1.0, 1e-3])
def test_scales(scale):
    run_and_check(1, 2, 2, 64, 20, 90, "bf16", scale=scale)
    run_and_check(1, 2, 2, 64, 35, 90, "f32", scale=scale)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_sharp_attention(dtype):
    """Scores of some hundreds: all but a few probabilities vanish, the running maximum moves."""
    run_and_check(1, 2, 2, 64, 33, 500, dtype, big=40.0)
    run_and_check(1, 2, 2, 64, 1, 500, dtype, big=40.0)


@pytest.mark.parametrize("U", [1, 40])
def test_workgroups_that_share_positions_and_those_that_do_not_agree(U):
    """Many positions of one item are shared among workgroups; of many items they are not."""
    run_and_check(1, 1, 1, 64, U, 4100, "bf16")
    run_and_check(1, 1, 1, 128, U, 2050, "f32")


def test_outputs_in_given_tensors_on_another_stream_and_in_a_graph():
    import torch
    B, H, D, U, T = 2, 2, 64, 10, 700
    a = make(B, H, H, D, U, T, "bf16")
    dev = {n: to(x, "bf16") for n, x in a.items()}
    o1, l1 = nm.nm_cross_attn_fwd(dev["q"], dev["k"], dev["v"], heads=H, want_lse=True)
    g1 = nm.nm_cross_attn_bwd(dev["do"], dev["q"], dev["k"], dev["v"], o1, l1, heads=H)
    wide = torch.full((B, 3 * H * D, U), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.empty_like(l1)
    outs = [torch.empty_like(t) for t in g1]
    ws = torch.empty(max(nm.nm_cross_attn_workspace_bytes(op, B, H, H, D, U, T) for op in (nm.NM_OP_ATTN_FWD, nm.NM_OP_ATTN_BWD)),
                     dtype=torch.uint8, device="cuda")

    def both():
        nm.nm_cross_attn_fwd(dev["q"], dev["k"], dev["v"], heads=H, o=wide[:, H * D:2 * H * D], lse=lse, workspace=ws)
        nm.nm_cross_attn_bwd(dev["do"], dev["q"], dev["k"], dev["v"], wide[:, H * D:2 * H * D], lse, heads=H, dq=outs[0], dk=outs[1], dv=outs[2], workspace=ws)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        both()
    torch.cuda.synchronize()

    def same():
        torch.cuda.synchronize()
        assert torch.equal(wide[:, H * D:2 * H * D], o1) and torch.equal(lse, l1) and all(torch.equal(x, y) for x, y in zip(outs, g1))
        assert (wide[:, :H * D] == 7).all() and (wide[:, 2 * H * D:] == 7).all()

    same()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for _ in range(3):
        for t in (*outs, lse):
            t.zero_()
        graph.replay()
        same()
