"""Attention over a paged cache on the GPU against the float64 oracle.

Tolerances (derived, per element).  A score is off by (D+4)*2^-24 of the sum of its terms' magnitudes and its product with the scale and log2(e)
by 2^-23 of itself, a probability by twice that (its own score and the sum) and eight roundings, a sum over n places by n*2^-24 of their
magnitudes.  In bfloat16 mode probabilities enter the second product in two terms (off by 2^-16) where 32 columns or fewer are left, else in one
(2^-8); the result is rounded once to the storage type."""
import numpy as np
import pytest

from oracle import token_oracle as orc
from paper_1909_09577_amd import binding as nm
from test_gpu_cross_attn import STEP, check, host, to
from test_gpu_head_norm import ints

pytestmark = pytest.mark.gpu


def run_and_check(B, H, Hkv, D, U, dtype, page, lengths, *, q_lengths=None, window=0, scale=None, table=None, max_pages=None, spare=2, seed=0, big=1.0,
                  poison=True, apart=False):
    import torch
    r = np.random.default_rng(seed)
    most = max(1, -(-max(max(lengths), 1) // page)) if max_pages is None else max_pages
    if table is None:
        table = r.permutation(B * most + spare)[:B * most].reshape(B, most)
    pages = int(max(B * most, table.max() + 1)) + spare if max_pages is None else B * most + spare
    q, k, v = (host(to(r.standard_normal(s) * m, dtype)) for s, m in (((B, H * D, U), big), ((pages, Hkv, page, D), 1.0), ((pages, Hkv, D, page), 1.0)))
    sc = D ** -0.5 if scale is None else scale
    o, lse, mag, terms = orc.paged_attn(q, k, v, table, lengths, H, Hkv, sc, q_lengths=q_lengths, window=window)
    if poison:  # rows that no token looks at
        used = np.zeros((pages, page), bool)
        for b in range(B):
            n, first = orc.new_tokens(lengths, q_lengths, b, U)
            for u in range(n):
                for p in range(max(0, first + u + 1 - window) if window else 0, first + u + 1):
                    at = orc.row_of(table, b, p, page, pages)
                    if at:
                        used[at] = True
        k[~used[:, None].repeat(Hkv, 1)] = np.nan
        v.transpose(0, 1, 3, 2)[~used[:, None].repeat(Hkv, 1)] = np.inf
        for b in range(B):
            q[b, :, orc.new_tokens(lengths, q_lengths, b, U)[0]:] = np.nan
    print(f"case {B} {H} {Hkv} {D} {U} {dtype} page {page} {lengths} {q_lengths} window {window}", flush=True)
    dq = to(q, dtype)
    out = None
    if apart:
        wide = torch.full((B, H * D + 48, U), float("nan"), device="cuda", dtype=dq.dtype)
        wide[:, :H * D] = dq
        dq, out = wide[:, :H * D], torch.empty((B, H * D + 16, U), device="cuda", dtype=dq.dtype)[:, :H * D]
    got, got_lse = nm.nm_paged_attn_fwd(dq, to(k, dtype), to(v, dtype), ints(table), ints(lengths), heads=H, kv_heads=Hkv, q_lengths=ints(q_lengths),
                                        window=window, scale=scale, o=out, want_lse=True)
    n = np.maximum(1, np.max(lengths) if len(lengths) else 1)
    score = terms * (D + 4) * 2.0 ** -24 + terms * 2.0 ** -23
    p_off = 2 * score + 8 * 2.0 ** -24 + (0 if dtype == "f32" else 2.0 ** -16 if H // Hkv * U <= 32 else 2.0 ** -8)
    tol = STEP[dtype] * np.abs(o) + (np.repeat(p_off, D, 1).reshape(B, H, D, U) if False else p_off[:, :, None].repeat(D, 2)).reshape(o.shape) * mag \
        + n * 2.0 ** -24 * mag
    check(host(got), o, tol, "o")
    got_lse = host(got_lse)
    empty = np.isneginf(lse)
    assert np.array_equal(np.isneginf(got_lse), empty)
    check(np.where(empty, 0, got_lse), np.where(empty, 0, lse), np.where(empty, 1, score + (n + 8) * 2.0 ** -24 + np.abs(np.where(empty, 0, lse)) * 2.0 ** -22), "lse")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [16, 32, 48, 64, 80, 96, 112, 128])
def test_widths(D, dtype):
    run_and_check(2, 4, 2, D, 1, dtype, 32, [70, 33])
    run_and_check(1, 4, 1, D, 9, dtype, 64, [200])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("heads", [(1, 1), (4, 1), (6, 3), (20, 1)], ids=str)
def test_pages_and_heads(heads, page, dtype):
    run_and_check(3, *heads, 64, 1, dtype, page, [1, page, 2 * page + 17])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("U", [2, 5, 8, 17, 40, 70, 150])
def test_chunks(U, dtype):
    run_and_check(2, 4, 2, 64, U, dtype, 16, [U, U + 83])
    run_and_check(1, 2, 2, 128, U, dtype, 64, [U + 301])


@pytest.mark.parametrize("U", [1, 6, 60])
@pytest.mark.parametrize("window", [1, 31, 32, 100])
def test_windows(U, window):
    run_and_check(2, 4, 2, 64, U, "bf16", 16, [U + 200, U], window=window)
    run_and_check(1, 2, 1, 48, U, "f32", 32, [U + 90], window=window)


@pytest.mark.parametrize("U", [4, 50])
def test_ragged_and_empty(U):
    run_and_check(5, 4, 2, 64, U, "bf16", 32, [100, 0, U, 3, -5], q_lengths=[1, U, 0, U, 2])
    run_and_check(3, 4, 4, 64, U, "f32", 16, [64, 2, 90], q_lengths=[-1, 100, 2])


def test_a_long_sequence_is_shared_among_workgroups():
    run_and_check(1, 4, 2, 64, 1, "bf16", 64, [3000])
    run_and_check(2, 2, 1, 128, 3, "bf16", 128, [2500, 1])
    run_and_check(1, 2, 2, 64, 2, "f32", 16, [1500])
    run_and_check(1, 2, 1, 80, 40, "bf16", 64, [2100])


@pytest.mark.parametrize("scale", [0.0, -0.3, 4.0])
def test_scales(scale):
    run_and_check(2, 4, 2, 64, 3, "bf16", 32, [50, 20], scale=scale)
    run_and_check(2, 4, 2, 64, 40, "f32", 32, [50, 60], scale=scale)


def test_large_scores():
    run_and_check(2, 4, 2, 64, 5, "bf16", 32, [150, 75], big=30.0)


@pytest.mark.parametrize("U", [1, 40])
def test_pages_that_are_not_there(U):
    """Their places are as masked; the table's end too."""
    run_and_check(2, 4, 2, 64, U, "bf16", 16, [100, 130], table=np.array([[0, -1, 3, 10 ** 6, 5, 6, 1], [7, 8, -2 ** 31, 2 ** 31 - 1, 9, 10, 11]]), max_pages=7)
    run_and_check(1, 2, 1, 64, U, "f32", 32, [70], table=np.array([[-1, -1, -1]]), max_pages=3)
    run_and_check(1, 2, 1, 64, U, "bf16", 64, [64 * 5], table=np.array([[-1, 0, 1]]), max_pages=3)


def test_sequences_that_share_pages():
    run_and_check(3, 4, 2, 64, 1, "bf16", 16, [40, 45, 33], table=np.array([[0, 1, 2], [0, 1, 3], [0, 1, 4]]))


def test_items_apart():
    run_and_check(3, 4, 2, 64, 7, "bf16", 16, [40, 45, 33], apart=True)
    run_and_check(3, 4, 2, 64, 37, "bf16", 16, [40, 45, 37], apart=True)


def test_offsets_beyond_32_bits():
    """The last pages of a cache of 5 GiB a tensor: byte offsets, and element offsets beyond 2^31, in 64 bits."""
    import torch
    page, D, H = 256, 128, 2
    pages = (5 << 30) // (page * D * 2)
    k = torch.empty(pages, 1, page, D, device="cuda", dtype=torch.bfloat16)
    v = torch.empty(pages, 1, D, page, device="cuda", dtype=torch.bfloat16)
    table = torch.tensor([[pages - 1, 0, pages - 2]], dtype=torch.int32, device="cuda")
    small = torch.tensor([[2, 0, 1]], dtype=torch.int32, device="cuda")
    ks, vs = (torch.randn(3, *t.shape[1:], device="cuda", generator=torch.Generator(device="cuda").manual_seed(i)).bfloat16() for i, t in enumerate((k, v)))
    for to_page, from_page in zip(table[0].tolist(), small[0].tolist()):
        k[to_page], v[to_page] = ks[from_page], vs[from_page]
    x = torch.randn(1, (H + 2) * D, 3, device="cuda").bfloat16()
    n = ints([700])
    for U in (3, 1):
        xs = x[:, :, :U].contiguous()
        q = nm.nm_head_norm_cache(xs, k, v, table, n, heads=H, kv_heads=1)
        q2 = nm.nm_head_norm_cache(xs, ks, vs, small, n, heads=H, kv_heads=1)
        o, _ = nm.nm_paged_attn_fwd(q, k, v, table, n, heads=H, kv_heads=1)
        o2, _ = nm.nm_paged_attn_fwd(q2, ks, vs, small, n, heads=H, kv_heads=1)
        torch.cuda.synchronize()
        assert torch.equal(o, o2) and torch.isfinite(o.float()).all()
    many = q.repeat(1, 1, 40).contiguous()
    a, _ = nm.nm_paged_attn_fwd(many, k, v, table, n, heads=H, kv_heads=1)
    b, _ = nm.nm_paged_attn_fwd(many, ks, vs, small, n, heads=H, kv_heads=1)
    assert torch.equal(a, b) and torch.isfinite(a.float()).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lengths", [[400, 37, 0], [1100, 33, 20], [70, 64, 40]], ids=str)
@pytest.mark.parametrize("U", [16, 33])
def test_joins_of_few_and_many_shares(U, lengths, dtype):
    run_and_check(3, 4, 2, 48, U, dtype, 32, lengths)
    run_and_check(3, 4, 1, 128, U, dtype, 16, lengths, q_lengths=[U, U - 1, 1])


@pytest.mark.parametrize("U", [1, 40])
def test_a_window_longer_than_anything(U):
    import torch
    g = torch.Generator(device="cuda").manual_seed(4)
    q, k, v = (torch.randn(*s, device="cuda", generator=g).bfloat16() for s in ((2, 4 * 32, U), (9, 2, 16, 32), (9, 2, 32, 16)))
    table, lengths = ints([[0, 3, 5, 7], [8, 1, 2, 4]]), ints([60, U // 2])
    want, got = (nm.nm_paged_attn_fwd(q, k, v, table, lengths, heads=4, kv_heads=2, window=w, want_lse=True) for w in (0, 2 ** 31 - 1))
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])
