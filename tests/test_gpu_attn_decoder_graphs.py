"""The attention decoder's calls on a stream of their own and replayed from a captured graph, every replay against the eager result."""
import pytest

pytestmark = pytest.mark.gpu


def replay_and_compare(calls, outputs, before_replay, expected):
    """Eager on another stream, then three replays with eager work between them."""
    import torch
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        calls()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outputs, expected))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for _ in range(3):
        before_replay()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outputs, expected))


@pytest.mark.parametrize("shape", [(2, 96, 50), (3, 640, 1), (1, 1100, 20)], ids=str)
def test_norms(shape):
    import torch
    from paper_1909_09577_amd import binding as nm
    B, C, T = shape
    g = torch.Generator(device="cuda").manual_seed(1)
    x, f, dy, dn = (torch.randn(B, C, T, device="cuda", generator=g).bfloat16() for _ in range(4))
    kw = {k: torch.rand(C, device="cuda", generator=g) + 0.5 for k in ("rscale", "post_weight", "post_bias", "next_weight", "next_bias")}
    kw.update(layer=True, gate=torch.rand(B, C, device="cuda", generator=g))
    y, n = nm.nm_residual_norm_fwd(x, f, **kw)
    want = nm.nm_residual_norm_bwd(dy, dn, y, f, **kw)
    names = [k for k in want if want[k] is not None]
    out = {k: torch.empty_like(want[k]) for k in names}
    y2, n2 = torch.empty_like(y), torch.empty_like(n)
    ws = torch.empty(nm.nm_residual_norm_bwd_workspace_bytes(B, C, T), dtype=torch.uint8, device="cuda")

    def calls():
        nm.nm_residual_norm_fwd(x, f, y=y2, n=n2, **kw)
        nm.nm_residual_norm_bwd(dy, dn, y2, f, out=out, workspace=ws, **kw)

    outputs = [y2, n2] + [out[k] for k in names]

    def wipe():
        for t in outputs:
            t.fill_(7)

    replay_and_compare(calls, outputs, wipe, [y, n] + [want[k] for k in names])


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw(bits):
    import torch
    from paper_1909_09577_amd import binding as nm
    g = torch.Generator(device="cuda").manual_seed(2)
    sizes = [5, 256, 4500]

    def make():
        p, grad = ([torch.randn(n, device="cuda", generator=g.manual_seed(n + i)) for n in sizes] for i in range(2))
        state = [[torch.zeros(n, device="cuda", dtype=torch.float32 if bits == 32 else torch.uint8) for n in sizes] for _ in range(2)]
        scales = [[torch.ones(-(-n // 256), device="cuda") for n in sizes] for _ in range(2)] if bits == 8 else [None, None]
        plan = nm.nm_adamw_plan(p, grad, *state, m_scales=scales[0], v_scales=scales[1], weight_decay=0.01)
        return p + state[0] + state[1] + (scales[0] + scales[1] if bits == 8 else []), plan

    want, plan = make()
    begin = [t.clone() for t in want]
    nm.nm_adamw_step(plan, lr=1e-3, step=1, seed=5)
    outputs, plan2 = make()

    def restore():
        for t, b in zip(outputs, begin):
            t.copy_(b)

    def calls():
        nm.nm_adamw_step(plan2, lr=1e-3, step=1, seed=5)

    replay_and_compare(calls, outputs, restore, want)


def test_a_stream_given_to_the_call():
    """Workspaces that a call makes for itself are not handed out again before the given stream is through with them."""
    import torch
    from paper_1909_09577_amd import binding as nm
    g = torch.Generator(device="cuda").manual_seed(3)
    r = lambda *s: torch.randn(*s, device="cuda", generator=g).bfloat16()  # noqa: E731
    q, k, v, do = r(1, 256, 40), r(1, 256, 2000), r(1, 256, 2000), r(1, 256, 40)
    o, lse = nm.nm_cross_attn_fwd(q, k, v, heads=4, want_lse=True)
    want = nm.nm_cross_attn_bwd(do, q, k, v, o, lse, heads=4)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    outs = [torch.empty_like(t) for t in want]
    torch.cuda.synchronize()
    for _ in range(3):
        nm.nm_cross_attn_bwd(do, q, k, v, o, lse, heads=4, dq=outs[0], dk=outs[1], dv=outs[2], stream=s)
        torch.full((4 << 20,), 7.0, device="cuda")  # takes the next free memory of the current stream
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))
