"""The calls on tokens on a stream of their own and replayed from a captured graph, every replay against the eager result; two calls
on two streams at once."""
import pytest

from test_gpu_attn_decoder_graphs import replay_and_compare

pytestmark = pytest.mark.gpu


def ints(values):
    import torch
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def normal(*shape, seed=1, dtype=None):
    import torch
    x = torch.randn(*shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed))
    return x.to(dtype or torch.bfloat16)


def wipe(outputs):
    def now():
        for t in outputs:
            t.fill_(7)
    return now


@pytest.mark.parametrize("B, U, V, C", [(3, 1, 50, 96), (5, 300, 700, 200)])
def test_embedding(B, U, V, C):
    import torch
    from paper_1909_09577_amd import binding as nm
    ids = torch.randint(0, V, (B, U), device="cuda", generator=torch.Generator(device="cuda").manual_seed(2))
    table, dout, lengths = normal(V, C), normal(B, C, U, seed=2), ints([U - b % 2 for b in range(B)])
    want = [nm.nm_embedding_fwd(ids, table, lengths=lengths), nm.nm_embedding_bwd(dout, ids, V, lengths=lengths)]
    outputs = [torch.empty_like(t) for t in want]
    ws = torch.empty(nm.nm_embedding_bwd_workspace_bytes(B, V, C, U), dtype=torch.uint8, device="cuda")

    def calls():
        nm.nm_embedding_fwd(ids, table, lengths=lengths, out=outputs[0])
        nm.nm_embedding_bwd(dout, ids, V, lengths=lengths, dtable=outputs[1], workspace=ws)

    replay_and_compare(calls, outputs, wipe(outputs), want)


@pytest.mark.parametrize("B, U", [(3, 1), (2, 150)])
def test_heads(B, U):
    import torch
    from paper_1909_09577_amd import binding as nm
    heads, kv_heads, D = 4, 2, 64
    x, dout = normal(B, 6 * D, U), normal(B, 6 * D, U, seed=2)
    kw = dict(heads=heads, kv_heads=kv_heads, q_weight=normal(D, dtype=torch.float32), k_weight=normal(D, seed=4, dtype=torch.float32),
              freqs=10000.0 ** (-torch.arange(0, D, 2, device="cuda", dtype=torch.float64) / D), lengths=ints([U - b % 2 for b in range(B)]))
    want = [nm.nm_head_norm_fwd(x, **kw), *nm.nm_head_norm_bwd(dout, x, **kw)]
    outputs = [torch.empty_like(t) for t in want]
    ws = torch.empty(nm.nm_head_norm_bwd_workspace_bytes(B, heads, kv_heads, D, U), dtype=torch.uint8, device="cuda")

    def calls():
        nm.nm_head_norm_fwd(x, out=outputs[0], **kw)
        nm.nm_head_norm_bwd(dout, x, dx=outputs[1], dq_weight=outputs[2], dk_weight=outputs[3], workspace=ws, **kw)

    replay_and_compare(calls, outputs, wipe(outputs), want)


@pytest.mark.parametrize("U", [1, 40])
def test_cache_and_its_attention(U):
    """Tokens go into the cache and are attended to by the next call; a replay writes what it reads."""
    import torch
    from paper_1909_09577_amd import binding as nm
    B, heads, kv_heads, D, page = 3, 4, 1, 64, 32
    x = normal(B, 6 * D, U)
    table = ints([[5, 1, 7, 2], [0, 8, 3, 11], [9, 4, 10, 6]])
    lengths, each = ints([100, U, 70]), ints([U, U, max(U - 3, 1)])
    turning = dict(heads=heads, kv_heads=kv_heads, freqs=10000.0 ** (-torch.arange(0, D, 2, device="cuda", dtype=torch.float64) / D), q_lengths=each)
    begin = normal(12, kv_heads, page, D, seed=3), normal(12, kv_heads, D, page, seed=4)

    def fresh():
        return [t.clone() for t in begin]

    k, v = fresh()
    q = nm.nm_head_norm_cache(x, k, v, table, lengths, **turning)
    o, lse = nm.nm_paged_attn_fwd(q, k, v, table, lengths, heads=heads, kv_heads=kv_heads, q_lengths=each, want_lse=True)
    want = [k, v, q, o, lse]
    outputs = fresh() + [torch.empty_like(t) for t in (q, o, lse)]
    ws = torch.empty(nm.nm_paged_attn_workspace_bytes(B, heads, kv_heads, D, U, page, table.shape[1]), dtype=torch.uint8, device="cuda")

    def calls():
        nm.nm_head_norm_cache(x, *outputs[:2], table, lengths, q=outputs[2], **turning)
        nm.nm_paged_attn_fwd(outputs[2], *outputs[:2], table, lengths, heads=heads, kv_heads=kv_heads, q_lengths=each, o=outputs[3], lse=outputs[4],
                             workspace=ws)

    def restore():
        wipe(outputs[2:])()
        for t, b in zip(outputs, begin):
            t.copy_(b)

    replay_and_compare(calls, outputs, restore, want)


@pytest.mark.parametrize("B, U, V, top", [(3, 1, 4000, 5), (4, 70, 1000, 0)])
def test_token_scores(B, U, V, top):
    import torch
    from paper_1909_09577_amd import binding as nm
    scores = normal(B, V, U)
    targets = torch.randint(0, V, (B, U), device="cuda", generator=torch.Generator(device="cuda").manual_seed(2))
    dlogp, dent, lengths = normal(B, U, dtype=torch.float32), normal(B, U, seed=5, dtype=torch.float32), ints([U - b % 2 for b in range(B)])
    of = nm.nm_token_scores_fwd(scores, targets, top=top, lengths=lengths)
    names = [n for n in of if of[n] is not None]
    want = [of[n] for n in names] + [nm.nm_token_scores_bwd(scores, targets, of["lse"], of["entropy"], dlogp, dent, lengths=lengths)]
    outputs = [torch.empty_like(t) for t in want]
    ws = torch.empty(nm.nm_token_scores_workspace_bytes(B, V, U, top), dtype=torch.uint8, device="cuda")
    out = dict(zip(names, outputs))

    def calls():
        nm.nm_token_scores_fwd(scores, targets, top=top, lengths=lengths, out=out, workspace=ws)
        nm.nm_token_scores_bwd(scores, targets, out["lse"], out["entropy"], dlogp, dent, lengths=lengths, dscores=outputs[-1])

    replay_and_compare(calls, outputs, wipe(outputs), want)


def test_calls_on_two_streams_at_once():
    """Each call takes a workspace of its own and leaves it to the allocator on its own stream."""
    import torch
    from paper_1909_09577_amd import binding as nm
    scores, ids = [normal(4, 3000, 20, seed=i) for i in range(2)], torch.randint(0, 90, (4, 20), device="cuda")
    dout = [normal(4, 128, 20, seed=i) for i in range(2)]
    want = [(nm.nm_token_scores_fwd(s, ids, top=3), nm.nm_embedding_bwd(d, ids, 90)) for s, d in zip(scores, dout)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(4):
        got = []
        for s, d, stream in zip(scores, dout, streams):
            stream.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(stream):
                got.append((nm.nm_token_scores_fwd(s, ids, top=3), nm.nm_embedding_bwd(d, ids, 90)))
        torch.cuda.synchronize()
        for (a, x), (b, y) in zip(got, want):
            assert torch.equal(x, y) and all(torch.equal(a[n], b[n]) for n in a if a[n] is not None)


def test_a_decoder_step_replayed():
    """Serving as a program does it: one captured step, whose token and filled cache the program moves on between replays."""
    import torch
    from paper_1909_09577_amd.attn_decoder import AttentionDecoder
    dec = AttentionDecoder(40, 128, 4, 2, 64, kv_heads=2, seed=1, positions="rotated")
    states, frames = normal(2, 64, 24), ints([24, 17])
    tokens = torch.randint(0, 40, (6, 2), device="cuda")
    run = dec.start(states, frames, 8, page=16)
    want = [dec.next(t, run).clone() for t in tokens]
    run = dec.start(states, frames, 8, page=16)
    token = tokens[0].clone()
    dec.next(token, run)  # the calls' first launches lie before the capture
    run["at"] = 0
    run["filled"].zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        logp = dec.next(token, run)
    for t, w in zip(tokens, want):
        token.copy_(t)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(logp, w)
