"""The attention decoder with rotated queries and keys: the calls on tokens together, as a model uses them.  Gradients of a whole step
against float64 differentiation of the same model, decoding from the paged cache (token by token and in ragged chunks) against the
teacher-forced pass.

Tolerances (derived, float32 storage): as those of the decoder with added positions, whose chain of some thirty calls this one has with
two more a layer: 36 * 100 * 2^-24 of the largest element, taken five times for the gains of the norms."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
TOL = 1.2e-3


def make(layer_norm=False, seed=3, **kw):
    import torch
    from paper_1909_09577_amd.attn_decoder import AttentionDecoder
    dec = AttentionDecoder(13, 64, 4, 2, 48, kv_heads=2, hidden=80, layer_norm=layer_norm, seed=seed, positions="rotated", **kw)
    g = torch.Generator(device="cuda").manual_seed(seed)
    for n in dec.vectors:  # no parameter at its special starting value
        dec.master[n].add_(0.2 * torch.randn(dec.master[n].shape, device="cuda", generator=g))
    return dec


def batch(dec, B=3, U=9, T=21, seed=0):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    tokens, targets = (torch.randint(0, dec.vocab, (B, U), device="cuda", generator=g) for _ in range(2))
    states = torch.randn(B, 48, T, device="cuda", generator=g).to(dec.dtype)
    n = torch.tensor([U, 1, U - 3], dtype=torch.int32, device="cuda")
    frames = torch.tensor([T - 4, T, 1], dtype=torch.int32, device="cuda")
    return tokens, targets, states, n, frames


def reference(dec, tokens, targets, states, n, frames):
    """Loss and gradients in float64 on the host, item by item on its valid tokens and states."""
    import torch
    P = {k: v.double().cpu().requires_grad_() for k, v in dec.master.items()}
    states = states.double().cpu().requires_grad_()
    H, G, D = dec.heads, dec.heads // dec.kv_heads, dec.dim
    freqs = dec.freqs.cpu()

    def norm(x, name):
        z = x - x.mean(0, keepdim=True) if dec.layer_norm else x
        z = z / (z.square().mean(0, keepdim=True) + 1e-5).sqrt() * P[name][:, None]
        return z + P[name + "_bias"][:, None] if dec.layer_norm else z

    def turn(x, weight):  # [heads*D, u]
        x = x.reshape(-1, D, x.shape[1])
        x = x / (x.square().mean(1, keepdim=True) + 1e-5).sqrt() * weight[:, None]
        angle = freqs[:, None] * torch.arange(x.shape[2], dtype=torch.float64)
        a, b = x[:, :D // 2], x[:, D // 2:]
        return torch.cat([a * angle.cos() - b * angle.sin(), b * angle.cos() + a * angle.sin()], 1).reshape(-1, x.shape[2])

    def attend(q, k, v, causal):
        out = []
        for h in range(H):
            s = (q[h * D:(h + 1) * D].T @ k[h // G * D:(h // G + 1) * D]) * D ** -0.5
            if causal:
                s = s.masked_fill(torch.ones_like(s).triu(1) > 0, -torch.inf)
            out.append(v[h // G * D:(h // G + 1) * D] @ torch.softmax(s, 1).T)
        return torch.cat(out)

    total, count = 0.0, int(n.sum())
    C, kv = dec.channels, dec.kv_heads * D
    for b in range(tokens.shape[0]):
        u, t = int(n[b]), int(frames[b])
        mat = lambda name: P[name][:, :, 0]  # noqa: E731
        h = P["table"][tokens[b, :u].cpu()].T * C ** 0.5
        x = norm(h, "0.self.next")
        for l in range(dec.layers):
            for block in ("self", "cross", "ffn"):
                if block == "self":
                    p = mat(f"{l}.self.in") @ x
                    f = attend(turn(p[:C], P[f"{l}.self.q_norm"]), turn(p[C:C + kv], P[f"{l}.self.k_norm"]), p[C + kv:], True)
                elif block == "cross":
                    p = mat(f"{l}.cross.states") @ states[b, :, :t]
                    f = attend(mat(f"{l}.cross.in") @ x, p[:kv], p[kv:], False)
                else:
                    f = torch.relu(mat(f"{l}.ffn.in") @ x)
                h = h + P[f"{l}.{block}.scale"][:, None] * norm(mat(f"{l}.{block}.out") @ f, f"{l}.{block}.post")
                x = norm(h, dec._norm_names(l, block))
        logp = torch.log_softmax(mat("classes") @ x + P["classes_bias"][:, None], 0)
        total = total - logp[targets[b, :u].cpu(), torch.arange(u)].sum() / count
    total.backward()
    return total.item(), {k: p.grad.numpy() for k, p in P.items()}, states.grad.numpy()


@pytest.mark.parametrize("layer_norm", [False, True])
def test_a_step_against_differentiation(layer_norm):
    import torch
    dec = make(layer_norm, dtype="f32", state_bits=32)
    tokens, targets, states, n, frames = batch(dec)
    ref_loss, ref, ref_states = reference(dec, tokens, targets, states, n, frames)
    logp, saved = dec.forward(tokens, states, n, frames)
    loss, dlogits = dec.loss(logp, targets, n)
    dstates = dec.backward(dlogits, saved)
    torch.cuda.synchronize()
    assert abs(loss.item() - ref_loss) <= TOL * abs(ref_loss)
    for name, r in [*ref.items(), ("states", ref_states)]:
        got = (dstates if name == "states" else dec.grad[name]).double().cpu().numpy()
        assert np.isfinite(got).all() and np.abs(got - r).max() <= TOL * np.abs(r).max(), name


def test_decoding_follows_the_teacher_forced_pass():
    import torch
    dec = make(True, dtype="f32", state_bits=32)
    tokens, _, states, n, frames = batch(dec)
    logp, _ = dec.forward(tokens, states, n, frames)
    run = dec.start(states, frames, tokens.shape[1], page=16)
    for cache in run["k"] + run["v"]:
        cache.fill_(float("nan"))  # what is not filled yet is not read
    for u in range(tokens.shape[1]):
        step = dec.next(tokens[:, u], run)
        there = u < n
        assert torch.allclose(step[there], logp[there, :, u], rtol=TOL, atol=TOL)
    with pytest.raises(ValueError):
        dec.next(tokens[:, 0], run)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_chunks_follow_the_teacher_forced_pass(dtype):
    """Prompts of different lengths in one chunk, then another chunk behind them, then tokens one by one.  In bfloat16 the two ways round the
    same some sixty intermediate tensors differently (2^-8 each, in random directions: about 8 * 2^-8 of a logit's size of order one)."""
    import torch
    dec = make(dtype=dtype, state_bits=32)
    U, tol = 40, TOL if dtype == "f32" else 0.15
    tokens, _, states, _, frames = batch(dec, U=U)
    full = torch.full((3,), U, dtype=torch.int32, device="cuda")
    logp, _ = dec.forward(tokens, states, full, frames)
    run = dec.start(states, frames, U + 20, page=16)
    for cache in run["k"] + run["v"]:
        cache.fill_(float("nan"))
    at = [0, 0, 0]
    for counts in ([17, 3, 10], [0, 12, 7], [1, 1, 1]):
        width = max(counts)
        chunk = torch.zeros(3, width, dtype=torch.int64, device="cuda")
        for b, c in enumerate(counts):
            chunk[b, :c] = tokens[b, at[b]:at[b] + c]
        got = dec.extend(chunk, run, torch.tensor(counts, dtype=torch.int32, device="cuda"))
        for b, c in enumerate(counts):
            assert (got[b, :, :c] - logp[b, :, at[b]:at[b] + c]).abs().max().item() <= tol if c else True
            at[b] += c
    ids, best = dec.best(got[:, :, 0], 3)
    want = got[:, :, 0].sort(dim=1, descending=True, stable=True)
    assert torch.equal(ids.long(), want.indices[:, :3]) and torch.allclose(best, want.values[:, :3], atol=1e-5)


def test_counts_beyond_a_chunk_are_its_width():
    import torch
    dec = make(dtype="f32", state_bits=32)
    tokens, _, states, _, frames = batch(dec)
    got = []
    for counts in ([9, 0, 4], [100, -5, 4]):
        run = dec.start(states, frames, 20, page=16)
        first = dec.extend(tokens, run, torch.tensor(counts, dtype=torch.int32, device="cuda"))
        got.append((first[0], first[2, :, :4], dec.next(tokens[:, 0], run)))
        assert run["filled"].tolist() == [10, 1, 5]
    assert all(torch.equal(a, b) for a, b in zip(*got))


def test_training_in_low_precision_with_8_bit_states():
    import torch
    from paper_1909_09577_amd.attn_decoder import AttentionDecoder, spelled
    dec = AttentionDecoder(8, 128, 4, 1, 64, kv_heads=2, seed=0, positions="rotated")
    for i in range(3):
        loss, dstates = dec.step(*spelled(16, 4, 32, 8, 64, dec.dtype, seed=i), lr=2e-3)
        assert torch.isfinite(loss) and torch.isfinite(dstates.float()).all()
    assert all(torch.isfinite(g).all() and g.abs().max() > 0 for g in dec.grad.values())
    assert all(torch.equal(dec.weights[n], dec.master[n].bfloat16()) for n in dec.master if n not in dec.vectors)


def test_what_the_form_refuses():
    from paper_1909_09577_amd.attn_decoder import AttentionDecoder
    with pytest.raises(ValueError):
        AttentionDecoder(8, 96, 4, 1, 64, positions="rotated")  # heads of 24 channels
    with pytest.raises(ValueError):
        AttentionDecoder(8, 128, 4, 1, 64, positions="learned")
    dec = AttentionDecoder(8, 128, 4, 1, 64)
    with pytest.raises(ValueError):
        dec.extend(None, {})
