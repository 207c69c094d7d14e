"""The attention decoder on the calls it is made of: gradients of a whole step against float64 differentiation of the same model,
token-by-token decoding against the teacher-forced pass, and training with 8-bit states.

Tolerances (derived, float32 storage): a result passes through some thirty calls one after the other, each off by at most n * 2^-24 of the
magnitudes it adds (n up to 100 terms) and gains of order one between them: 30 * 100 * 2^-24 = 2e-4 of the largest element of a gradient, taken
five times for the gains of the norms (1/rms up to some units)."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
TOL = 1e-3


def make(layer_norm, seed=3, **kw):
    import torch
    from paper_1909_09577_amd.attn_decoder import AttentionDecoder
    dec = AttentionDecoder(13, 64, 4, 2, 48, kv_heads=2, hidden=80, layer_norm=layer_norm, seed=seed, **kw)
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
    pos = dec._positions(0, tokens.shape[1]).double().cpu()
    H, G, D = dec.heads, dec.heads // dec.kv_heads, dec.dim

    def norm(x, name):
        z = x - x.mean(0, keepdim=True) if dec.layer_norm else x
        z = z / (z.square().mean(0, keepdim=True) + 1e-5).sqrt() * P[name][:, None]
        return z + P[name + "_bias"][:, None] if dec.layer_norm else z

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
        h = mat("table")[:, tokens[b, :u].cpu()] + pos[:, :u]
        x = norm(h, "0.self.next")
        for l in range(dec.layers):
            for block in ("self", "cross", "ffn"):
                if block == "self":
                    p = mat(f"{l}.self.in") @ x
                    f = attend(p[:C], p[C:C + kv], p[C + kv:], True)
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
    run = dec.start(states, frames, tokens.shape[1])
    for cache in run["cache"]:
        cache.fill_(float("nan"))  # what is not filled yet is not read
    for u in range(tokens.shape[1]):
        step = dec.next(tokens[:, u], run)
        there = u < n
        assert torch.allclose(step[there], logp[there, :, u], rtol=TOL, atol=TOL)
    with pytest.raises(ValueError):
        dec.next(tokens[:, 0], run)


def test_training_in_low_precision_with_8_bit_states():
    import torch
    from paper_1909_09577_amd.attn_decoder import AttentionDecoder, spelled
    dec = AttentionDecoder(8, 128, 4, 1, 64, kv_heads=2, seed=0)
    losses = []
    for i in range(60):
        loss, _ = dec.step(*spelled(16, 4, 32, 8, 64, dec.dtype, seed=i), lr=2e-3)
        losses.append(loss)
    torch.cuda.synchronize()
    losses = [x.item() for x in losses]
    assert np.isfinite(losses).all() and np.mean(losses[-5:]) < 0.5 * losses[0]
    assert all(torch.equal(dec.weights[n], dec.master[n].bfloat16()) for n in dec.master if n not in dec.vectors)
