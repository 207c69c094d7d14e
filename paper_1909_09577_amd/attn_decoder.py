"""A small attention decoder over the encoder's states: training steps and token-by-token decoding through the C ABI.

Each layer has three blocks -- attention to the tokens written so far, attention to the encoder's states, two 1x1 convolutions with a
ReLU between them -- and around each block the norms, the learned scale and the residual add, which are one call.  Projections are
1x1 convolutions of the encoder's layout [batch][channels][time]; the tokens' attention to each other is the same call as that to the
states, over windows that end with the token; every weight and every vector moves in one AdamW call.  This module only wires
calls into libnmconv1d: torch provides device memory, the token table's one-hot rows and the loss's element-wise gradient.

    python -m paper_1909_09577_amd.attn_decoder      # learns to copy a transcript that the states spell out, then decodes it
"""
from __future__ import annotations

from . import binding as nm


def _conv(x, w, **kw):
    return nm.nm_conv1d_block_fwd(x, w, **kw)


class AttentionDecoder:
    """vocab classes, `channels` wide, `heads` heads over kv_heads shared ones, `layers` layers, states of `states` channels.
    dtype: "bf16" (float32 masters, bfloat16 copies) or "f32"; state_bits: of AdamW's moments, 8 or 32."""

    def __init__(self, vocab, channels, heads, layers, states, kv_heads=None, hidden=None, dtype="bf16", state_bits=8, weight_decay=0.01,
                 layer_norm=False, seed=0, device="cuda"):
        import torch
        self.vocab, self.channels, self.heads, self.layers, self.layer_norm = vocab, channels, heads, layers, layer_norm
        self.kv_heads = heads if kv_heads is None else kv_heads
        self.dim = channels // heads
        if self.dim * heads != channels or heads % self.kv_heads:
            raise ValueError("heads must divide channels, kv_heads heads")
        self.dtype = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.device, self.steps, self.seed = device, 0, seed
        kv, hidden = self.kv_heads * self.dim, hidden or 4 * channels
        gen = torch.Generator(device=device)
        gen.manual_seed(seed)
        self.master, self.vectors = {}, set()

        def weight(name, cout, cin, gain=1.0):
            self.master[name] = torch.randn(cout, cin, 1, device=device, generator=gen) * (gain * cin ** -0.5)

        def vector(name, n, value):
            self.master[name] = torch.full((n,), value, device=device)
            self.vectors.add(name)

        weight("table", channels, vocab, vocab ** 0.5 * 0.5)
        for l in range(layers):
            weight(f"{l}.self.in", channels + 2 * kv, channels)
            weight(f"{l}.cross.in", channels, channels)
            weight(f"{l}.cross.states", 2 * kv, states)
            weight(f"{l}.ffn.in", hidden, channels)
            for block, cin in (("self", channels), ("cross", channels), ("ffn", hidden)):
                weight(f"{l}.{block}.out", channels, cin)
                vector(f"{l}.{block}.scale", channels, 0.5)
                for norm in ("next", "post"):  # in front of the block, and of its output
                    vector(f"{l}.{block}.{norm}", channels, 1.0)
                    if layer_norm:
                        vector(f"{l}.{block}.{norm}_bias", channels, 0.0)
        vector("last", channels, 1.0)
        if layer_norm:
            vector("last_bias", channels, 0.0)
        weight("classes", vocab, channels)
        vector("classes_bias", vocab, 0.0)
        self.grad = {n: torch.zeros_like(p) for n, p in self.master.items()}
        low = self.dtype != torch.float32
        self.weights = {n: p if n in self.vectors or not low else p.to(self.dtype) for n, p in self.master.items()}  # what calls read
        names = list(self.master)
        state = {"dtype": torch.float32 if state_bits == 32 else torch.uint8, "device": device}
        scales = None if state_bits == 32 else [[torch.ones(-(-p.numel() // 256), device=device) for p in self.master.values()] for _ in range(2)]
        self.plan = nm.nm_adamw_plan(
            [self.master[n] for n in names], [self.grad[n] for n in names], *([torch.zeros(self.master[n].numel(), **state) for n in names] for _ in range(2)),
            m_scales=scales and scales[0], v_scales=scales and scales[1],
            copies=[self.weights[n] if low and n not in self.vectors else None for n in names],
            weight_decay=[0.0 if n in self.vectors else weight_decay for n in names])

    # ---- pieces -------------------------------------------------------------------------------------
    def _norm_names(self, l, block):
        """The norm behind block `block` of layer l: that of the next block's input."""
        if block == "self":
            return f"{l}.cross.next"
        if block == "cross":
            return f"{l}.ffn.next"
        return f"{l + 1}.self.next" if l + 1 < self.layers else "last"

    def _bias(self, name):
        return self.weights.get(name + "_bias")

    def _positions(self, first, count):
        """[channels, count]: sines and cosines of the positions first .. first + count - 1."""
        import torch
        c = torch.arange(self.channels, device=self.device, dtype=torch.float64)
        at = torch.arange(first, first + count, device=self.device, dtype=torch.float64)
        angle = at[None] * (10000.0 ** (-(c // 2) * 2 / self.channels))[:, None]
        return torch.where((c % 2 == 0)[:, None], angle.sin(), angle.cos()).mul(0.5).to(self.dtype)

    def _embed(self, tokens, first):
        """(one-hot rows [B, vocab, U], h [B, channels, U]) of token numbers [B, U]."""
        import torch
        rows = (tokens[:, None] == torch.arange(self.vocab, device=self.device)[None, :, None]).to(self.dtype)
        pos = self._positions(first, tokens.shape[1])[None].expand(tokens.shape[0], -1, -1).contiguous()
        return rows, _conv(rows, self.weights["table"], residual=pos)

    def _around(self, l, block, h, f, lengths):
        """Behind a block: h + scale * norm(f), and the norm in front of the next one."""
        w, name, nxt = self.weights, f"{l}.{block}", self._norm_names(l, block)
        return nm.nm_residual_norm_fwd(h, f, rscale=w[name + ".scale"], post_weight=w[name + ".post"], post_bias=self._bias(name + ".post"),
                                       next_weight=w[nxt], next_bias=self._bias(nxt), layer=self.layer_norm, lengths=lengths)

    def _around_bwd(self, l, block, dh, dn, h, f, lengths):
        w, g, name, nxt = self.weights, self.grad, f"{l}.{block}", self._norm_names(l, block)
        out = {"drscale": g[name + ".scale"], "dpost_weight": g[name + ".post"], "dpost_bias": g.get(name + ".post_bias"), "dnext_weight": g[nxt],
               "dnext_bias": g.get(nxt + "_bias")}
        got = nm.nm_residual_norm_bwd(dh, dn, h, f, rscale=w[name + ".scale"], post_weight=w[name + ".post"], post_bias=self._bias(name + ".post"),
                                      next_weight=w[nxt], next_bias=self._bias(nxt), layer=self.layer_norm, lengths=lengths, out=out)
        return got["dx"], got["df"]

    def _conv_bwd(self, name, x, dy, **kw):
        return nm.nm_conv1d_bwd(x, dy, self.weights[name], dw=self.grad[name], **kw)[0]

    def _split(self, t):
        """Queries, keys and values of a projection's output, in place."""
        n, kv = t.shape[1] - 2 * self.kv_heads * self.dim, self.kv_heads * self.dim
        return t[:, :n], t[:, n:n + kv], t[:, n + kv:]

    # ---- training -----------------------------------------------------------------------------------
    def forward(self, tokens, states, token_lengths, state_lengths):
        """(log-probabilities [B, vocab, U] of every next token, what backward() needs); tokens int64 [B, U], states
        [B, channels, T], lengths int32 [B]."""
        import torch
        B, U = tokens.shape
        w, heads = self.weights, {"heads": self.heads, "kv_heads": self.kv_heads}
        u = torch.arange(U, device=self.device, dtype=torch.int32)
        past = torch.stack([torch.zeros_like(u), u + 1], 1).expand(B, U, 2).contiguous()
        own = dict(heads, lengths=token_lengths, q_lengths=token_lengths, windows=past)
        to_states = dict(heads, lengths=state_lengths, q_lengths=token_lengths)
        rows, h = self._embed(tokens, 0)
        saved = {"rows": rows, "h0": h, "states": states, "own": own, "to_states": to_states, "lengths": token_lengths, "layers": []}
        _, n = nm.nm_residual_norm_fwd(h, next_weight=w["0.self.next"], next_bias=self._bias("0.self.next"), layer=self.layer_norm, lengths=token_lengths)
        for l in range(self.layers):
            s = {"self.n": n}
            s["qkv"] = _conv(n, w[f"{l}.self.in"])
            s["self.o"], s["self.lse"] = nm.nm_cross_attn_fwd(*self._split(s["qkv"]), want_lse=True, **own)
            s["self.f"] = _conv(s["self.o"], w[f"{l}.self.out"])
            s["self.h"], n = h, s["cross.n"] = self._around(l, "self", h, s["self.f"], token_lengths)
            s["q"], s["kv"] = _conv(n, w[f"{l}.cross.in"]), _conv(states, w[f"{l}.cross.states"])
            s["cross.o"], s["cross.lse"] = nm.nm_cross_attn_fwd(s["q"], *self._split(s["kv"])[1:], want_lse=True, **to_states)
            s["cross.f"] = _conv(s["cross.o"], w[f"{l}.cross.out"])
            s["cross.h"], n = h, s["ffn.n"] = self._around(l, "cross", h, s["cross.f"], token_lengths)
            s["hidden"] = _conv(n, w[f"{l}.ffn.in"], relu=True)
            s["ffn.f"] = _conv(s["hidden"], w[f"{l}.ffn.out"])
            s["ffn.h"], n = h, _ = self._around(l, "ffn", h, s["ffn.f"], token_lengths)
            saved["layers"].append(s)
        saved["n"] = n
        logp = nm.nm_decoder_logsoftmax_fwd(n, w["classes"][:, :, 0], w["classes_bias"])
        return logp, saved

    def backward(self, dlogits, saved):
        """Gradients of every parameter (self.grad) and of the states (returned) from those of the class scores, [B, vocab, U] float32,
        zero behind every item's tokens."""
        import torch
        g, lengths = self.grad, saved["lengths"]
        g["classes_bias"].copy_(dlogits.sum((0, 2)))
        dn, dh = self._conv_bwd("classes", saved["n"], dlogits.to(self.dtype)), None
        dstates = None
        for l in reversed(range(self.layers)):
            s = saved["layers"][l]
            dh, df = self._around_bwd(l, "ffn", dh, dn, s["ffn.h"], s["ffn.f"], lengths)
            dhidden = self._conv_bwd(f"{l}.ffn.out", s["hidden"], df)
            dn = self._conv_bwd(f"{l}.ffn.in", s["ffn.n"], dhidden, y=s["hidden"], relu=True)
            dh, df = self._around_bwd(l, "cross", dh, dn, s["cross.h"], s["cross.f"], lengths)
            do = self._conv_bwd(f"{l}.cross.out", s["cross.o"], df)
            dkv = torch.empty_like(s["kv"])
            dq, _, _ = nm.nm_cross_attn_bwd(do, s["q"], *self._split(s["kv"])[1:], s["cross.o"], s["cross.lse"], dk=self._split(dkv)[1],
                                            dv=self._split(dkv)[2], **saved["to_states"])
            dstates = self._conv_bwd(f"{l}.cross.states", saved["states"], dkv, dx=dstates, accumulate_dx=dstates is not None)
            dn = self._conv_bwd(f"{l}.cross.in", s["cross.n"], dq)
            dh, df = self._around_bwd(l, "self", dh, dn, s["self.h"], s["self.f"], lengths)
            do = self._conv_bwd(f"{l}.self.out", s["self.o"], df)
            dqkv = torch.empty_like(s["qkv"])
            dq, dk, dv = self._split(dqkv)
            nm.nm_cross_attn_bwd(do, *self._split(s["qkv"]), s["self.o"], s["self.lse"], dq=dq, dk=dk, dv=dv, **saved["own"])
            dn = self._conv_bwd(f"{l}.self.in", s["self.n"], dqkv)
        first = "0.self.next"
        got = nm.nm_residual_norm_bwd(dh, dn, saved["h0"], next_weight=self.weights[first], next_bias=self._bias(first), layer=self.layer_norm,
                                      lengths=lengths, out={"dnext_weight": g[first], "dnext_bias": g.get(first + "_bias")})
        nm.nm_conv1d_bwd_weight(saved["rows"], got["dx"], 1, dw=g["table"])
        return dstates

    def loss(self, logp, targets, token_lengths):
        """(mean negative log-probability of the targets int64 [B, U], its gradient with respect to the class scores)."""
        import torch
        there = torch.arange(targets.shape[1], device=self.device)[None] < token_lengths[:, None]
        per = there.float() / there.sum().clamp_min(1)
        picked = logp.gather(1, targets[:, None]).squeeze(1)
        grad = (logp.exp() - (targets[:, None] == torch.arange(self.vocab, device=self.device)[None, :, None]).float()) * per[:, None]
        return -(picked * per).sum(), torch.where(there[:, None], grad, 0.0)

    def step(self, tokens, targets, states, token_lengths, state_lengths, *, lr, beta1=0.9, beta2=0.98, eps=1e-8):
        """One training step; returns (loss before it, gradient of the states)."""
        logp, saved = self.forward(tokens, states, token_lengths, state_lengths)
        loss, dlogits = self.loss(logp, targets, token_lengths)
        dstates = self.backward(dlogits, saved)
        self.steps += 1
        nm.nm_adamw_step(self.plan, lr=lr, beta1=beta1, beta2=beta2, eps=eps, step=self.steps, seed=self.seed * 0x9E3779B1 + self.steps)
        return loss, dstates

    # ---- decoding -----------------------------------------------------------------------------------
    def start(self, states, state_lengths, room):
        """What the tokens of a batch of utterances need: every layer's keys and values of the states, and room for those of `room`
        tokens (channel-major, a token's column is filled when it is known)."""
        import torch
        B, width = states.shape[0], 2 * self.kv_heads * self.dim
        return {"kv": [_conv(states, self.weights[f"{l}.cross.states"]) for l in range(self.layers)], "state_lengths": state_lengths, "at": 0, "room": room,
                "cache": [torch.empty(B, width, room, dtype=self.dtype, device=self.device) for _ in range(self.layers)],
                "filled": torch.zeros(B, dtype=torch.int32, device=self.device)}

    def next(self, tokens, run):
        """Log-probabilities [B, vocab] of what follows the tokens int64 [B], the latest of every utterance."""
        if run["at"] >= run["room"]:
            raise ValueError("no room for another token")
        w, heads = self.weights, {"heads": self.heads, "kv_heads": self.kv_heads}
        _, h = self._embed(tokens[:, None], run["at"])
        run["filled"] += 1
        _, n = nm.nm_residual_norm_fwd(h, next_weight=w["0.self.next"], next_bias=self._bias("0.self.next"), layer=self.layer_norm)
        for l in range(self.layers):
            qkv = _conv(n, w[f"{l}.self.in"])
            q, cache = self._split(qkv)[0], run["cache"][l]
            cache[:, :, run["at"]] = qkv[:, q.shape[1]:, 0]
            o, _ = nm.nm_cross_attn_fwd(q, *self._split(cache)[1:], lengths=run["filled"], **heads)
            h, n = self._around(l, "self", h, _conv(o, w[f"{l}.self.out"]), None)
            o, _ = nm.nm_cross_attn_fwd(_conv(n, w[f"{l}.cross.in"]), *self._split(run["kv"][l])[1:], lengths=run["state_lengths"], **heads)
            h, n = self._around(l, "cross", h, _conv(o, w[f"{l}.cross.out"]), None)
            h, n = self._around(l, "ffn", h, _conv(_conv(n, w[f"{l}.ffn.in"], relu=True), w[f"{l}.ffn.out"]), None)
        run["at"] += 1
        return nm.nm_decoder_logsoftmax_fwd(n, w["classes"][:, :, 0], w["classes_bias"])[:, :, 0]


def spelled(batch, tokens, frames, vocab, channels, dtype, seed, device="cuda"):
    """A task for trying the decoder: transcripts of 2 to `tokens` symbols (0 begins and ends them) and states that hold every symbol for
    frames/tokens frames.  (tokens in, targets, states, token lengths, state lengths)"""
    import torch
    gen = torch.Generator(device=device)
    gen.manual_seed(seed)
    ints = lambda lo, hi, *shape: torch.randint(lo, hi, shape, device=device, generator=gen)  # noqa: E731
    symbols, n = ints(1, vocab, batch, tokens), ints(2, tokens + 1, batch)
    u = torch.arange(tokens, device=device)[None]
    symbols = torch.where(u < n[:, None], symbols, 0)
    ins = torch.cat([torch.zeros_like(symbols[:, :1]), symbols], 1)
    targets = torch.cat([symbols, torch.zeros_like(symbols[:, :1])], 1)
    per = frames // tokens
    code = torch.randn(vocab, channels, device=device, generator=torch.Generator(device=device).manual_seed(1234))
    place = torch.randn(tokens, channels, device=device, generator=torch.Generator(device=device).manual_seed(4321))
    at = (torch.arange(frames, device=device) // per).clamp_max(tokens - 1)
    states = (code[symbols[:, at]] + place[at][None]).transpose(1, 2).to(dtype).contiguous()
    return ins, targets, states, (n + 1).to(torch.int32), (n * per).to(torch.int32)


def main():
    import torch
    vocab, room = 29, 12
    dec = AttentionDecoder(vocab, 256, 4, 2, 256, kv_heads=2, seed=1)
    for i in range(400):
        batch = spelled(32, room, 96, vocab, 256, dec.dtype, seed=i)
        loss, _ = dec.step(*batch, lr=2e-3 * min((i + 1) / 50, (400 - i) / 350))
        if i % 50 == 0 or i == 399:
            print(f"step {i}: loss {loss.item():.3f}", flush=True)
    ins, targets, states, n, frames = spelled(8, room, 96, vocab, 256, dec.dtype, seed=10 ** 6)
    run, token, out = dec.start(states, frames, room + 1), ins[:, 0], []
    for _ in range(room + 1):
        token = dec.next(token, run).argmax(1)
        out.append(token)
    there = torch.arange(room + 1, device="cuda")[None] < n[:, None]
    right = (torch.stack(out, 1) == targets)[there].float().mean().item()
    print(f"decoded symbols that are right: {100 * right:.1f} %")


if __name__ == "__main__":
    main()
