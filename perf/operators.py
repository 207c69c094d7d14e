"""The workloads on which the operators of an attention decoder over the encoder's states are timed and checked: cross
attention, the norms around a block with its gate and residual scale, and the AdamW step that ends a training step.

A case is a dict of plain values.  Its "kind" says which call one pass makes:

  attn_fwd   cross attention of U decoder tokens to T encoder frames: outputs and log-sum-exp (U = 1 to 8: a decoding step,
             the hypotheses of a beam search side by side)
  attn_bwd   its backward pass, from saved outputs
  norm_fwd   y = x + rscale * gate * post_norm(f) and n = next_norm(y) in one pass (T = 1: a decoding step)
  norm_bwd   its backward pass, parameter gradients included
  adamw      one step over every tensor of an encoder, states in 32 or in 8 bits

Tensors are channel-major, [batch][channels][time], like the encoder's activations; heads lie side by side in the channels.
"lengths" makes a padded batch: every utterance has its own number of frames and of tokens.  "windows" gives every token a
range of frames of its own around its place in the utterance.  Sizes: the encoder's channel counts (256 to 1024) in heads of 64, 80, 96 and 128,
training batches of 32 utterances of 16 seconds, utterances of minutes for long-form transcription, single tokens.
"""
import math

import torch

own = False  # set from outside: False computes the operators in their plain form, True calls the library

SCALE_BLOCK = 256  # elements that share a scale of the 8-bit states
E4M3_MAX = 448.0
ADAMW = {"lr": 1e-3, "beta1": 0.9, "beta2": 0.98, "eps": 1e-8, "weight_decay": 0.01}
EPS = 1e-5

DEFAULTS = {"dtype": "bf16", "lengths": False, "windows": False, "layer": False, "gate": "item", "bits": 32, "width": 1}


def listed():
    return [
        # one token of one utterance of 12 seconds: the smallest call, launches and latency count
        {"name": "step_b1_u1", "kind": "attn_fwd", "B": 1, "H": 16, "Hkv": 16, "D": 64, "U": 1, "T": 600},
        # a decoding step of a serving batch, eight hypotheses per utterance, shared key and value heads
        {"name": "step_beams_gqa", "kind": "attn_fwd", "B": 32, "H": 16, "Hkv": 4, "D": 64, "U": 8, "T": 800, "lengths": True},
        # a training step's batch: 32 utterances of up to 16 seconds and their transcripts
        {"name": "train_fwd_b32", "kind": "attn_fwd", "B": 32, "H": 16, "Hkv": 16, "D": 64, "U": 150, "T": 800, "lengths": True},
        {"name": "train_bwd_b32", "kind": "attn_bwd", "B": 32, "H": 16, "Hkv": 16, "D": 64, "U": 150, "T": 800, "lengths": True},
        # recordings of two and a half minutes, of no particular length, wide heads
        {"name": "long_fwd_d128", "kind": "attn_fwd", "B": 4, "H": 8, "Hkv": 8, "D": 128, "U": 700, "T": 7501},
        # a minute, shared key and value heads, every token looks at the frames around its place
        {"name": "windows_bwd_gqa", "kind": "attn_bwd", "B": 4, "H": 8, "Hkv": 2, "D": 128, "U": 333, "T": 3001, "windows": True},
        # the float32 mode: a model debugged without low precision, on a small batch
        {"name": "f32_bwd", "kind": "attn_bwd", "B": 4, "H": 4, "Hkv": 4, "D": 64, "U": 40, "T": 401, "dtype": "f32", "lengths": True},
        # around a block on the encoder's frames in training, a gate per utterance and channel
        {"name": "norm_fwd_1024", "kind": "norm_fwd", "B": 32, "C": 1024, "T": 800, "layer": True},
        # the backward pass on a padded batch of odd length, a gate per element
        {"name": "norm_bwd_ragged_768", "kind": "norm_bwd", "B": 16, "C": 768, "T": 777, "gate": "element", "lengths": True},
        # a decoding step of a serving batch
        {"name": "norm_step", "kind": "norm_fwd", "B": 16, "C": 1024, "T": 1},
        # the weights of the whole 64-layer encoder, states in float32 and in 8 bits
        {"name": "adamw_encoder", "kind": "adamw", "width": 4},
        {"name": "adamw_encoder_8bit", "kind": "adamw", "width": 4, "bits": 8},
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of these ranges, no costlier than the largest of its kind above."""
    kind = rng.choice(["step", "attn_fwd", "attn_fwd", "attn_bwd", "attn_bwd", "f32", "norm_fwd", "norm_bwd", "norm_step", "adamw"])

    def odd(n):  # half of the lengths as they come, half in whole groups
        return n if n < 16 or rng.random() < 0.5 else n // 8 * 8

    if kind == "adamw":
        return {"kind": "adamw", "width": rng.randint(1, 3), "bits": rng.choice([8, 32]), "tail": rng.randint(1, 5000)}
    if kind.startswith("norm"):
        c = {"kind": kind, "C": rng.choice([256, 384, 512, 640, 768, 896, 1024]), "layer": rng.random() < 0.5,
             "gate": rng.choice(["none", "item", "element"]), "dtype": "f32" if rng.random() < 0.25 else "bf16"}
        if kind == "norm_step":
            return dict(c, kind="norm_fwd", B=_log_uniform(rng, 1, 64), T=rng.choice([1, 1, 2, 5, 8]))
        return dict(c, B=_log_uniform(rng, 1, 16), T=odd(_log_uniform(rng, 20, 800)), lengths=rng.random() < 0.5)
    d = rng.choice([64, 64, 80, 96, 128])
    h = {64: rng.choice([4, 8, 12, 16]), 80: 8, 96: 8, 128: rng.choice([4, 8])}[d]
    c = {"kind": kind, "H": h, "Hkv": rng.choice([h, h, h // 2, h // 4]), "D": d, "lengths": rng.random() < 0.5, "windows": rng.random() < 0.25}
    if kind == "step":
        return dict(c, kind="attn_fwd", B=_log_uniform(rng, 1, 32), U=rng.randint(1, 8), T=odd(_log_uniform(rng, 50, 7501)))
    if kind == "f32":
        return dict(c, kind=rng.choice(["attn_fwd", "attn_bwd"]), dtype="f32", B=_log_uniform(rng, 1, 4), U=_log_uniform(rng, 1, 100),
                    T=odd(_log_uniform(rng, 50, 800)))
    t = odd(_log_uniform(rng, 50, 4000))
    return dict(c, B=_log_uniform(rng, 1, 32 if t < 1000 else 4), U=_log_uniform(rng, 10, 200 if t < 1000 else 400), T=t)


# ---- inputs -----------------------------------------------------------------------------------------------------
def _full(case):
    return dict(DEFAULTS, **case)


def _storage(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _encoder_tensors(width, tail):
    """Element counts of the weights (decayed) and of the vectors (not decayed) of the 64-layer encoder with width/4 of its channels,
    and of one more tensor of `tail` elements."""
    def ch(n):
        return n * width // 4

    weights, vectors, cin = [ch(256) * 64 * 11], [ch(256)] * 2, ch(256)
    for c, k in [(256, 11), (256, 11), (384, 13), (384, 13), (512, 17), (512, 17), (640, 21), (640, 21), (768, 25), (768, 25)]:
        weights += [ch(c) * cin, ch(c) * cin * k] + [ch(c) * ch(c) * k] * 4
        vectors += [ch(c)] * 12
        cin = ch(c)
    weights += [ch(896) * cin * 29, ch(1024) * ch(896), 29 * ch(1024)]
    vectors += [ch(896)] * 2 + [ch(1024)] * 2 + [29]
    return weights, vectors + ([tail] if tail else [])


def _lengths(g, b, n):
    """b lengths between half of n and n, the longest of them n; int32."""
    ln = torch.randint((n + 1) // 2, n + 1, (b,), device="cuda", generator=g, dtype=torch.int32)
    ln[torch.randint(0, b, (1,), device="cuda", generator=g)] = n
    return ln


def _attn_inputs(c, g, dt):
    B, H, Hkv, D, U, T = (c[k] for k in ("B", "H", "Hkv", "D", "U", "T"))
    s = {"heads": H, "kv_heads": Hkv, "scale": D ** -0.5}
    s["q"] = (1.5 * torch.randn(B, H * D, U, device="cuda", generator=g)).to(dt)
    kv = torch.randn(B, 2 * Hkv * D, T, device="cuda", generator=g).to(dt)  # one projection's output: keys, then values
    s["k"], s["v"] = kv[:, :Hkv * D], kv[:, Hkv * D:]
    s["lengths"] = _lengths(g, B, T) if c["lengths"] else None
    s["q_lengths"] = _lengths(g, B, U) if c["lengths"] else None
    s["windows"] = None
    if c["windows"]:
        at = torch.arange(U, device="cuda")[None] * (T / U) + torch.randn(B, U, device="cuda", generator=g) * (T / 50)
        w = T / 8
        s["windows"] = torch.stack([at - w, at + w], dim=2).round().clamp(0, T).to(torch.int32).contiguous()
    if c["kind"] == "attn_bwd":
        o, lse = _attn_fwd(s)
        s["o"], s["lse"] = o, lse
        s["do"] = torch.randn(B, H * D, U, device="cuda", generator=g).to(dt)
    return s


def _norm_inputs(c, g, dt):
    B, C, T = c["B"], c["C"], c["T"]
    draw_act = lambda: torch.randn(B, C, T, device="cuda", generator=g).to(dt)  # noqa: E731
    vec = lambda mid, spread: mid + spread * torch.randn(C, device="cuda", generator=g)  # noqa: E731
    s = {"layer": c["layer"], "f": draw_act(), "rscale": vec(0.5, 0.1), "post_weight": vec(1.0, 0.1), "next_weight": vec(1.0, 0.1)}
    s["post_bias"], s["next_bias"] = (vec(0.0, 0.1), vec(0.0, 0.1)) if c["layer"] else (None, None)
    s["gate"] = {"none": lambda: None, "item": lambda: torch.rand(B, C, device="cuda", generator=g),
                 "element": lambda: torch.rand(B, C, T, device="cuda", generator=g).to(dt)}[c["gate"]]()
    s["lengths"] = _lengths(g, B, T) if c["lengths"] else None
    if c["kind"] == "norm_fwd":
        s["x"] = draw_act()
    else:
        s["y"], s["dy"], s["dn"] = draw_act(), draw_act(), draw_act()
    return s


def _adamw_inputs(c, g):
    """Parameters, gradients and the states of some hundred steps, each in one flat buffer in which every tensor begins at a whole
    block of 256 elements (zeros behind its end)."""
    weights, vectors = _encoder_tensors(c["width"], c.get("tail", 0))
    sizes = weights + vectors
    padded = [-(-n // SCALE_BLOCK) * SCALE_BLOCK for n in sizes]
    total = sum(padded)
    flat = lambda mul: torch.randn(total, device="cuda", generator=g).mul_(mul)  # noqa: E731
    s = {"bits": c["bits"], "step": 300, "seed": int(torch.randint(0, 1 << 31, (1,), device="cuda", generator=g)),
         "param": flat(0.02), "grad": flat(1e-3), "decayed": sum(padded[:len(weights)])}
    m, r = flat(3e-4), flat(3e-4).abs_().add_(5e-4)  # first moment, root of the second
    at = 0
    for n, p in zip(sizes, padded):
        for t in (s["param"], s["grad"], m, r):
            t[at + n:at + p] = 0
        at += p
    s["copy"] = s["param"].to(torch.bfloat16)
    if c["bits"] == 8:
        for name, t in (("m", m), ("r", r)):
            sc = t.view(-1, SCALE_BLOCK).abs().amax(1) / E4M3_MAX
            s[name + "_scale"] = torch.where(sc > 0, sc, 1.0)
            s[name + "_codes"] = (t.view(-1, SCALE_BLOCK) / s[name + "_scale"][:, None]).to(torch.float8_e4m3fn).view(-1).view(torch.uint8)
    else:
        s["m"], s["v"] = m, r.square_()
    if own:  # the handle that a training program makes once, when it has its tensors
        from paper_1909_09577_amd import binding as nm

        def cut(t, per=1):
            out, at = [], 0
            for n, p in zip(sizes, padded):
                out.append(t[at // per:at // per + -(-n // per)])
                at += p
            return out

        decay = [ADAMW["weight_decay"]] * len(weights) + [0.0] * len(vectors)
        if c["bits"] == 8:
            s["plan"] = nm.nm_adamw_plan(cut(s["param"]), cut(s["grad"]), cut(s["m_codes"]), cut(s["r_codes"]),
                                         m_scales=cut(s["m_scale"], SCALE_BLOCK), v_scales=cut(s["r_scale"], SCALE_BLOCK),
                                         copies=cut(s["copy"]), weight_decay=decay)
        else:
            s["plan"] = nm.nm_adamw_plan(cut(s["param"]), cut(s["grad"]), cut(s["m"]), cut(s["v"]), copies=cut(s["copy"]),
                                         weight_decay=decay)
    return s


def prepare(case, seed):
    c = _full(case)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt = _storage(c)
    s = _adamw_inputs(c, g) if c["kind"] == "adamw" else _norm_inputs(c, g, dt) if c["kind"].startswith("norm") else _attn_inputs(c, g, dt)
    s["kind"] = c["kind"]
    return s


# ---- one pass ---------------------------------------------------------------------------------------------------
def run(s):
    kind = s["kind"]
    if own:
        from paper_1909_09577_amd import binding as nm
        if kind == "adamw":
            return _adamw_own(nm, s)
        if kind.startswith("norm"):
            names = ("layer", "gate", "rscale", "post_weight", "post_bias", "next_weight", "next_bias", "lengths")
            kw = {k: s[k] for k in names}
            if kind == "norm_fwd":
                return nm.nm_residual_norm_fwd(s["x"], s["f"], eps=EPS, **kw)
            return nm.nm_residual_norm_bwd(s["dy"], s["dn"], s["y"], s["f"], eps=EPS, **kw)  # a dict of gradients
        kw = {k: s[k] for k in ("heads", "kv_heads", "scale", "lengths", "q_lengths", "windows")}
        if kind == "attn_fwd":
            return nm.nm_cross_attn_fwd(s["q"], s["k"], s["v"], want_lse=True, **kw)
        return nm.nm_cross_attn_bwd(s["do"], s["q"], s["k"], s["v"], s["o"], s["lse"], **kw)
    if kind == "adamw":
        return _adamw(s)
    return {"attn_fwd": _attn_fwd, "attn_bwd": _attn_bwd, "norm_fwd": _norm_fwd, "norm_bwd": _norm_bwd}[kind](s)


def _adamw_outputs(s):
    """Parameters and states after the step; what is held in 8 bits as the values it stands for (m, and the root of v)."""
    if s["bits"] == 32:
        return {"param": s["param"], "copy": s["copy"], "m": s["m"], "v": s["v"]}
    out = {"param": s["param"], "copy": s["copy"]}
    for name in ("m", "r"):
        codes = s[name + "_codes"].view(torch.float8_e4m3fn).to(torch.float32).view(-1, SCALE_BLOCK)
        out[name] = codes * s[name + "_scale"][:, None]
    return out


def _adamw_own(nm, s):
    a = ADAMW
    nm.nm_adamw_step(s["plan"], lr=a["lr"], beta1=a["beta1"], beta2=a["beta2"], eps=a["eps"], step=s["step"], seed=s["seed"] + s["step"])
    s["step"] += 1
    return _adamw_outputs(s)


# ---- the plain forms ----------------------------------------------------------------------------------------------
def _allowed(s, B, U, T):
    """[B, U, T] truth values: which frames a token may look at."""
    t = torch.arange(T, device="cuda")[None, None]
    ok = torch.ones(B, U, T, dtype=torch.bool, device="cuda")
    if s["lengths"] is not None:
        ok = ok & (t < s["lengths"][:, None, None])
    if s["q_lengths"] is not None:
        ok = ok & (torch.arange(U, device="cuda")[None, :, None] < s["q_lengths"][:, None, None])
    if s["windows"] is not None:
        ok = ok & (t >= s["windows"][:, :, :1]) & (t < s["windows"][:, :, 1:])
    return ok


def _heads(x, heads, groups):
    """[B, heads*D, N] as [B*heads/groups, groups, N, D] in float32."""
    B, HD, N = x.shape
    return x.float().reshape(B * heads // groups, groups, HD // heads, N).transpose(2, 3)


def _probabilities(s):
    B, HD, U = s["q"].shape
    T, H, Hkv = s["k"].shape[2], s["heads"], s["kv_heads"]
    G = H // Hkv
    q = _heads(s["q"], H, G)                                        # [B*Hkv, G, U, D]
    k, v = _heads(s["k"], Hkv, 1)[:, 0], _heads(s["v"], Hkv, 1)[:, 0]  # [B*Hkv, T, D]
    D = q.shape[3]
    sc = torch.bmm(q.reshape(-1, G * U, D), k.transpose(1, 2).contiguous()).mul_(s["scale"]).reshape(B, Hkv, G, U, T)
    if s["lengths"] is not None or s["windows"] is not None:
        sc.masked_fill_(~_allowed(s, B, U, T)[:, None, None], -math.inf)
    top = sc.amax(-1, keepdim=True)
    top = torch.where(top > -math.inf, top, 0.0)
    p = sc.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    p = p.div_(torch.where(total > 0, total, 1.0))
    lse = (top + total.log())[..., 0].reshape(B, H, U)
    return q, k, v, p.reshape(B * Hkv, G * U, T), lse


def _attn_fwd(s):
    q, k, v, p, lse = _probabilities(s)
    B, HD, U = s["q"].shape
    o = torch.bmm(p, v.contiguous()).reshape(-1, U, q.shape[3]).transpose(1, 2).reshape(B, HD, U)
    return o.to(s["q"].dtype).contiguous(), lse


def _attn_bwd(s):
    q, k, v, p, _ = _probabilities(s)
    B, HD, U = s["q"].shape
    n, G, _, D = q.shape
    T = k.shape[1]
    do = _heads(s["do"], s["heads"], G).reshape(n, G * U, D)
    q = q.reshape(n, G * U, D)
    dv = torch.bmm(do.transpose(1, 2).contiguous(), p)              # [n, D, T]
    dp = torch.bmm(do, v.transpose(1, 2).contiguous())
    ds = dp.sub_((dp * p).sum(-1, keepdim=True)).mul_(p).mul_(s["scale"])
    dk = torch.bmm(q.transpose(1, 2).contiguous(), ds)
    dq = torch.bmm(ds, k.contiguous())                              # [n, G*U, D]
    dq = dq.reshape(-1, U, D).transpose(1, 2).reshape(B, HD, U)
    dt = s["q"].dtype
    return dq.to(dt).contiguous(), dk.reshape(B, -1, T).to(dt), dv.reshape(B, -1, T).to(dt)


def _normed(z, s, weight, bias):
    """(z normalised over the channels, 1/deviation, with weight and bias), float32."""
    zc = z - z.mean(1, keepdim=True) if s["layer"] else z
    rstd = (zc.square().mean(1, keepdim=True) + EPS).rsqrt()
    hat = zc * rstd
    out = hat * weight[None, :, None]
    return hat, rstd, out if bias is None else out + bias[None, :, None]


def _valid(s, B, T):
    """[B, 1, T] truth values of the positions inside an utterance, or None."""
    return None if s["lengths"] is None else (torch.arange(T, device="cuda")[None] < s["lengths"][:, None])[:, None]


def _gain(s):
    """rscale * gate, broadcast over the activations."""
    r = s["rscale"][None, :, None]
    gate = s["gate"]
    return r if gate is None else r * (gate.float() if gate.dim() == 3 else gate[:, :, None])


def _norm_fwd(s):
    x = s["x"].float()
    _, _, h = _normed(s["f"].float(), s, s["post_weight"], s["post_bias"])
    y = (x + _gain(s) * h).to(s["x"].dtype)
    _, _, n = _normed(y.float(), s, s["next_weight"], s["next_bias"])
    n = n.to(y.dtype)
    ok = _valid(s, x.shape[0], x.shape[2])
    return (y, n) if ok is None else (torch.where(ok, y, 0), torch.where(ok, n, 0))


def _norm_back(d, hat, rstd, s, weight):
    """Gradient with respect to a norm's input from that of its output."""
    dh = d * weight[None, :, None]
    out = dh - hat * (dh * hat).mean(1, keepdim=True)
    if s["layer"]:
        out = out - dh.mean(1, keepdim=True)
    return out * rstd


def _norm_bwd(s):
    dt, layer, gate = s["dy"].dtype, s["layer"], s["gate"]
    dy, dn, y, f = (s[k].float() for k in ("dy", "dn", "y", "f"))
    ok = _valid(s, dy.shape[0], dy.shape[2])
    if ok is not None:
        dy, dn = torch.where(ok, dy, 0.0), torch.where(ok, dn, 0.0)
    hat, rstd, _ = _normed(y, s, s["next_weight"], s["next_bias"])
    out = {"dnext_weight": (dn * hat).sum((0, 2)), "dnext_bias": dn.sum((0, 2)) if layer else None}
    grad = dy + _norm_back(dn, hat, rstd, s, s["next_weight"])
    out["dx"] = grad.to(dt)
    hat, rstd, h = _normed(f, s, s["post_weight"], s["post_bias"])
    g3 = 1.0 if gate is None else gate.float() if gate.dim() == 3 else gate[:, :, None]
    gh = grad * h
    out["drscale"] = (gh * g3).sum((0, 2))
    out["dgate"] = None
    if gate is not None:
        dgate = gh * s["rscale"][None, :, None]
        out["dgate"] = dgate.to(dt) if gate.dim() == 3 else dgate.sum(2)
    dh = grad * _gain(s)
    out["dpost_weight"], out["dpost_bias"] = (dh * hat).sum((0, 2)), dh.sum((0, 2)) if layer else None
    out["df"] = _norm_back(dh, hat, rstd, s, s["post_weight"]).to(dt)
    return out


def _mixed(seed, n):
    """32 well-mixed bits for each of n elements from a seed and the element's number: multiplications by the leading bits of the
    fractional parts of the golden ratio and of the roots of two and three, shifts between them, in 32-bit arithmetic."""
    low = 0xFFFFFFFF
    h = (torch.arange(n, device="cuda", dtype=torch.int64) * 0x9E3779B9 & low) ^ (seed & low)
    h = (h ^ (h >> 16)) * 0x6A09E667 & low
    h = (h ^ (h >> 13)) * 0xBB67AE85 & low
    return h ^ (h >> 16)


def _to_codes(t, u, positive):
    """(E4M3 codes, a scale per block) of float64 values t: value/scale is rounded down or up to a neighbour, up where the rest is
    at least 1 - u.  positive: values above zero do not become zero."""
    amax = t.view(-1, SCALE_BLOCK).abs().amax(1)
    scale = torch.where(amax > 0, (amax / E4M3_MAX).float().clamp_min(2.0 ** -126), 1.0)
    y = (t.view(-1, SCALE_BLOCK).abs() / scale.double()[:, None]).view(-1)
    ulp = torch.ldexp(torch.ones_like(y), (torch.frexp(y).exponent - 1).clamp_min(-6) - 3)
    q = ((y / ulp + u).floor_() * ulp).clamp_max_(E4M3_MAX)
    if positive:
        q = torch.where((y > 0) & (q == 0), 2.0 ** -9, q)
    return torch.where(t < 0, -q, q).float().to(torch.float8_e4m3fn).view(torch.uint8), scale


def _adamw(s):
    a, t = ADAMW, s["step"]
    p, g, nd = s["param"], s["grad"], s["decayed"]
    size, root = a["lr"] / (1 - a["beta1"] ** t), (1 - a["beta2"] ** t) ** -0.5
    if s["bits"] == 32:
        m, v = s["m"], s["v"]
        m.mul_(a["beta1"]).add_(g * (1 - a["beta1"]))
        v.mul_(a["beta2"]).add_(g.square().mul_(1 - a["beta2"]))
        r = v.sqrt()
    else:  # which neighbour a value is rounded to is decided in 64 bits
        wide = lambda n: (s[n + "_codes"].view(torch.float8_e4m3fn).double().view(-1, SCALE_BLOCK) * s[n + "_scale"].double()[:, None]).view(-1)  # noqa: E731
        gd = g.double()
        m = wide("m").mul_(a["beta1"]).add_(gd * (1 - a["beta1"]))
        r = wide("r").square_().mul_(a["beta2"]).add_(gd.square_().mul_(1 - a["beta2"])).sqrt_()
        bits = _mixed(s["seed"] + t, p.numel())
        for name, val, u in (("m", m, bits & 0xFFFF), ("r", r, bits >> 16)):
            codes, scale = _to_codes(val, u.double() / 65536, name == "r")
            s[name + "_codes"].copy_(codes)
            s[name + "_scale"].copy_(scale)
        m, r = m.float(), r.float()
    p[:nd].mul_(1 - a["lr"] * a["weight_decay"])
    p.sub_(m.mul(size).div_(r.mul_(root).add_(a["eps"])))
    s["copy"].copy_(p)
    s["step"] += 1
    return _adamw_outputs(s)


# ---- the definitions in 64 bits, written apart -----------------------------------------------------------------------
def exact(case, seed):
    c = _full(case)
    s = prepare(case, seed)
    if c["kind"] == "adamw":
        return _adamw_exact(c, s)
    if c["kind"].startswith("norm"):
        return _norm_exact(c, s)
    return _attn_exact(c, s)


def _attn_exact(c, s):
    """Item by item and head by head, gradients by differentiating the probabilities."""
    B, H, Hkv, D, U, T = (c[k] for k in ("B", "H", "Hkv", "D", "U", "T"))
    f64 = torch.float64
    bwd = c["kind"] == "attn_bwd"
    o = torch.zeros(B, H, D, U, dtype=f64, device="cuda")
    lse = torch.full((B, H, U), -math.inf, dtype=f64, device="cuda")
    dq, dk, dv = torch.zeros_like(o), *(torch.zeros(B, Hkv, D, T, dtype=f64, device="cuda") for _ in range(2))
    frames, tokens = torch.arange(T, device="cuda"), torch.arange(U, device="cuda")
    for b in range(B):
        lo, hi = torch.zeros(U, device="cuda", dtype=torch.int64), torch.full((U,), T, device="cuda", dtype=torch.int64)
        if s["windows"] is not None:
            lo, hi = s["windows"][b, :, 0].long(), s["windows"][b, :, 1].long()
        if s["lengths"] is not None:
            hi = torch.minimum(hi, s["lengths"][b].long())
            hi = torch.where(tokens < s["q_lengths"][b], hi, 0)
        out = (frames[None] < lo[:, None]) | (frames[None] >= hi[:, None])       # [U, T]
        some = ~out.all(1)
        q = s["q"][b].to(f64).view(H, D, U)
        k, v = (s[x][b].to(f64).reshape(Hkv, D, T).repeat_interleave(H // Hkv, 0) for x in ("k", "v"))
        z = torch.matmul(q.transpose(1, 2).contiguous(), k) * s["scale"]        # [H, U, T]
        z[:, out] = -math.inf
        z[:, ~some] = 0.0
        l = torch.logsumexp(z, 2)
        p = torch.exp(z - l[..., None]) * some[None, :, None]
        if not bwd:
            lse[b] = torch.where(some[None], l, -math.inf)
            o[b] = torch.matmul(v, p.transpose(1, 2).contiguous())
            continue
        do = s["do"][b].to(f64).view(H, D, U)
        dv[b] = torch.matmul(do, p).view(Hkv, -1, D, T).sum(1)
        dp = torch.matmul(do.transpose(1, 2).contiguous(), v)
        ds = (p * dp - p * (p * dp).sum(2, keepdim=True)) * s["scale"]
        dk[b] = torch.matmul(q, ds).view(Hkv, -1, D, T).sum(1)
        dq[b] = torch.matmul(k, ds.transpose(1, 2).contiguous())
    if bwd:
        return dq.view(B, H * D, U), dk.view(B, Hkv * D, T), dv.view(B, Hkv * D, T)
    return o.view(B, H * D, U), lse


def _norm_exact(c, s):
    """Utterance by utterance, on its valid positions alone, as [positions, channels]; gradients by torch's differentiation of
    elementary operations."""
    B, C, T = c["B"], c["C"], c["T"]
    f64 = torch.float64
    bwd = c["kind"] == "norm_bwd"
    par = {k: s[k].to(f64).requires_grad_(bwd) for k in ("rscale", "post_weight", "post_bias", "next_weight", "next_bias") if s[k] is not None}
    gate = None if s["gate"] is None else s["gate"].to(f64).requires_grad_(bwd)

    def norm(z, w, b):
        z = z - z.mean(1, keepdim=True) if c["layer"] else z
        z = z / (z.pow(2).mean(1, keepdim=True) + EPS).sqrt() * par[w]
        return z + par[b] if b in par else z

    out = {k: torch.zeros(B, C, T, dtype=f64, device="cuda") for k in (("dx", "df") if bwd else ("y", "n"))}
    for b in range(B):
        n = T if s["lengths"] is None else int(s["lengths"][b])
        f = s["f"][b, :, :n].t().to(f64).requires_grad_(bwd)
        g = 1.0 if gate is None else gate[b] if gate.dim() == 2 else gate[b, :, :n].t()
        if not bwd:
            y = s["x"][b, :, :n].t().to(f64) + par["rscale"] * g * norm(f, "post_weight", "post_bias")
            out["y"][b, :, :n] = y.t()
            out["n"][b, :, :n] = norm(y.to(s["x"].dtype).to(f64), "next_weight", "next_bias").t()
            continue
        y = s["y"][b, :, :n].t().to(f64).requires_grad_()
        dn, dy = (s[k][b, :, :n].t().to(f64) for k in ("dn", "dy"))
        (norm(y, "next_weight", "next_bias") * dn).sum().backward()
        dx = dy + y.grad
        (par["rscale"] * g * norm(f, "post_weight", "post_bias") * dx).sum().backward()
        out["dx"][b, :, :n], out["df"][b, :, :n] = dx.t(), f.grad.t()
    if not bwd:
        return out["y"], out["n"]
    out.update({"d" + k: (par[k].grad if k in par else None) for k in ("rscale", "post_weight", "post_bias", "next_weight", "next_bias")})
    out["dgate"] = None if gate is None else gate.grad
    return out


def _adamw_exact(c, s):
    """In runs of blocks, every step of the definition in 64 bits."""
    f64 = torch.float64
    lr, b1, b2, eps, wd = (ADAMW[k] for k in ("lr", "beta1", "beta2", "eps", "weight_decay"))
    t, n, run_of = s["step"], s["param"].numel(), 1 << 25
    names = ("m", "v") if c["bits"] == 32 else ("m", "r")
    got = {k: torch.empty(n, dtype=f64, device="cuda") for k in ("param",) + names}
    for at in range(0, n, run_of):
        to = min(n, at + run_of)
        cut, blocks = slice(at, to), slice(at // SCALE_BLOCK, to // SCALE_BLOCK)
        p, g = s["param"][cut].to(f64), s["grad"][cut].to(f64)
        if c["bits"] == 32:
            m, v = s["m"][cut].to(f64), s["v"][cut].to(f64)
        else:
            m, v = (s[k + "_codes"][cut].view(torch.float8_e4m3fn).to(f64) * s[k + "_scale"][blocks].to(f64).repeat_interleave(SCALE_BLOCK)
                    for k in names)
            v = v ** 2
        m = b1 * m + (1 - b1) * g
        v = b2 * v + (1 - b2) * g * g
        decay = torch.where(torch.arange(at, to, device="cuda") < s["decayed"], 1 - lr * wd, 1.0)
        got["param"][cut] = p * decay - lr * (m / (1 - b1 ** t)) / ((v / (1 - b2 ** t)).sqrt() + eps)
        if c["bits"] == 32:
            got["m"][cut], got["v"][cut] = m, v
            continue
        h = (torch.arange(at, to, device="cuda") * 0x9E3779B9) % 2 ** 32
        h = h ^ ((s["seed"] + t) % 2 ** 32)
        h = (((h >> 16) ^ h) * 0x6A09E667) % 2 ** 32
        h = (((h >> 13) ^ h) * 0xBB67AE85) % 2 ** 32
        h = (h >> 16) ^ h
        for k, x, u in (("m", m, h % 65536), ("r", v.sqrt(), h // 65536)):
            sc = x.abs().view(-1, SCALE_BLOCK).max(1).values / E4M3_MAX
            sc = torch.where(sc > 0, sc.float().clamp_min(2.0 ** -126).to(f64), 1.0).repeat_interleave(SCALE_BLOCK)
            z = x.abs() / sc
            step = 2.0 ** (torch.floor(torch.log2(z.clamp_min(2.0 ** -6))) - 3)
            q = torch.floor(z / step + u.to(f64) / 65536) * step
            q = q.clamp(max=E4M3_MAX)
            if k == "r":
                q = torch.where((x > 0) & (q == 0), 2.0 ** -9, q)
            got[k][cut] = q * x.sign() * sc
    got["copy"] = got["param"]
    if c["bits"] == 8:
        got["m"], got["r"] = got["m"].view(-1, SCALE_BLOCK), got["r"].view(-1, SCALE_BLOCK)
    return got


# ---- what a pass cannot do without --------------------------------------------------------------------------------
def work(case):
    """Bytes (each input read once, each output written once) and operations of one pass; padded batches are taken to be three
    quarters full, which is what their lengths average to."""
    c = _full(case)
    e = 4 if c["dtype"] == "f32" else 2
    part = 0.75 if c["lengths"] else 1.0
    if c["kind"] == "adamw":
        n = sum(sum(v) for v in _encoder_tensors(c["width"], c.get("tail", 0)))
        # parameter in and out, gradient in, bfloat16 copy out; both states in and out
        return {"bytes": n * (4 + 4 + 4 + 2 + (16 if c["bits"] == 32 else 4 + 16 / SCALE_BLOCK)), "flops": 14 * n}
    if c["kind"].startswith("norm"):
        n = c["B"] * c["C"] * c["T"]
        gate = n if c["gate"] == "element" else 0
        if c["kind"] == "norm_fwd":  # x, f in; y, n out
            return {"bytes": e * ((2 * n + gate) * part + 2 * n), "flops": 14 * n * part}
        # dy, dn, y, f in; dx, df out
        return {"bytes": e * ((4 * n + gate) * part + 2 * n + gate), "flops": 40 * n * part}
    B, H, Hkv, D, U, T = (c[k] for k in ("B", "H", "Hkv", "D", "U", "T"))
    q, kv, lse = B * H * D * U, B * Hkv * D * T, 4 * B * H * U
    frames = T * part
    if c["windows"]:
        frames = min(frames, T * 0.24)  # a quarter of the utterance, less at its ends
    if c["kind"] == "attn_fwd":
        return {"bytes": e * (q * (part + 1) + 2 * kv * part) + lse, "flops": 4 * B * H * U * part * frames * D}
    return {"bytes": e * (q * (3 * part + 1) + 2 * kv * (part + 1)) + lse, "flops": 10 * B * H * U * part * frames * D}
