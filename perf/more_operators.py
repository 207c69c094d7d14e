"""The workloads on which the operators that take a token through an attention decoder are timed and checked: the lookup of its
embedding, the norms and the rotation of its queries and keys, attention over a paged cache, the scoring of the tokens that follow.

A case is a dict of plain values.  Its "kind" says which call one pass makes:

  embed_fwd    columns of a table for token numbers, times a scale: [batch][channels][tokens]
  embed_bwd    the table's gradient
  heads_fwd    RMS norm of every head of the queries and keys and their rotation by position
  heads_bwd    its backward pass, gradients of the norms' weights included
  heads_cache  the serving form: queries come back, keys and values go into the pages of a cache
  paged        attention of U new tokens per sequence to what the cache holds (U = 1: a decoding step)
  scores_fwd   log-probabilities of given tokens, entropies, the likeliest alternatives
  scores_bwd   the gradient with respect to the scores

Activations are channel-major, [batch][channels][tokens], like the encoder's; heads lie side by side in the channels.  Pages hold keys as
[kv head][row][channel] and values as [kv head][channel][row].  Sizes: the encoder's channel counts (256 to 1024) in heads of 64, 80, 96 and
128; its decoder's 29 symbols and vocabularies of word pieces; batches of 32 transcripts, transcripts of long recordings, single tokens.
"lengths" makes a padded batch; token numbers are distributed as words are, the few frequent ones taking most places.
"""
import math

import torch

own = False  # set from outside: False computes the operators in their plain form, True calls the library

EPS = 1e-5
BASE = 10000.0  # of the rotation's frequencies

DEFAULTS = {"dtype": "bf16", "lengths": False, "norm": True, "pairs": False, "far": False, "rot": 0, "window": 0, "top": 0, "barred": False,
            "entropy": False, "grad": "same"}


def listed():
    return [
        # a decoding step of a serving batch: the smallest call, launches and latency count
        {"name": "embed_step", "kind": "embed_fwd", "B": 32, "U": 1, "V": 5000, "C": 1024},
        # a training step's transcripts: the gradient over a padded batch
        {"name": "embed_bwd_train", "kind": "embed_bwd", "B": 32, "U": 150, "V": 5000, "C": 1024, "lengths": True},
        # transcripts of long recordings, of no particular length, a large vocabulary
        {"name": "embed_bwd_long", "kind": "embed_bwd", "B": 16, "U": 1601, "V": 32000, "C": 512},
        # queries and shared keys of a training step's batch
        {"name": "heads_fwd_train", "kind": "heads_fwd", "B": 32, "U": 150, "H": 16, "Hkv": 4, "D": 64, "rot": 64, "lengths": True},
        # the backward pass on long transcripts, wide heads, far into a recording
        {"name": "heads_bwd_long", "kind": "heads_bwd", "B": 4, "U": 1333, "H": 8, "Hkv": 2, "D": 128, "rot": 128, "far": True},
        # a decoding step of a serving batch, into the cache
        {"name": "heads_cache_step", "kind": "heads_cache", "B": 32, "U": 1, "T": 500, "page": 64, "H": 16, "Hkv": 4, "D": 64, "rot": 64},
        # one sequence, one token
        {"name": "paged_step_b1", "kind": "paged", "B": 1, "U": 1, "T": 2000, "page": 64, "H": 16, "Hkv": 4, "D": 64},
        # a serving batch of long sequences of different lengths, one token each
        {"name": "paged_step_b32", "kind": "paged", "B": 32, "U": 1, "T": 8001, "page": 64, "H": 16, "Hkv": 2, "D": 128, "lengths": True},
        # chunks of prompts behind what is cached already
        {"name": "paged_chunk", "kind": "paged", "B": 4, "U": 500, "T": 6000, "page": 128, "H": 8, "Hkv": 2, "D": 128, "lengths": True},
        # a decoding step over a large vocabulary with alternatives for a beam search
        {"name": "scores_step", "kind": "scores_fwd", "B": 16, "U": 1, "V": 32000, "top": 8, "dtype": "f32"},
        # scoring a training step's batch
        {"name": "scores_fwd_train", "kind": "scores_fwd", "B": 32, "U": 150, "V": 5000, "top": 4, "lengths": True},
        # the loss's gradient with an entropy term, float32 scores to a bfloat16 gradient, odd length
        {"name": "scores_bwd_train", "kind": "scores_bwd", "B": 16, "U": 333, "V": 5000, "dtype": "f32", "grad": "bf16", "entropy": True},
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of these ranges, no costlier than the largest above."""
    kind = rng.choice(["embed_fwd", "embed_bwd", "embed_bwd", "heads_fwd", "heads_bwd", "heads_cache", "step", "chunk", "scores_fwd", "scores_fwd",
                       "scores_bwd"])

    def odd(n):  # half of the lengths as they come, half in whole groups
        return n if n < 16 or rng.random() < 0.5 else n // 8 * 8

    c = {"kind": kind, "dtype": "f32" if rng.random() < 0.25 else "bf16", "lengths": rng.random() < 0.5}
    if kind.startswith("embed"):
        c.update(V=_log_uniform(rng, 29, 32000), C=rng.choice([256, 384, 512, 640, 768, 896, 1024]), B=_log_uniform(rng, 1, 32))
        return dict(c, U=1 if kind == "embed_fwd" and rng.random() < 0.3 else odd(_log_uniform(rng, 2, min(800, 12000 // c["B"]))))
    if kind.startswith("scores"):
        c.update(V=_log_uniform(rng, 29, 32000), B=_log_uniform(rng, 1, 32), barred=rng.random() < 0.3)
        most = max(1, min(800, 24000000 // (c["V"] * c["B"])))
        c["U"] = 1 if rng.random() < 0.3 else odd(_log_uniform(rng, 1, most))
        if kind == "scores_fwd":
            return dict(c, top=rng.choice([0, 1, 4, 5, 8, 16]))
        return dict(c, entropy=rng.random() < 0.5, grad=rng.choice(["same", "bf16"]))
    d = rng.choice([64, 64, 80, 96, 128])
    h = {64: rng.choice([4, 8, 12, 16]), 80: 8, 96: 8, 128: rng.choice([4, 8])}[d]
    c.update(H=h, Hkv=rng.choice([h, h // 2, h // 4]), D=d)
    if kind.startswith("heads"):
        c.update(rot=rng.choice([d, d, d // 2, 0]), pairs=rng.random() < 0.5, norm=rng.random() < 0.75)
        if not c["norm"] and not c["rot"]:
            c["rot"] = d
        if kind == "heads_cache":
            u = rng.choice([1, 1, 1, 4, _log_uniform(rng, 2, 300)])
            return dict(c, B=_log_uniform(rng, 1, 32 if u < 8 else 4), U=u, T=u + _log_uniform(rng, 10, 500), page=rng.choice([16, 32, 64, 128]))
        b = _log_uniform(rng, 1, 32)
        return dict(c, B=b, U=odd(_log_uniform(rng, 10, min(1333, 4800 // b))), far=rng.random() < 0.3)
    c.update(kind="paged", page=rng.choice([16, 32, 64, 128, 256]), window=rng.choice([0, 0, 0, 300]))
    if kind == "step":
        b = _log_uniform(rng, 1, 32)
        u = rng.choice([1, 1, 1, 2, 5, 8])
        most = 180000000 // (4 * b * c["Hkv"] * d * (2 if c["dtype"] == "f32" else 1))  # rows, by the bytes that a pass reads
        return dict(c, B=b, U=u, T=u + _log_uniform(rng, 50, min(8000, most)))
    u = odd(_log_uniform(rng, 10, 400))
    if c["dtype"] == "f32":
        u = min(u, 100)
    return dict(c, B=_log_uniform(rng, 1, 4), U=u, T=u + odd(_log_uniform(rng, 50, 4000)))


# ---- inputs -----------------------------------------------------------------------------------------------------
def _full(case):
    return dict(DEFAULTS, **case)


def _storage(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _lengths(g, b, n):
    """b lengths between half of n and n, the longest of them n; int32."""
    ln = torch.randint((n + 1) // 2, n + 1, (b,), device="cuda", generator=g, dtype=torch.int32)
    ln[torch.randint(0, b, (1,), device="cuda", generator=g)] = n
    return ln


def _tokens(c, g):
    """Token numbers [B, U]: the n-th most frequent one as often as 1/n says, numbers in no order of frequency."""
    u = torch.rand(c["B"], c["U"], device="cuda", generator=g, dtype=torch.float64)
    rank = ((c["V"] + 1.0) ** u).floor().long().sub_(1).clamp_(0, c["V"] - 1)
    return torch.randperm(c["V"], device="cuda", generator=g)[rank]


def _embed_inputs(c, g, dt):
    s = {"ids": _tokens(c, g), "V": c["V"], "scale": c["C"] ** 0.5}
    s["lengths"] = _lengths(g, c["B"], c["U"]) if c["lengths"] else None
    if c["kind"] == "embed_fwd":
        s["table"] = (torch.randn(c["V"], c["C"], device="cuda", generator=g) * c["C"] ** -0.5).to(dt)
    else:
        s["dout"] = torch.randn(c["B"], c["C"], c["U"], device="cuda", generator=g).to(dt)
    return s


def _pages(c, g, dt, filled):
    """A cache whose sequences lie on pages in no order, some pages of it in other hands; -1 in the table where a sequence has no page."""
    B, T, P = c["B"], c["T"], c["page"]
    n = -(-T // P)
    pages = B * n + 3
    table = torch.randperm(pages, device="cuda", generator=g)[:B * n].view(B, n).to(torch.int32)
    used = torch.arange(n, device="cuda")[None] * P < filled[:, None]
    return {"page_table": torch.where(used, table, -1).contiguous(), "P": P,
            "k_cache": torch.randn(pages, c["Hkv"], P, c["D"], device="cuda", generator=g).to(dt),
            "v_cache": torch.randn(pages, c["Hkv"], c["D"], P, device="cuda", generator=g).to(dt)}


def _sequences(c, g):
    """Tokens that each sequence has, the new ones among them (T at most), and how many are new (U at most)."""
    if not c["lengths"]:
        return torch.full((c["B"],), c["T"], device="cuda", dtype=torch.int32), None
    return _lengths(g, c["B"], c["T"] - c["U"]) + c["U"], _lengths(g, c["B"], c["U"]) if c["U"] > 8 else None


def _heads_inputs(c, g, dt):
    B, U, H, Hkv, D = (c[k] for k in ("B", "U", "H", "Hkv", "D"))
    s = {"heads": H, "kv_heads": Hkv, "norm": c["norm"], "pairs": c["pairs"], "positions": None, "lengths": None, "freqs": None}
    gain = torch.exp(0.3 * torch.randn(B, H + 2 * Hkv, 1, 1, device="cuda", generator=g))
    qkv = (gain * torch.randn(B, H + 2 * Hkv, D, U, device="cuda", generator=g)).to(dt).view(B, -1, U)  # one projection's output
    for name in ("q_weight", "k_weight"):
        s[name] = 1 + 0.2 * torch.randn(D, device="cuda", generator=g) if c["norm"] else None
    if c["rot"]:
        s["freqs"] = BASE ** (-torch.arange(0, c["rot"], 2, device="cuda", dtype=torch.float64) / c["rot"])
    if c["kind"] == "heads_cache":
        s["x"] = qkv
        s["lengths"], s["q_lengths"] = _sequences(c, g)
        s.update(_pages(c, g, dt, s["lengths"]))
        return s
    s["x"] = qkv[:, :(H + Hkv) * D]
    if c["far"]:  # every item somewhere in a recording of hours
        first = torch.randint(0, 500000, (B, 1), device="cuda", generator=g)
        s["positions"] = (first + torch.arange(U, device="cuda")[None]).to(torch.int32)
    s["lengths"] = _lengths(g, B, U) if c["lengths"] else None
    if c["kind"] == "heads_bwd":
        s["dout"] = torch.randn(B, (H + Hkv) * D, U, device="cuda", generator=g).to(dt)
    return s


def _paged_inputs(c, g, dt):
    s = {"heads": c["H"], "kv_heads": c["Hkv"], "scale": c["D"] ** -0.5, "window": c["window"]}
    s["q"] = (1.5 * torch.randn(c["B"], c["H"] * c["D"], c["U"], device="cuda", generator=g)).to(dt)
    s["lengths"], s["q_lengths"] = _sequences(c, g)
    s.update(_pages(c, g, dt, s["lengths"]))
    return s


def _scores_inputs(c, g, dt):
    B, V, U = c["B"], c["V"], c["U"]
    s = {"top": c["top"], "targets": _tokens(c, g), "lengths": _lengths(g, B, U) if c["lengths"] else None}
    s["scores"] = (2.5 * torch.randn(B, V, U, device="cuda", generator=g)).to(dt)
    if c["barred"]:  # classes that a rule does not allow here
        s["scores"][:, 3::8] = -math.inf
        s["targets"] -= (s["targets"] % 8 == 3).long()
    if c["kind"] == "scores_bwd":
        out = _scores_fwd(s)
        s["lse"], s["entropy"] = out["lse"], out["entropy"]
        s["dlogp"] = -torch.rand(B, U, device="cuda", generator=g) - 0.5
        s["dentropy"] = 0.1 * torch.randn(B, U, device="cuda", generator=g) if c["entropy"] else None
        s["grad_dtype"] = torch.bfloat16 if c["grad"] == "bf16" else dt
    return s


def prepare(case, seed):
    c = _full(case)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    make = {"embed": _embed_inputs, "heads": _heads_inputs, "paged": _paged_inputs, "scores": _scores_inputs}[c["kind"].split("_")[0]]
    return dict(make(c, g, _storage(c)), kind=c["kind"])


# ---- one pass ---------------------------------------------------------------------------------------------------
def run(s):
    kind = s["kind"]
    if own:
        from paper_1909_09577_amd import binding as nm
        return _own(nm, kind, s)
    return {"embed_fwd": _embed_fwd, "embed_bwd": _embed_bwd, "heads_fwd": _heads_fwd, "heads_bwd": _heads_bwd, "heads_cache": _heads_cache,
            "paged": _paged, "scores_fwd": _scores_fwd, "scores_bwd": _scores_bwd}[kind](s)


def _own(nm, kind, s):
    if kind == "embed_fwd":
        return nm.nm_embedding_fwd(s["ids"], s["table"], scale=s["scale"], lengths=s["lengths"])
    if kind == "embed_bwd":
        return nm.nm_embedding_bwd(s["dout"], s["ids"], s["V"], scale=s["scale"], lengths=s["lengths"])
    if kind == "scores_fwd":
        return nm.nm_token_scores_fwd(s["scores"], s["targets"], top=s["top"], lengths=s["lengths"])
    if kind == "scores_bwd":
        return nm.nm_token_scores_bwd(s["scores"], s["targets"], s["lse"], s["entropy"], s["dlogp"], s["dentropy"], lengths=s["lengths"],
                                      dtype=s["grad_dtype"])
    kw = {k: s[k] for k in ("heads", "kv_heads")}
    if kind == "paged":
        return nm.nm_paged_attn_fwd(s["q"], s["k_cache"], s["v_cache"], s["page_table"], s["lengths"], q_lengths=s["q_lengths"], scale=s["scale"],
                                    window=s["window"], want_lse=True, **kw)
    kw.update({k: s[k] for k in ("norm", "pairs", "q_weight", "k_weight", "freqs")}, eps=EPS)
    if kind == "heads_fwd":
        return nm.nm_head_norm_fwd(s["x"], positions=s["positions"], lengths=s["lengths"], **kw)
    if kind == "heads_bwd":
        return nm.nm_head_norm_bwd(s["dout"], s["x"], positions=s["positions"], lengths=s["lengths"], **kw)
    q = nm.nm_head_norm_cache(s["x"], s["k_cache"], s["v_cache"], s["page_table"], s["lengths"], q_lengths=s["q_lengths"], **kw)
    return q, s["k_cache"], s["v_cache"]


# ---- the plain forms ----------------------------------------------------------------------------------------------
def _valid(lengths, n):
    """[B, n] truth values of the places inside an item; None: all are."""
    return None if lengths is None else torch.arange(n, device="cuda")[None] < lengths[:, None]


def _embed_fwd(s):
    out = s["table"][s["ids"]].float().mul_(s["scale"])  # [B, U, C]
    ok = _valid(s["lengths"], s["ids"].shape[1])
    if ok is not None:
        out = out.masked_fill_(~ok[..., None], 0.0)
    return out.transpose(1, 2).to(s["table"].dtype).contiguous()


def _embed_bwd(s):
    B, C, U = s["dout"].shape
    rows = s["dout"].float().transpose(1, 2)
    ok = _valid(s["lengths"], U)
    if ok is not None:
        rows = rows.masked_fill(~ok[..., None], 0.0)
    out = torch.zeros(s["V"], C, device="cuda")
    return out.index_add_(0, s["ids"].reshape(-1), rows.reshape(-1, C)).mul_(s["scale"])


def _weights(s):
    """[H + Hkv, D, 1] of the queries' and the keys' norms, or 1."""
    if s["q_weight"] is None:
        return 1.0
    both = torch.stack([s["q_weight"], s["k_weight"]])
    return both.repeat_interleave(torch.tensor([s["heads"], s["kv_heads"]], device="cuda"), 0, output_size=s["heads"] + s["kv_heads"])[..., None]


def _turned(x, s, positions, back=False):
    """x [B, heads, D, U] with its first channels turned by their angles, which are made in float64; positions [B or 1, U]."""
    if s["freqs"] is None:
        return x
    angle = positions[:, None, None, :].double() * s["freqs"][:, None]
    cos, sin = angle.cos().float(), angle.sin().float()
    if back:
        sin = -sin
    half = s["freqs"].numel()
    out = x.clone()
    one, two = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if s["pairs"] else (slice(0, half), slice(half, 2 * half))
    a, b = x[:, :, one], x[:, :, two]
    out[:, :, one], out[:, :, two] = a * cos - b * sin, b * cos + a * sin
    return out


def _places(s, B, U):
    return torch.arange(U, device="cuda")[None] if s["positions"] is None else s["positions"]


def _normed(x, s):
    """(x over its rms, 1/rms) of x [B, heads, D, U]."""
    r = (x.square().mean(2, keepdim=True) + EPS).rsqrt()
    return x * r, r


def _heads_fwd(s):
    B, HD, U = s["x"].shape
    x = s["x"].float().reshape(B, s["heads"] + s["kv_heads"], -1, U)
    if s["norm"]:
        x = _normed(x, s)[0] * _weights(s)
    out = _turned(x, s, _places(s, B, U))
    ok = _valid(s["lengths"], U)
    if ok is not None:
        out = torch.where(ok[:, None, None], out, 0.0)
    return out.reshape(B, HD, U).to(s["x"].dtype)


def _heads_bwd(s):
    B, HD, U = s["x"].shape
    H = s["heads"]
    split = lambda t: t.float().reshape(B, H + s["kv_heads"], -1, U)  # noqa: E731
    d = split(s["dout"])
    ok = _valid(s["lengths"], U)
    if ok is not None:
        d = torch.where(ok[:, None, None], d, 0.0)
    d = _turned(d, s, _places(s, B, U), back=True)
    dq_weight = dk_weight = None
    if s["norm"]:
        hat, r = _normed(split(s["x"]), s)
        dw = (d * hat).double().sum((0, 3)).float()
        dq_weight, dk_weight = dw[:H].sum(0), dw[H:].sum(0)
        d = d * _weights(s)
        d = (d - hat * (d * hat).mean(2, keepdim=True)) * r
        if ok is not None:
            d = torch.where(ok[:, None, None], d, 0.0)
    return d.reshape(B, HD, U).to(s["x"].dtype), dq_weight, dk_weight


def _at(s, U):
    """([B, U] positions of the new tokens, which of them there are)."""
    n = torch.full_like(s["lengths"], U) if s["q_lengths"] is None else s["q_lengths"]
    u = torch.arange(U, device="cuda")[None]
    return (s["lengths"] - n)[:, None] + u, u < n[:, None]


def _heads_cache(s):
    B, _, U = s["x"].shape
    H, Hkv, P = s["heads"], s["kv_heads"], s["P"]
    x = s["x"].float().reshape(B, H + 2 * Hkv, -1, U)
    at, there = _at(s, U)
    qk = x[:, :H + Hkv]
    if s["norm"]:
        qk = _normed(qk, s)[0] * _weights(s)
    qk = _turned(qk, s, at).to(s["x"].dtype)
    qk = torch.where(there[:, None, None], qk, 0.0)
    page = s["page_table"].gather(1, at.clamp_min(0).long() // P).long()
    row = at.long() % P
    k, v = qk[:, H:].permute(0, 3, 1, 2), s["x"].reshape(B, H + 2 * Hkv, -1, U)[:, H + Hkv:].permute(0, 3, 1, 2)  # [B, U, Hkv, D]
    if s["q_lengths"] is not None:
        page, row, k, v = page[there], row[there], k[there], v[there]
    s["k_cache"][page, :, row] = k
    s["v_cache"][page, :, :, row] = v
    return qk[:, :H].reshape(B, -1, U), s["k_cache"], s["v_cache"]


def _paged(s):
    B, HD, U = s["q"].shape
    H, Hkv, P = s["heads"], s["kv_heads"], s["P"]
    D, G = HD // H, H // Hkv
    table = s["page_table"].long()
    n = table.shape[1]
    T = n * P
    k = s["k_cache"][table.clamp_min(0)].transpose(1, 2).reshape(B * Hkv, T, D).float()
    v = s["v_cache"][table.clamp_min(0)].permute(0, 2, 1, 4, 3).reshape(B * Hkv, T, D).float()
    q = s["q"].float().reshape(B * Hkv, G, D, U).transpose(2, 3).reshape(B * Hkv, G * U, D)
    sc = torch.bmm(q, k.transpose(1, 2).contiguous()).mul_(s["scale"]).view(B, Hkv, G, U, T)
    at, there = _at(s, U)
    pos = torch.arange(T, device="cuda")
    ok = there[..., None] & (pos <= at[..., None]) & (table >= 0).repeat_interleave(P, 1)[:, None]
    if s["window"]:
        ok &= pos > at[..., None] - s["window"]
    sc.masked_fill_(~ok[:, None, None], -math.inf)
    top = sc.amax(-1, keepdim=True)
    top = torch.where(top > -math.inf, top, 0.0)
    p = sc.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    p = p.div_(torch.where(total > 0, total, 1.0)).view(B * Hkv, G * U, T)
    o = torch.bmm(p, v).view(B, H, U, D).transpose(2, 3).reshape(B, HD, U)
    return o.to(s["q"].dtype), (top + total.log()).reshape(B, H, U)


def _scores_fwd(s):
    z = s["scores"].float()
    B, V, U = z.shape
    top = z.amax(1, keepdim=True)
    e = (z - top).exp_()
    total = e.sum(1, keepdim=True)
    lse = top + total.log()
    entropy = total.log() - (e * (z - top).clamp_min_(-1e30)).sum(1, keepdim=True) / total  # (zero times what is barred is zero)
    out = {"lse": lse[:, 0], "entropy": entropy[:, 0], "logp": (z.gather(1, s["targets"][:, None]) - lse)[:, 0]}
    if s["top"]:
        best, ids = z.sort(dim=1, descending=True, stable=True)
        out["top_logp"], out["top_ids"] = best[:, :s["top"]] - lse, ids[:, :s["top"]].to(torch.int32)
    ok = _valid(s["lengths"], U)
    if ok is not None:
        out = {k: v.masked_fill(~(ok if v.dim() == 2 else ok[:, None]), -1 if k == "top_ids" else 0) for k, v in out.items()}
    return {k: v.contiguous() for k, v in out.items()}


def _scores_bwd(s):
    z = s["scores"].float()
    logp = z - s["lse"][:, None]
    p = logp.exp()
    out = p * -s["dlogp"][:, None]
    out.scatter_add_(1, s["targets"][:, None], s["dlogp"][:, None])
    if s["dentropy"] is not None:
        out -= s["dentropy"][:, None] * p * (logp.clamp_min_(-1e30) + s["entropy"][:, None])
    ok = _valid(s["lengths"], z.shape[2])
    if ok is not None:
        out.masked_fill_(~ok[:, None], 0.0)
    return out.to(s["grad_dtype"])


# ---- the definitions in 64 bits, written apart -----------------------------------------------------------------------
def exact(case, seed):
    c = _full(case)
    s = prepare(case, seed)
    return {"embed": _embed_exact, "heads": _heads_exact, "paged": _paged_exact, "scores": _scores_exact}[c["kind"].split("_")[0]](c, s)


def _embed_exact(c, s):
    """Item by item; the gradient by differentiating the lookup."""
    B, U, V, C = c["B"], c["U"], c["V"], c["C"]
    fwd = c["kind"] == "embed_fwd"
    table = (s["table"].double() if fwd else torch.zeros(V, C, device="cuda", dtype=torch.float64)).requires_grad_(not fwd)
    out = torch.zeros(B, C, U, dtype=torch.float64, device="cuda")
    for b in range(B):
        n = U if s["lengths"] is None else int(s["lengths"][b])
        cols = table.t()[:, s["ids"][b, :n]] * s["scale"]
        if fwd:
            out[b, :, :n] = cols
        else:
            (cols * s["dout"][b, :, :n].double()).sum().backward()
    return out if fwd else table.grad


def _rotation(c, at):
    """[U, D, D] matrices that turn a head's channels at the positions `at`."""
    D, rot = c["D"], c["rot"]
    m = torch.eye(D, dtype=torch.float64, device="cuda").repeat(at.numel(), 1, 1)
    for i in range(rot // 2):
        angle = at.double() * BASE ** (-2.0 * i / rot)
        x, y = (2 * i, 2 * i + 1) if c["pairs"] else (i, i + rot // 2)
        m[:, x, x], m[:, y, y], m[:, x, y], m[:, y, x] = angle.cos(), angle.cos(), -angle.sin(), angle.sin()
    return m


def _heads_exact(c, s):
    """Item by item as [U, heads, D], the rotation as a matrix; gradients by torch's differentiation of elementary operations."""
    B, U, H, Hkv, D = (c[k] for k in ("B", "U", "H", "Hkv", "D"))
    f64 = torch.float64
    bwd, cache = c["kind"] == "heads_bwd", c["kind"] == "heads_cache"
    weights = [s[k].to(f64).requires_grad_(bwd) if c["norm"] else None for k in ("q_weight", "k_weight")]
    out = torch.zeros(B, (H + Hkv) * D, U, dtype=f64, device="cuda")
    kc, vc = (s["k_cache"].to(f64), s["v_cache"].to(f64)) if cache else (None, None)
    for b in range(B):
        n, first = U, 0
        if cache:
            n = U if s["q_lengths"] is None else int(s["q_lengths"][b])
            first = int(s["lengths"][b]) - n
        elif s["lengths"] is not None:
            n = int(s["lengths"][b])
        at = first + torch.arange(n, device="cuda") if s["positions"] is None else s["positions"][b, :n]
        x = s["x"][b, :(H + Hkv) * D, :n].to(f64).view(H + Hkv, D, n).permute(2, 0, 1).contiguous().requires_grad_(bwd)
        y = x
        if c["norm"]:
            y = x / (x.pow(2).sum(2, keepdim=True) / D + EPS).sqrt()
            y = torch.cat([y[:, :H] * weights[0], y[:, H:] * weights[1]], 1)
        y = torch.matmul(y, _rotation(c, at).transpose(1, 2).contiguous())
        if bwd:
            (y * s["dout"][b, :, :n].to(f64).view(H + Hkv, D, n).permute(2, 0, 1)).sum().backward()
            out[b, :, :n] = x.grad.permute(1, 2, 0).reshape(-1, n)
        else:
            out[b, :, :n] = y.permute(1, 2, 0).reshape(-1, n)
        for u in range(n if cache else 0):
            page, row = int(s["page_table"][b, (first + u) // c["page"]]), (first + u) % c["page"]
            kc[page, :, row] = y[u, H:]
            vc[page, :, :, row] = s["x"][b, (H + Hkv) * D:, u].to(f64).view(Hkv, D)
    if bwd:
        return (out, *(None if w is None else w.grad for w in weights))
    return (out[:, :H * D], kc, vc) if cache else out


def _paged_exact(c, s):
    """Item by item and head by head over the rows of the sequence alone."""
    B, U, H, Hkv, D, P = (c[k] for k in ("B", "U", "H", "Hkv", "D", "page"))
    f64 = torch.float64
    o = torch.zeros(B, H, D, U, dtype=f64, device="cuda")
    lse = torch.full((B, H, U), -math.inf, dtype=f64, device="cuda")
    for b in range(B):
        total = int(s["lengths"][b])
        n = U if s["q_lengths"] is None else int(s["q_lengths"][b])
        pages = s["page_table"][b, :-(-total // P)].long()
        k = s["k_cache"][pages].to(f64).permute(1, 0, 2, 3).reshape(Hkv, -1, D)[:, :total]
        v = s["v_cache"][pages].to(f64).permute(1, 2, 0, 3).reshape(Hkv, D, -1)[:, :, :total]
        q = s["q"][b].to(f64).view(H, D, U)[:, :, :n]
        at = total - n + torch.arange(n, device="cuda")
        pos = torch.arange(total, device="cuda")[None]
        out = pos > at[:, None]
        if c["window"]:
            out |= pos <= at[:, None] - c["window"]
        for h in range(H):
            z = torch.matmul(q[h].t().contiguous(), k[h // (H // Hkv)].t().contiguous()) * s["scale"]
            z = z.masked_fill(out, -math.inf)
            lse[b, h, :n] = torch.logsumexp(z, 1)
            o[b, h, :, :n] = torch.matmul(v[h // (H // Hkv)], torch.softmax(z, 1).t().contiguous())
    return o.view(B, H * D, U), lse


def _scores_exact(c, s):
    """Item by item on its valid places alone; the gradient by differentiating the sum that it is the gradient of."""
    B, V, U, k = c["B"], c["V"], c["U"], c["top"]
    f64 = torch.float64
    bwd = c["kind"] == "scores_bwd"
    out = {"logp": torch.zeros(B, U, dtype=f64, device="cuda")}
    for name in ("entropy", "lse"):
        out[name] = torch.zeros_like(out["logp"])
    if k:
        out["top_logp"], out["top_ids"] = torch.zeros(B, k, U, dtype=f64, device="cuda"), None
    grad = torch.zeros(B, V, U, dtype=f64, device="cuda") if bwd else None
    for b in range(B):
        n = U if s["lengths"] is None else int(s["lengths"][b])
        z = s["scores"][b, :, :n].to(f64).t().contiguous().requires_grad_(bwd)  # [n, V]
        barred = torch.isinf(z.detach())
        logp = torch.log_softmax(z, 1)
        safe = logp.masked_fill(barred, 0.0)
        entropy = -(safe.exp().masked_fill(barred, 0.0) * safe).sum(1)
        picked = logp.gather(1, s["targets"][b, :n, None])[:, 0]
        if bwd:
            total = (picked * s["dlogp"][b, :n].to(f64)).sum()
            if s["dentropy"] is not None:
                total = total + (entropy * s["dentropy"][b, :n].to(f64)).sum()
            total.backward()
            grad[b, :, :n] = z.grad.t()
            continue
        out["logp"][b, :n], out["entropy"][b, :n], out["lse"][b, :n] = picked, entropy, torch.logsumexp(z, 1)
        if k:
            out["top_logp"][b, :, :n] = torch.topk(logp, k, 1).values.t()
    return grad if bwd else out


# ---- what a pass cannot do without --------------------------------------------------------------------------------
def work(case):
    """Bytes (each input read once, each output written once) and operations of one pass; padded batches are taken to be three
    quarters full, which is what their lengths average to."""
    c = _full(case)
    e = 4 if c["dtype"] == "f32" else 2
    part = 0.75 if c["lengths"] and c["U"] > 1 else 1.0
    B, U = c["B"], c["U"]
    if c["kind"] == "embed_fwd":
        return {"bytes": e * c["C"] * (min(c["V"], B * U * part) + B * U) + 8 * B * U, "flops": B * U * c["C"] * part}
    if c["kind"] == "embed_bwd":
        return {"bytes": e * B * U * c["C"] * part + 4 * c["V"] * c["C"] + 8 * B * U, "flops": 2 * B * U * c["C"] * part}
    if c["kind"].startswith("scores"):
        n = B * c["V"] * U
        if c["kind"] == "scores_fwd":
            return {"bytes": e * n * part + B * U * (20 + 8 * c["top"]), "flops": 6 * n * part}
        return {"bytes": e * n * part + (2 if c["grad"] == "bf16" else e) * n + 24 * B * U, "flops": 8 * n * part}
    H, Hkv, D = c["H"], c["Hkv"], c["D"]
    n = B * (H + Hkv) * D * U
    if c["kind"] == "heads_fwd":
        return {"bytes": e * n * (part + 1), "flops": 10 * n * part}
    if c["kind"] == "heads_bwd":  # dout and x in, dx out
        return {"bytes": e * n * (2 * part + 1), "flops": 25 * n * part}
    part = 0.75 if c["lengths"] and U > 8 else 1.0
    if c["kind"] == "heads_cache":  # queries, keys, values in; queries, keys, values out
        return {"bytes": 2 * e * B * (H + 2 * Hkv) * D * U * part, "flops": 10 * n * part}
    T = (c["T"] - U) * (0.75 if c["lengths"] else 1.0) + U / 2  # a token's reach, on average
    rows = T + U / 2
    if c["window"]:
        T, rows = min(T, c["window"]), min(rows, c["window"] + U)
    return {"bytes": e * (B * H * D * U * (part + 1) + 2 * B * Hkv * D * rows) + 4 * B * H * U, "flops": 4 * B * H * D * U * part * T}
