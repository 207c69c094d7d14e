"""Plain float64 implementations of the attention decoder's operators (numpy, loops over items and heads), from the definitions in
include/nm_attention.h, nm_norm.h and nm_adamw.h.  Used by the tests only; shares no code with the library."""
from __future__ import annotations

import numpy as np

F = np.float64


# ---- cross attention ----------------------------------------------------------------------------------------------------
def allowed(B, U, T, lengths=None, q_lengths=None, windows=None):
    """[B, U, T] truth values: which states a token may look at."""
    ok = np.zeros((B, U, T), bool)
    for b in range(B):
        n = T if lengths is None else min(max(int(lengths[b]), 0), T)
        nu = U if q_lengths is None else min(max(int(q_lengths[b]), 0), U)
        for u in range(nu):
            lo, hi = 0, n
            if windows is not None:
                lo, hi = max(lo, int(windows[b, u, 0])), min(hi, int(windows[b, u, 1]))
            if lo < hi:
                ok[b, u, lo:hi] = True
    return ok


def _views(x, heads):
    B, HD, N = x.shape
    return np.asarray(x, F).reshape(B, heads, HD // heads, N)


def attn_fwd(q, k, v, heads, kv_heads, scale, ok):
    """(o, lse, p [B,H,U,T], sum_t p|v| of every output)."""
    B, HD, U = q.shape
    T, G = k.shape[2], heads // kv_heads
    q, k, v = _views(q, heads), _views(k, kv_heads), _views(v, kv_heads)
    o, mag = np.zeros(q.shape), np.zeros(q.shape)
    lse = np.full((B, heads, U), -np.inf)
    p = np.zeros((B, heads, U, T))
    for b in range(B):
        for h in range(heads):
            kk, vv = k[b, h // G], v[b, h // G]
            for u in range(U):
                at = np.flatnonzero(ok[b, u])
                if not len(at):
                    continue
                s = scale * (q[b, h, :, u] @ kk[:, at])
                top = s.max()
                e = np.exp(s - top)
                lse[b, h, u] = top + np.log(e.sum())
                p[b, h, u, at] = e / e.sum()
                o[b, h, :, u] = vv[:, at] @ p[b, h, u, at]
                mag[b, h, :, u] = np.abs(vv[:, at]) @ p[b, h, u, at]
    return o.reshape(B, HD, U), lse, p, mag.reshape(B, HD, U)


def attn_bwd(do, q, k, v, o, p, heads, kv_heads, scale):
    """(dq, dk, dv) and the sums of the magnitudes of their terms: {"dv": sum p|do|, "dk": ..., "dq": ..., "dk_parts": ..., "dq_parts": ...},
    where *_parts take p(|dp| + |delta|) in place of |ds|."""
    B, HD, U = q.shape
    T, G = k.shape[2], heads // kv_heads
    do_, q_, o_ = _views(do, heads), _views(q, heads), _views(o, heads)
    k_, v_ = _views(k, kv_heads), _views(v, kv_heads)
    dq, dk, dv = np.zeros(q_.shape), np.zeros(k_.shape), np.zeros(v_.shape)
    mag = {n: np.zeros(q_.shape if n.startswith("dq") else k_.shape) for n in ("dq", "dk", "dv", "dq_parts", "dk_parts")}
    for b in range(B):
        for h in range(heads):
            c = h // G
            pp = p[b, h]
            live = pp.sum(1) > 0
            kk, vv = np.where(np.isfinite(k_[b, c]), k_[b, c], 0), np.where(np.isfinite(v_[b, c]), v_[b, c], 0)
            g, qq, oo = (np.where(live, x[b, h], 0) for x in (do_, q_, o_))
            delta = (g * oo).sum(0)
            dp = g.T @ vv
            ds = pp * (dp - delta[:, None])
            parts = pp * (np.abs(g).T @ np.abs(vv) + np.abs(delta)[:, None])
            dv[b, c] += g @ pp
            dk[b, c] += scale * (qq @ ds)
            dq[b, h] = scale * (kk @ ds.T)
            s = abs(scale)
            mag["dv"][b, c] += np.abs(g) @ pp
            mag["dk"][b, c] += s * (np.abs(qq) @ np.abs(ds))
            mag["dq"][b, h] = s * (np.abs(kk) @ np.abs(ds).T)
            mag["dk_parts"][b, c] += s * (np.abs(qq) @ parts)
            mag["dq_parts"][b, h] = s * (np.abs(kk) @ parts.T)
    shape = {"dq": q.shape, "dk": k.shape, "dv": k.shape}
    return (dq.reshape(q.shape), dk.reshape(k.shape), dv.reshape(k.shape),
            {n: m.reshape(shape[n[:2]]) for n, m in mag.items()})


# ---- norms around a block ------------------------------------------------------------------------------------------------
def _norm(z, weight, bias, layer, eps):
    """z [C]: (normalised, 1/deviation, with weight and bias)."""
    zc = z - z.mean() if layer else z
    r = 1 / np.sqrt((zc * zc).mean() + eps)
    hat = zc * r
    return hat, r, hat * (1 if weight is None else weight) + (0 if bias is None else bias)


def _gate_at(gate, b, t):
    return 1.0 if gate is None else gate[b] if gate.ndim == 2 else gate[b, :, t]


def norm_fwd(x, f=None, gate=None, rscale=None, post=False, post_weight=None, post_bias=None, nxt=True, next_weight=None,
             next_bias=None, layer=False, eps=1e-5, lengths=None, store=lambda a: a):
    """(y unrounded, n of the stored y); store: rounding to the storage type."""
    B, C, T = x.shape
    y, n = np.zeros(x.shape), np.zeros(x.shape)
    for b in range(B):
        for t in range(T if lengths is None else min(max(int(lengths[b]), 0), T)):
            y[b, :, t] = x[b, :, t]
            if f is not None:
                h = _norm(f[b, :, t], post_weight, post_bias, layer, eps)[2] if post else f[b, :, t]
                y[b, :, t] += (1 if rscale is None else rscale) * _gate_at(gate, b, t) * h
            if nxt:
                n[b, :, t] = _norm(store(y[b, :, t]), next_weight, next_bias, layer, eps)[2]
    return y, n


def _norm_back(d, hat, r, weight, layer):
    dh = d * (1 if weight is None else weight)
    out = dh - hat * (dh * hat).mean()
    return r * (out - dh.mean() if layer else out)


def norm_bwd(dy, dn, y, f=None, gate=None, rscale=None, post=False, post_weight=None, post_bias=None, next_weight=None, layer=False,
             eps=1e-5, lengths=None):
    """Gradients, and under "abs_*" the sums of the magnitudes of the terms of every sum over time."""
    like = dn if dy is None else dy
    B, C, T = like.shape
    out = {k: np.zeros(like.shape) for k in ("dx", "df", "dgate_element")}
    vec = ("drscale", "dpost_weight", "dpost_bias", "dnext_weight", "dnext_bias")
    out.update({k: np.zeros(C) for k in vec})
    out.update({"abs_" + k: np.zeros(C) for k in vec})
    out["dgate_item"], out["abs_dgate_item"] = np.zeros((B, C)), np.zeros((B, C))

    def add(name, v, b=None):
        at = slice(None) if b is None else b
        out[name][at] += v
        out["abs_" + name][at] += np.abs(v)

    rs = 1.0 if rscale is None else rscale
    for b in range(B):
        for t in range(T if lengths is None else min(max(int(lengths[b]), 0), T)):
            g = np.zeros(C) if dy is None else dy[b, :, t].astype(F)
            if dn is not None:
                hat, r, _ = _norm(y[b, :, t], None, None, layer, eps)
                g = g + _norm_back(dn[b, :, t], hat, r, next_weight, layer)
                add("dnext_weight", dn[b, :, t] * hat)
                add("dnext_bias", dn[b, :, t])
            out["dx"][b, :, t] = g
            if f is None:
                continue
            z, gt = f[b, :, t], _gate_at(gate, b, t)
            h = z
            dh = rs * gt * g
            if post:
                hat, r, h = _norm(z, post_weight, post_bias, layer, eps)
                add("dpost_weight", dh * hat)
                add("dpost_bias", dh)
                out["df"][b, :, t] = _norm_back(dh, hat, r, post_weight, layer)
            else:
                out["df"][b, :, t] = dh
            out["dgate_element"][b, :, t] = rs * g * h
            add("dgate_item", rs * g * h, b)
            add("drscale", g * gt * h)
    return out


# ---- AdamW -----------------------------------------------------------------------------------------------------------------
def e4m3_values():
    """The 256 values of the codes (no infinities; 0x7f and 0xff are NaN)."""
    out = np.empty(256)
    for c in range(256):
        e, m = c >> 3 & 15, c & 7
        v = m * 2.0 ** -9 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        out[c] = np.nan if c & 127 == 127 else (-v if c >> 7 else v)
    return out


def mixed(element, seed):
    M = 0xFFFFFFFF
    h = (int(element) * 0x9E3779B9 & M) ^ (seed & M)
    h = (h ^ h >> 16) * 0x6A09E667 & M
    h = (h ^ h >> 13) * 0xBB67AE85 & M
    return h ^ h >> 16


def _encode(v, scale, u, positive):
    """Code of one value."""
    if not np.isfinite(v):
        return 127
    values = e4m3_values()[:127]
    z = abs(v) / scale
    e = max(int(np.floor(np.log2(z))), -6) if z > 0 else -6
    ulp = 2.0 ** (e - 3)
    q = min(np.floor(z / ulp + u / 65536) * ulp, 448.0)
    code = int(np.searchsorted(values, q))
    assert values[code] == q
    if positive and code == 0 and z > 0:
        code = 1
    return code | (128 if v < 0 else 0)


def _scale(v):
    fin = np.abs(v[np.isfinite(v)])
    amax = fin.max() if fin.size else 0.0
    return F(max(np.float32(amax / 448), np.float32(2.0 ** -126))) if amax > 0 else F(1)


def adamw(param, grad, m, v, step, lr, beta1, beta2, eps, weight_decay, grad_scale=1.0):
    """(param, m, v) in float64, states in full precision."""
    g = np.asarray(grad, F) * grad_scale
    m = beta1 * np.asarray(m, F) + (1 - beta1) * g
    v = beta2 * np.asarray(v, F) + (1 - beta2) * g * g
    p = np.asarray(param, F) * (1 - lr * weight_decay) - lr / (1 - beta1 ** step) * m / (np.sqrt(v / (1 - beta2 ** step)) + eps)
    return p, m, v


def adamw8(param, grad, m_codes, m_scale, r_codes, r_scale, first_block, seed, step, lr, beta1, beta2, eps, weight_decay,
           grad_scale=1.0):
    """(param, m codes, m scales, r codes, r scales) of one tensor whose first block is number first_block of the plan."""
    val = e4m3_values()
    n = len(param)
    blk = np.arange(n) // 256
    m = val[m_codes] * np.asarray(m_scale, F)[blk]
    r = val[r_codes] * np.asarray(r_scale, F)[blk]
    p, m, v = adamw(param, grad, m, r * r, step, lr, beta1, beta2, eps, weight_decay, grad_scale)
    r = np.sqrt(v)
    mc, rc = np.empty(n, np.uint8), np.empty(n, np.uint8)
    ms, rs = np.empty(blk[-1] + 1), np.empty(blk[-1] + 1)
    for i in range(blk[-1] + 1):
        at = slice(256 * i, min(256 * i + 256, n))
        ms[i], rs[i] = _scale(m[at]), _scale(r[at])
        for j in range(at.start, at.stop):
            bits = mixed(256 * (first_block + i) + j - at.start, seed)
            mc[j] = _encode(m[j], ms[i], bits & 0xFFFF, False)
            rc[j] = _encode(r[j], rs[i], bits >> 16, True)
    return p, mc, ms, rc, rs
