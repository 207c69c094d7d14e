"""Plain float64 implementations of the operators on a decoder's tokens (numpy, loops over items, heads and tokens), from the definitions
in include/nm_embedding.h, nm_head_norm.h, nm_paged_attention.h and nm_token_scores.h.  Used by the tests only; shares no code with
the library.  `mag` results are sums of the magnitudes of what a result is the sum of."""
from __future__ import annotations

import numpy as np

F = np.float64


def clipped(v, n):
    return min(max(int(v), 0), n)


# ---- embedding ------------------------------------------------------------------------------------------------------------
def embedding_fwd(ids, table, scale, lengths=None):
    B, U = ids.shape
    V, C = table.shape
    out = np.zeros((B, C, U))
    for b in range(B):
        for u in range(U if lengths is None else clipped(lengths[b], U)):
            if 0 <= ids[b, u] < V:
                out[b, :, u] = scale * np.asarray(table[ids[b, u]], F)
    return out


def embedding_bwd(dout, ids, V, scale, lengths=None):
    """(dtable, mag, how often every token occurs)"""
    B, C, U = dout.shape
    out, mag, count = np.zeros((V, C)), np.zeros((V, C)), np.zeros(V, int)
    for b in range(B):
        for u in range(U if lengths is None else clipped(lengths[b], U)):
            v = ids[b, u]
            if 0 <= v < V:
                out[v] += scale * dout[b, :, u]
                mag[v] += np.abs(scale * dout[b, :, u])
                count[v] += 1
    return out, mag, count


# ---- norms and rotation of heads ---------------------------------------------------------------------------------------------
def pairs_of(D, rot, pairs):
    half = rot // 2
    return [(2 * i, 2 * i + 1) if pairs else (i, i + half) for i in range(half)]


def turned(n, position, freqs, pairs, back=False):
    """(n [..., D] turned, mag)"""
    out, mag = n.copy(), np.abs(n)
    for i, (a, b) in enumerate(pairs_of(n.shape[-1], 2 * len(freqs), pairs)):
        angle = float(position) * float(freqs[i]) * (-1 if back else 1)
        out[..., a] = n[..., a] * np.cos(angle) - n[..., b] * np.sin(angle)
        out[..., b] = n[..., b] * np.cos(angle) + n[..., a] * np.sin(angle)
        mag[..., a] = mag[..., b] = np.abs(n[..., a]) + np.abs(n[..., b])
    return out, mag


def head_norm_fwd(x, heads, kv_heads, *, norm, qw=None, kw=None, eps=1e-5, freqs=(), pairs=False, positions=None, lengths=None):
    """(out, mag) like x."""
    B, C, U = x.shape
    N = heads + kv_heads
    D = C // N
    x = np.asarray(x, F).reshape(B, N, D, U)
    out, mag = np.zeros(x.shape), np.zeros(x.shape)
    for b in range(B):
        for u in range(U if lengths is None else clipped(lengths[b], U)):
            for h in range(N):
                n = x[b, h, :, u].copy()
                if norm:
                    w = qw if h < heads else kw
                    n = n / np.sqrt((n * n).mean() + eps) * (1.0 if w is None else np.asarray(w, F))
                out[b, h, :, u], mag[b, h, :, u] = turned(n, u if positions is None else positions[b, u], freqs, pairs)
    return out.reshape(B, C, U), mag.reshape(B, C, U)


def head_norm_bwd(dout, x, heads, kv_heads, *, norm, qw=None, kw=None, eps=1e-5, freqs=(), pairs=False, positions=None, lengths=None):
    """(dx, dqw, dkw, mags: {"dx", "dqw", "dkw"}); dw of a norm without a weight is that of ones."""
    B, C, U = x.shape
    N = heads + kv_heads
    D = C // N
    x, g = np.asarray(x, F).reshape(B, N, D, U), np.asarray(dout, F).reshape(B, N, D, U)
    dx, mx = np.zeros(x.shape), np.zeros(x.shape)
    dw, mw = np.zeros((2, D)), np.zeros((2, D))
    for b in range(B):
        for u in range(U if lengths is None else clipped(lengths[b], U)):
            for h in range(N):
                d, md = turned(g[b, h, :, u], u if positions is None else positions[b, u], freqs, pairs, back=True)
                if not norm:
                    dx[b, h, :, u], mx[b, h, :, u] = d, md
                    continue
                z, key = x[b, h, :, u], int(h >= heads)
                w = kw if key else qw
                w = np.ones(D) if w is None else np.asarray(w, F)
                r = 1 / np.sqrt((z * z).mean() + eps)
                dw[key] += d * z * r
                mw[key] += md * np.abs(z) * r
                dx[b, h, :, u] = r * (w * d - z * r * (w * d * z * r).mean())
                mx[b, h, :, u] = r * (np.abs(w) * md + np.abs(z) * r * (np.abs(w) * md * np.abs(z) * r).mean())
    return dx.reshape(B, C, U), dw[0], dw[1], {"dx": mx.reshape(B, C, U), "dqw": mw[0], "dkw": mw[1]}


# ---- the paged cache -----------------------------------------------------------------------------------------------------------
def new_tokens(lengths, q_lengths, b, U):
    """(how many tokens of item b are new, place of the first)"""
    n = U if q_lengths is None else clipped(q_lengths[b], U)
    return n, max(int(lengths[b]), 0) - n


def row_of(table, b, place, page, pages):
    """(page, row) of a sequence's place, or None"""
    if place < 0 or place // page >= table.shape[1] or not 0 <= table[b, place // page] < pages:
        return None
    return int(table[b, place // page]), place % page


def head_norm_cache(x, k_cache, v_cache, table, lengths, heads, kv_heads, *, q_lengths=None, **kw):
    """(q, k_cache, v_cache, and their mags; of untouched places of the cache the magnitude is 0); caches float64 copies."""
    B, C, U = x.shape
    N = heads + 2 * kv_heads
    D = C // N
    pages, _, page, _ = k_cache.shape
    k_cache, v_cache = np.array(k_cache, F), np.array(v_cache, F)
    mk, mv = np.zeros(k_cache.shape), np.zeros(v_cache.shape)
    q, mq = np.zeros((B, heads * D, U)), np.zeros((B, heads * D, U))
    for b in range(B):
        n, first = new_tokens(lengths, q_lengths, b, U)
        where = np.arange(first, first + U)[None]
        qk, mag = head_norm_fwd(x[b:b + 1, :(heads + kv_heads) * D], heads, kv_heads, positions=where, lengths=[n], **kw)
        q[b], mq[b] = qk[0, :heads * D], mag[0, :heads * D]
        for u in range(n):
            at = row_of(table, b, first + u, page, pages)
            if at:
                k_cache[at[0], :, at[1]] = qk[0, heads * D:, u].reshape(kv_heads, D)
                mk[at[0], :, at[1]] = mag[0, heads * D:, u].reshape(kv_heads, D)
                v_cache[at[0], :, :, at[1]] = x[b, (heads + kv_heads) * D:, u].reshape(kv_heads, D)
    return (q, k_cache, v_cache), (mq, mk, mv)


def paged_attn(q, k_cache, v_cache, table, lengths, heads, kv_heads, scale, *, q_lengths=None, window=0):
    """(o, lse, sum p|v|, largest sum of the magnitudes of a score's terms for every token [B, heads, U])"""
    B, HD, U = q.shape
    D, G = HD // heads, heads // kv_heads
    pages, _, page, _ = k_cache.shape
    q = np.asarray(q, F).reshape(B, heads, D, U)
    o, mag = np.zeros(q.shape), np.zeros(q.shape)
    lse, terms = np.full((B, heads, U), -np.inf), np.zeros((B, heads, U))
    for b in range(B):
        n, first = new_tokens(lengths, q_lengths, b, U)
        for u in range(n):
            places = [row_of(table, b, p, page, pages) for p in range(max(0, first + u + 1 - window) if window else 0, first + u + 1)]
            places = [p for p in places if p]
            if not places:
                continue
            pg, row = (np.array([p[i] for p in places]) for i in (0, 1))
            for h in range(heads):
                k, v = np.asarray(k_cache[pg, h // G, row], F), np.asarray(v_cache[pg, h // G, :, row], F)  # [places, D]
                s = scale * (k @ q[b, h, :, u])
                terms[b, h, u] = (np.abs(k) @ np.abs(q[b, h, :, u])).max() * abs(scale)
                e = np.exp(s - s.max())
                lse[b, h, u] = s.max() + np.log(e.sum())
                o[b, h, :, u] = (e / e.sum()) @ v
                mag[b, h, :, u] = (e / e.sum()) @ np.abs(v)
    return o.reshape(B, HD, U), lse, mag.reshape(B, HD, U), terms


# ---- token scores ---------------------------------------------------------------------------------------------------------------
def token_scores(scores, targets=None, top=0, lengths=None):
    """{"logp", "entropy", "lse" [B, U], "top_ids", "top_logp" [B, top, U]}"""
    B, V, U = scores.shape
    out = {"entropy": np.zeros((B, U)), "lse": np.zeros((B, U)), "logp": np.zeros((B, U)), "top_ids": np.full((B, top, U), -1),
           "top_logp": np.zeros((B, top, U))}
    for b in range(B):
        for u in range(U if lengths is None else clipped(lengths[b], U)):
            z = np.asarray(scores[b, :, u], F)
            best = z.max()
            nan = np.isnan(z).any()
            lse = np.nan if nan else best if np.isinf(best) and best < 0 else best + np.log(np.exp(z - best).sum())
            out["lse"][b, u] = lse
            some = z > -np.inf
            q = np.exp(z[some] - lse)
            out["entropy"][b, u] = np.nan if nan else -(q * (z[some] - lse)).sum()
            order = np.argsort(-np.where(np.isnan(z), -np.inf, z), kind="stable")[:top]
            out["top_ids"][b, :, u] = order
            out["top_logp"][b, :, u] = -np.inf if lse == -np.inf else z[order] - lse
            if targets is not None and 0 <= targets[b, u] < V:
                out["logp"][b, u] = -np.inf if lse == -np.inf else z[targets[b, u]] - lse
    return out


def token_scores_bwd(scores, targets, dlogp, dentropy, lengths=None):
    """(dscores, mag, logq with 0 for barred classes)"""
    B, V, U = scores.shape
    out, mag, logs = (np.zeros((B, V, U)) for _ in range(3))
    ref = token_scores(scores, targets, 0, lengths)
    for b in range(B):
        for u in range(U if lengths is None else clipped(lengths[b], U)):
            if ref["lse"][b, u] == -np.inf:
                continue
            z = np.asarray(scores[b, :, u], F)
            x = np.where(z > -np.inf, z - ref["lse"][b, u], 0.0)
            q = np.where(z > -np.inf, np.exp(x), 0.0)
            logs[b, :, u] = x
            if targets is not None and 0 <= targets[b, u] < V:
                hot = np.arange(V) == targets[b, u]
                out[b, :, u] += dlogp[b, u] * (hot - q)
                mag[b, :, u] += abs(dlogp[b, u]) * (hot + q)
            if dentropy is not None:
                out[b, :, u] -= dentropy[b, u] * q * (x + ref["entropy"][b, u])
                mag[b, :, u] += abs(dentropy[b, u]) * q * (np.abs(x) + ref["entropy"][b, u])
    return out, mag, logs
