"""Float64 oracle of the token models' operators: RMS norm with the residual's
addition, embedding, attention over packed sequences, and their gradients.

Attention also returns bounds of the rounding that the documented arithmetic may
add: probabilities and score gradients rounded to bf16 (half a step: 2^-8 of the
value), everything else in fp32 (2^-24 an operation).
"""
import numpy as np

U16, U24 = 2.0 ** -8, 2.0 ** -24  # half a step of bf16 and fp32, of the value


# ---------------------------------------------------------------- RMS norm --
def rms_stat(h, eps):
    return 1.0 / np.sqrt((h * h).mean(1) + eps)


def rms_apply(h, st, w):
    return h * st[:, None] * w


def rms_backward(g, gh, h, st, w):
    """d, dw and the magnitudes that enter each of their elements."""
    xhat = h * st[:, None]
    du = g * w
    d = st[:, None] * (du - xhat * (du * xhat).mean(1, keepdims=True))
    mag = st[:, None] * (np.abs(du) + np.abs(xhat) * np.abs(du * xhat).mean(1, keepdims=True))
    if gh is not None:
        d, mag = d + gh, mag + np.abs(gh)
    return d, (g * xhat).sum(0), mag, np.abs(g * xhat).sum(0)


def group_scales(u, group):
    """The scale of each group of columns of an 8-bit output."""
    c = u.shape[1]
    group = group or c
    return np.stack([np.maximum(np.abs(u[:, a:a + group]).max(1), 1e-30) / 448.0 for a in range(0, c, group)], 1)


# --------------------------------------------------------------- embedding --
def embed(ids, w, scale):
    ok = (ids >= 0) & (ids < len(w))
    return np.where(ok[:, None], w[np.where(ok, ids, 0)] * scale, 0.0)


def embed_backward(ids, g, vocab, scale):
    d, mag = np.zeros((vocab, g.shape[1])), np.zeros((vocab, g.shape[1]))
    ok = (ids >= 0) & (ids < vocab)
    np.add.at(d, ids[ok], g[ok])
    np.add.at(mag, ids[ok], np.abs(g[ok]))
    return d * scale, mag * abs(scale)


# --------------------------------------------------------------- attention --
def visible(lq, lk, causal):
    """[lq, lk]: does query i see key j?"""
    seen = np.ones((lq, lk), bool)
    return np.tril(seen, lk - lq) if causal else seen


def _finite(*mats):
    return [np.where(np.isfinite(m), m, 0.0) for m in mats]


def _odd(m):
    """Rows that hold an infinity or a NaN."""
    return ~np.isfinite(m).all(1)


def attention(q, k, v, qoff, koff, causal, scale):
    """o [tq, heads, dim], lse [heads, tq] and their error bounds.  Rows of no sequence are NaN.
    What a query does not see plays no part, whatever it holds; infinities and NaNs that it sees do."""
    tq, heads, dim = q.shape
    rep = heads // k.shape[1]
    o, eo = np.full((tq, heads, dim), np.nan), np.full((tq, heads, dim), np.nan)
    lse, el = np.full((heads, tq), np.nan), np.full((heads, tq), np.nan)
    for a, b, c, d in zip(qoff, qoff[1:], koff, koff[1:]):
        lq, lk = b - a, d - c
        seen = visible(lq, lk, causal)
        for h in range(heads):
            Q, K, V = q[a:b, h], k[c:d, h // rep], v[c:d, h // rep]
            Qf, Kf, Vf = _finite(Q, K, V)
            e = np.where(seen, Qf @ Kf.T * scale, -np.inf)
            mag = np.where(seen, np.abs(Qf) @ np.abs(Kf).T * scale, 0.0)
            if lk == 0 or lq == 0:
                o[a:b, h], eo[a:b, h], lse[h, a:b], el[h, a:b] = 0, 1e-30, -np.inf, 0
                continue
            top = e.max(1)
            base = np.where(np.isinf(top), 0.0, top)[:, None]
            p = np.exp(e - base)
            z = p.sum(1)
            none = z == 0
            p = p / np.where(none, 1, z)[:, None]
            o[a:b, h] = p @ Vf
            with np.errstate(divide="ignore"):
                lse[h, a:b] = base[:, 0] + np.log(z)
            # a score is off by dim products and sums and a few operations more, its exponential
            # (a power of two, in hardware to about 2^-22) by as much of itself; a sum of lk terms
            rel = (dim + 16) * U24 * 2 * (mag.max(1) + np.abs(base[:, 0])) + (lk + 64) * U24
            # o is the mean of the values by the rounded weights, so with weights off by u p at most it is off by
            # sum u p |v - o| <= u (sum p |v| + |o|), and rounded itself
            eo[a:b, h] = (U16 + 2 * rel)[:, None] * (p @ np.abs(Vf)) + 2 * U16 * np.abs(o[a:b, h]) + 1e-30
            el[h, a:b] = np.where(none, 0, rel + 4 * U24 * np.abs(np.where(none, 0, lse[h, a:b])))
            # rows with infinities and NaNs, of the keys that they see alone
            for i in np.flatnonzero((seen & (_odd(K) | _odd(V))).any(1) | (_odd(Q) & seen.any(1))):
                with np.errstate(invalid="ignore", divide="ignore"):
                    e = (Q[i] * K[seen[i]]).sum(1) * scale
                    p = np.exp(e - e.max())
                    o[a + i, h] = (p[:, None] * V[seen[i]]).sum(0) / p.sum()
                    lse[h, a + i] = e.max() + np.log(p.sum())
    return o, lse, eo, el


def attention_backward(g, q, k, v, o, lse, qoff, koff, causal, scale):
    """dq, dk, dv and their error bounds, for the o and lse that the call is given."""
    tq, heads, dim = q.shape
    rep = heads // k.shape[1]
    out = [np.full(t.shape, np.nan) for t in (q, k, v)]
    err = [np.full(t.shape, np.nan) for t in (q, k, v)]
    for a, b, c, d in zip(qoff, qoff[1:], koff, koff[1:]):
        lq, lk = b - a, d - c
        seen = visible(lq, lk, causal)
        for t, e in zip(out, err):
            n = slice(a, b) if t is out[0] else slice(c, d)
            t[n], e[n] = 0, 0
        if lq == 0 or lk == 0:
            continue
        for h in range(heads):
            kh = h // rep
            raw = q[a:b, h], k[c:d, kh], v[c:d, kh], g[a:b, h], o[a:b, h]
            Q, K, V, G, O = _finite(*raw)
            L = lse[h, a:b]
            fin = np.isfinite(L)
            Lf = np.where(fin, L, 0.0)
            # rows with infinities and NaNs are added below, of the keys that they see alone
            s = seen & ~np.isneginf(L)[:, None]
            odd = (s & (_odd(raw[1]) | _odd(raw[2]))).any(1) | _odd(raw[0]) | _odd(raw[3]) | _odd(raw[4]) | np.isnan(L)
            rest, s = s & odd[:, None], s & fin[:, None] & ~odd[:, None]
            e = Q @ K.T * scale
            mag = np.abs(Q) @ np.abs(K).T * scale
            p = np.where(s, np.exp(np.where(s, e - Lf[:, None], 0.0)), 0.0)
            dp, delta = G @ V.T, (G * O).sum(1)
            ds = p * (dp - delta[:, None])
            rel = (dim + 16) * U24 * 2 * (mag + np.abs(Lf)[:, None]) + 64 * U24
            ep = p * (U16 + rel)
            eds = (U16 + rel) * np.abs(ds) + p * (dim + 16) * U24 * (np.abs(G) @ np.abs(V).T +
                                                                    (np.abs(G) * np.abs(O)).sum(1)[:, None])
            chain = (max(lq * rep, lk) + 64) * U24
            out[0][a:b, h] = ds @ K * scale
            err[0][a:b, h] = (eds + chain * np.abs(ds)) @ np.abs(K) * scale
            out[1][c:d, kh] += ds.T @ Q * scale
            err[1][c:d, kh] += (eds + chain * np.abs(ds)).T @ np.abs(Q) * scale
            out[2][c:d, kh] += p.T @ G
            err[2][c:d, kh] += (ep + chain * p).T @ np.abs(G)
            for i in np.flatnonzero(rest.any(1)):
                n = rest[i]
                Qi, Gi, Oi, Kn, Vn = raw[0][i], raw[3][i], raw[4][i], raw[1][n], raw[2][n]
                with np.errstate(invalid="ignore", over="ignore"):
                    p = np.exp((Qi * Kn).sum(1) * scale - L[i])[:, None]
                    ds = p * ((Gi * Vn).sum(1) - (Gi * Oi).sum())[:, None] * scale
                    out[0][a + i, h] += (ds * Kn).sum(0)
                    out[1][c:d, kh][n] += ds * Qi
                    out[2][c:d, kh][n] += p * Gi
    for t, e in zip(out, err):
        e += U16 * np.abs(t) + 1e-30
    return out, err
