"""Rotary positions, attention and the distillation loss in 64 bits (numpy), by their definitions, with bounds of the
errors that fp32 sums and one rounding to the output's type leave (lm_ref has the rules: SUM(n) for a sum of n terms,
half a step of the type for a rounding)."""
import numpy as np

from lm_ref import SUM, U32, half_step

# Below 2^-126 a weight, or its product, may be taken as 0 (the units flush subnormal numbers): each is off by at most TINY
# then, and so is every sum by TINY times what multiplies the weight, and by TINY for every term.
TINY = 2.0 ** -126


# ---------------------------------------------------------------------------
# rotary
# ---------------------------------------------------------------------------

def rotary(X, pos, sections, freq, adjacent, inverse, dt):
    """X [N][T][H][D]; pos [axes][N][T]; returns (Y, bound)."""
    P = sum(sections)
    axis = np.repeat(np.arange(len(sections)), sections)
    ang = np.moveaxis(pos[axis].astype(np.float64), 0, -1) * freq[:P]                  # [N][T][P]
    c, s = np.cos(ang)[:, :, None], np.sin(ang)[:, :, None]
    if inverse:
        s = -s
    Y = X.copy()
    at = (slice(0, 2 * P, 2), slice(1, 2 * P, 2)) if adjacent else (slice(0, P), slice(P, 2 * P))
    a, b = X[..., at[0]], X[..., at[1]]
    Y[..., at[0]], Y[..., at[1]] = a * c - b * s, b * c + a * s
    # sine and cosine: the angle less whole turns is off by 2^-52 of the angle (two roundings) and half a step of fp32 of
    # half a turn, the function by 2 steps; two products and a sum, half a step each
    err = np.zeros_like(X)
    e = 2.0 ** -51 * np.abs(ang)[:, :, None] + 10 * U32
    mag = (np.abs(a) + np.abs(b)) * e
    err[..., at[0]], err[..., at[1]] = mag, mag
    return Y, err + half_step(dt) * (np.abs(Y) + err) * (err > 0)


# ---------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------

class Mask:
    def __init__(self, N, Tq, Tk, causal=False, last=False, lens=None, prefix=None, docs=None):
        self.L = np.clip(lens, 0, Tk) if lens is not None else np.full(N, Tk)
        i, j = np.arange(Tq), np.arange(Tk)
        self.see, self.far = [], []
        for n in range(N):
            L = int(self.L[n])
            p = i + (L - Tq if last else 0)
            see = ((p >= 0) & (p < L))[:, None] & (j < L)[None]
            if causal:
                see &= (j[None] <= p[:, None]) | (j[None] < (prefix[n] if prefix is not None else 0))
            if docs is not None and Tk > 0:
                d = docs[n][np.clip(p, 0, Tk - 1)]
                see &= (d[:, None] == docs[n][None]) & (d >= 0)[:, None]
            self.see.append(see)
            self.far.append(np.abs(p[:, None] - j[None]))


def _scores(q, k, scale, cap, slope, far, see):
    """Scores, the cap's derivative, and the scores' error bound."""
    with np.errstate(invalid="ignore", over="ignore"):
        x = scale * (q @ k.T)
        ex = abs(scale) * SUM(q.shape[1]) * (np.abs(q) @ np.abs(k).T) + 2 * U32 * np.abs(x)
        bend, s = np.ones_like(x), x
        if cap > 0:
            t = np.tanh(x / cap)
            # tanh has slope <= 1; its own form is off by 10 half steps of itself (the shorter polynomial), its coefficients' and
            # steps' roundings 10 more, the products with the cap 4
            s, bend = cap * t, 1 - t * t
            ex = ex + 24 * U32 * np.abs(s)
        bias = slope * far
        s = s - bias
        # the bias, its difference, the factor log2 e, the maximum's or lse's difference: half a step each, of what is largest
        es = ex + 4 * U32 * (np.abs(s) + np.abs(bias))
    return np.where(see, s, -np.inf), bend, np.where(see, es, 0.0)


def _over_visible(w, x, see):
    """sum_j w[i][j] x[j] over the visible j (a hidden x is not looked at, whatever it is)."""
    if np.isfinite(x).all():
        return w @ x
    return (w[:, :, None] * np.where(see[:, :, None], x[None], 0.0)).sum(1)


def attention(Q, K, V, mask, scale, cap=0.0, slopes=None, dt=None):
    """Q [N][Tq][Hq][D], K, V [N][Tk][Hk][D] -> O, lse and the bounds of their errors."""
    N, Tq, Hq, D = Q.shape
    Tk, Hk = K.shape[1:3]
    G, h = Hq // Hk, half_step(dt)
    hp = h if h > 1e-6 else 0.0                       # weights are rounded to bf16 for bf16 inputs, kept in fp32 else
    O, lse = np.zeros_like(Q), np.full((N, Hq, Tq), -np.inf)
    eO, el = np.zeros_like(Q), np.zeros((N, Hq, Tq))
    for n in range(N):
        see = mask.see[n]
        used = see.any(0)
        for hq in range(Hq):
            k, v = K[n, used, hq // G], V[n, used, hq // G]
            sl = 0.0 if slopes is None else slopes[hq]
            s, _, es = _scores(Q[n, :, hq], k, scale, cap, sl, mask.far[n][:, used], see[:, used])
            rows = see.any(1)
            if not rows.any():
                continue
            s, es = s[rows], es[rows]
            with np.errstate(invalid="ignore"):
                top = s.max(1, keepdims=True)
                w = np.where(see[rows][:, used], np.exp(s - top), 0.0)
            tot = w.sum(1, keepdims=True)
            p = w / tot
            with np.errstate(invalid="ignore"):
                sub = see[rows][:, used]
                o = _over_visible(p, v, sub)
                mag = _over_visible(p, np.abs(v), sub)
            # a weight is off by its score's error, the maximum's that it is taken from and 4 half steps (exp2, rescaling
            # counted with the sum); the sum by as much
            e = es.max(1, keepdims=True)
            n_keys = w.shape[1]
            rel = 2 * (2 * e + 4 * U32) + 2 * SUM(n_keys) + hp
            O[n, rows, hq] = o
            flushed = TINY * (n_keys + 1 + _over_visible(sub.astype(float), np.abs(v), sub))
            eO[n, rows, hq] = rel * mag + h * (np.abs(o) + rel * mag) + flushed
            lse[n, hq, rows] = (top + np.log(tot))[:, 0]
            el[n, hq, rows] = (2 * e + SUM(n_keys) + 8 * U32 * (1 + np.abs(top) + np.abs(np.log(tot))))[:, 0]
    return (O, lse), (eO, el)


def attention_grads(Q, K, V, dO, mask, scale, cap=0.0, slopes=None, dt=None):
    """dQ, dK, dV and their bounds, where the call takes O and lse as the forward call gives them in type dt."""
    N, Tq, Hq, D = Q.shape
    Tk, Hk = K.shape[1:3]
    G, h = Hq // Hk, half_step(dt)
    hp = h if h > 1e-6 else 0.0
    (O, lse), (eO, el) = attention(Q, K, V, mask, scale, cap, slopes, dt)
    out = [np.zeros_like(Q), np.zeros_like(K), np.zeros_like(V)]
    err = [np.zeros_like(Q), np.zeros_like(K), np.zeros_like(V)]
    for n in range(N):
        see = mask.see[n]
        for hq in range(Hq):
            g_ = hq // G
            rows, used = see.any(1), see.any(0)
            if not rows.any():
                continue
            sub = see[rows][:, used]
            q, k, v, d = Q[n, rows, hq], K[n, used, g_], V[n, used, g_], dO[n, rows, hq]
            sl = 0.0 if slopes is None else slopes[hq]
            s, bend, es = _scores(q, k, scale, cap, sl, mask.far[n][rows][:, used], sub)
            with np.errstate(invalid="ignore"):
                p = np.where(sub, np.exp(s - lse[n, hq, rows][:, None]), 0.0)
                dp = d @ v.T
                delta = (d * O[n, rows, hq]).sum(1, keepdims=True)
                g = np.where(sub, p * (dp - delta) * bend * scale, 0.0)
                ep = 2 * (es + el[n, hq, rows][:, None] + 4 * U32 * (1 + np.abs(lse[n, hq, rows][:, None])))
                edp = SUM(D) * (np.abs(d) @ np.abs(v).T)
                edelta = (np.abs(d) * eO[n, rows, hq]).sum(1, keepdims=True) + SUM(D) * (
                    np.abs(d) * (np.abs(O[n, rows, hq]) + eO[n, rows, hq])).sum(1, keepdims=True)
                # the cap's derivative: 16 half steps of 1
                eg = np.where(sub, np.abs(g) * (ep + hp + 8 * U32) + abs(scale) * p * (
                    (edp + edelta) * bend + (np.abs(dp - delta) + edp + edelta) * (16 * U32 + 2 * es / max(cap, 1e-30)) * (cap > 0)),
                    0.0)
                eg = eg + np.where(sub, TINY * (1 + abs(scale) * (np.abs(dp - delta) + edp + edelta)), 0.0)
                nq, nk = int(rows.sum()) * G, int(used.sum())
                out[0][n, rows, hq] = _over_visible(g, k, sub)
                err[0][n, rows, hq] = _over_visible(eg + SUM(nk) * (np.abs(g) + eg), np.abs(k), sub)
                out[1][n, used, g_] += _over_visible(g.T, q, sub.T)
                err[1][n, used, g_] += _over_visible((eg + SUM(nq) * (np.abs(g) + eg)).T, np.abs(q), sub.T)
                out[2][n, used, g_] += _over_visible(p.T, d, sub.T)
                ev = np.where(sub, p * (ep + hp + SUM(nq) * (1 + ep)) + TINY, 0.0)
                err[2][n, used, g_] += _over_visible(ev.T, np.abs(d), sub.T)
    return out, [e + h * (np.abs(o) + e) + TINY * (2 + Tk + Tq * G) for o, e in zip(out, err)]


# ---------------------------------------------------------------------------
# distillation
# ---------------------------------------------------------------------------

def distill(Z, ids, logits, labels, alpha, tau, weight, dt):
    """loss, dZ and their bounds; rows one by one."""
    M, V = Z.shape
    loss, dZ = np.zeros(M), np.zeros((M, V))
    el, eZ = np.zeros(M), np.zeros((M, V))
    for m in range(M):
        w = 1.0 if weight is None else weight[m]
        if w == 0:
            continue
        z = Z[m]

        def soften(t):
            with np.errstate(invalid="ignore", over="ignore"):
                top = z.max() / t
                e = np.exp(z / t - top)
                q = e / e.sum()
                # an argument's difference and product are off by 3 half steps of its size, exp2 by 2, the sum as a sum
                far = np.where(np.isfinite(z), np.abs(z / t - top), 0.0)
                rel = 3 * U32 * far + 4 * U32 + SUM(V) + 3 * U32 * (q * far).sum()
                return top + np.log(e.sum()), q, rel
        ok = np.zeros(0, dtype=bool) if ids is None else (ids[m] >= 0) & (ids[m] < V)
        if alpha > 0 and ok.any():
            k, t = ids[m][ok], logits[m][ok].astype(np.float64) / tau
            tt = t.max() + np.log(np.exp(t - t.max()).sum())
            P = np.exp(t - tt)
            far = np.where(P > 0, np.abs(t - t.max()), 0.0)
            ls, q, rel = soften(tau)
            with np.errstate(invalid="ignore"):
                terms = np.where(P > 0, P * ((t - tt) - (z[k] / tau - ls)), 0.0)
                size = np.where(P > 0, P * (np.abs(t) + abs(tt) + np.abs(z[k] / tau) + abs(ls) + far + 2), 0.0)
            loss[m] += alpha * tau ** 2 * terms.sum()
            # every logarithm and difference: 4 half steps of its size, the softmax sums' errors, P's own
            el[m] += alpha * tau ** 2 * (12 * U32 * size + P * (SUM(V) + SUM(len(k)) + 3 * U32 * 20)).sum()
            el[m] += alpha * tau ** 2 * (np.abs(np.where(P > 0, terms, 0.0)) * (8 + len(k)) * U32 * (1 + far)).sum()
            g = alpha * tau * q
            eg = np.abs(g) * (rel + 6 * U32)
            np.add.at(g, k, -alpha * tau * P)
            np.add.at(eg, k, alpha * tau * P * (8 * U32 * (1 + far) + SUM(len(k))))
            dZ[m] += g
            eZ[m] += eg
        if labels is not None and alpha < 1 and 0 <= labels[m] < V:
            ls, q, rel = soften(1.0)
            x = z[labels[m]]
            loss[m] += (1 - alpha) * (ls - x)
            el[m] += (1 - alpha) * (SUM(V) + 60 * U32 + 8 * U32 * (abs(ls) + abs(x) + abs(z.max())))
            g = (1 - alpha) * q
            eg = np.abs(g) * (rel + 6 * U32)
            g[labels[m]] -= 1 - alpha
            eg[labels[m]] += (1 - alpha) * 4 * U32
            dZ[m] += g
            eZ[m] += eg
        loss[m] *= w
        dZ[m] *= w
        el[m] = abs(w) * el[m] + 4 * U32 * abs(loss[m])
        eZ[m] = abs(w) * eZ[m] + 4 * U32 * np.abs(dZ[m])
    return loss, dZ, el + 1e-37, eZ + half_step(dt) * (np.abs(dZ) + eZ) + 1e-37
