"""The language-model operators in 64 bits (numpy / torch on the CPU), by their definitions, and error bounds.

Bounds.  u = 2^-24 is half a step of fp32.  A sum of n terms formed in fp32 in
any order is off by at most (n + 1) u sum |terms| to first order; SUM doubles
that (second order, and matrix units that align products before they add).
Rounding once to the output's type adds half a step of that type relative to
the value, torch.finfo(t).eps / 2.
"""
import math

import numpy as np
import torch

U32 = 2.0 ** -24
C0, C1 = math.sqrt(2.0 / math.pi), 0.044715


def half_step(dt):
    return torch.finfo(dt).eps / 2


def SUM(n):
    return 2.0 * (n + 1) * U32


def f64(t):
    return t.detach().cpu().double().numpy()


def within(got, want, bound, what=""):
    """got (a tensor) within `bound` (an array) of want everywhere; where want is not finite, got is the same."""
    x = f64(got)
    assert x.shape == want.shape, (x.shape, want.shape)
    fin = np.isfinite(want)
    assert np.array_equal(np.isnan(x), np.isnan(want)), "%s: NaN in other places" % what
    assert np.array_equal(x[~fin & ~np.isnan(want)], want[~fin & ~np.isnan(want)]), "%s: infinities" % what
    bound = np.broadcast_to(bound, want.shape)[fin]
    over = np.abs(x[fin] - want[fin]) - bound
    assert over.size == 0 or over.max() <= 0, "%s: off by %.3g more than %.3g" % (what, over.max(), bound[over.argmax()])


def clip_factors(norm, C):
    """min(1, C / (norm + 1e-6)); 0 for a negative norm, NaN for a NaN or infinite one."""
    norm = np.asarray(norm, dtype=np.float64)
    with np.errstate(invalid="ignore"):
        c = np.minimum(1.0, C / (norm + 1e-6)) if math.isfinite(C) else np.ones_like(norm)
    c[~np.isfinite(norm)] = np.nan
    c[norm < 0] = 0.0
    return c


def lookup(ids, E, scale):
    ok = (ids >= 0) & (ids < E.shape[0])
    y = scale * E[np.where(ok, ids, 0)]
    y[~ok] = 0.0
    return y


def tokens(ids, B, V, scale, norm, C):
    """(sum, bound of the fp32 error): sum[v] = scale * sum of c_n B[n][t] over ids[n][t] = v."""
    N, T, D = B.shape
    out, mag, cnt = np.zeros((V, D)), np.zeros((V, D)), np.zeros(V)
    c = np.ones(N) if norm is None else clip_factors(norm, C)
    for n in range(N):
        if norm is not None and norm[n] < 0:
            continue                                 # a padding row: not looked at
        ok = (ids[n] >= 0) & (ids[n] < V)
        with np.errstate(invalid="ignore"):
            np.add.at(out, ids[n][ok], scale * c[n] * B[n][ok])
            np.add.at(mag, ids[n][ok], np.abs(scale * c[n] * B[n][ok]))
        np.add.at(cnt, ids[n][ok], 1)
    # the sum, the factor (two roundings in c, one each in C / (norm + 1e-6)) and the scale
    return out, (SUM(1) * (cnt + 5))[:, None] * mag


def gate(act, g):
    """sigmoid(w), w = g (SiLU) or 2 sqrt(2/pi) (g + 0.044715 g^3): act(g) = g gate(g) for both activations; and w'."""
    w = g if act == 0 else 2 * C0 * (g + C1 * g ** 3)
    dw = np.ones_like(g) if act == 0 else 2 * C0 * (1 + 3 * C1 * g ** 2)
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-w)), dw


def act_and_slope(act, g):
    p, dw = gate(act, g)
    return g * p, p + g * p * (1 - p) * dw


def ffn_forward(act, X, Wg, Wu, dt):
    """H, G, U and the bounds of their errors in type dt."""
    K, h = X.shape[1], half_step(dt)
    G, U = X @ Wg.T, X @ Wu.T
    eg, eu = SUM(K) * (np.abs(X) @ np.abs(Wg).T), SUM(K) * (np.abs(X) @ np.abs(Wu).T)
    a, _ = act_and_slope(act, G)
    H = a * U
    # |act'| <= 1.13 for both; expf, the sum, the quotient and the products of act and H: 16 half steps, and an
    # error of w (relative 8 u) moves the gate by at most |w| gate (1 - gate) 8 u <= 0.28 * 8 u
    ea = 1.13 * eg + 20 * U32 * np.abs(G) * 0.3 + 16 * U32 * np.abs(a)
    eh = ea * np.abs(U) + np.abs(a) * eu + ea * eu + 2 * U32 * np.abs(H)
    tiny = float(torch.finfo(dt).tiny)               # results below the normal range may be flushed
    return (H, G, U), (eh + h * (np.abs(H) + eh) + tiny, eg + h * (np.abs(G) + eg) + tiny,
                       eu + h * (np.abs(U) + eu) + tiny)


def ffn_backprops(act, dH, G, U, dt):
    h = half_step(dt)
    a, s = act_and_slope(act, G)
    BG, BU = dH * U * s, dH * a
    p, dw = gate(act, G)
    # as above for the gate; the slope's second term has five more roundings and p (1 - p) <= 1/4
    ea = 20 * U32 * np.abs(G) * 0.3 + 16 * U32 * np.abs(a)
    es = 32 * U32 * (p + np.abs(G * dw) * np.minimum(p, 1 - p) + 0.3 * (1 + np.abs(G * dw) * 0.25))
    tiny = float(torch.finfo(dt).tiny)
    eg = np.abs(dH * U) * es + 3 * U32 * np.abs(BG)
    eu = np.abs(dH) * ea + 3 * U32 * np.abs(BU)
    return (BG, BU), (eg + h * (np.abs(BG) + eg) + tiny, eu + h * (np.abs(BU) + eu) + tiny)


def ffn_dx(BG, BU, Wg, Wu, dt):
    dX = BG @ Wg + BU @ Wu
    e = SUM(2 * BG.shape[1]) * (np.abs(BG) @ np.abs(Wg) + np.abs(BU) @ np.abs(Wu))
    return dX, e + half_step(dt) * (np.abs(dX) + e) + float(torch.finfo(dt).tiny)


def global_norm(arrays):
    return math.sqrt(sum(math.fsum((a.reshape(-1).astype(np.float64) ** 2).tolist()) for a in arrays))
