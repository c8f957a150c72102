"""The gated feed-forward block over the range of its values: slopes between the tails, fp32 values of every size, and
what one row's values may do to the others."""
import math
import sys

import numpy as np
import pytest
import torch

import lm_ref as R
from paper_2109_12298_amd import binding as dp

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def say(*a):
    print("[case]", *a, file=sys.stderr, flush=True)


def ws(n):
    return torch.full((max(n, 16),), 0xFF, dtype=torch.uint8, device=DEV)       # NaN in every type


def forward(X, Wg, Wu, act):
    (M, K), F, dt = X.shape, Wg.shape[0], dp.dtype_of(X)
    outs = [torch.full((M, F), 7.0, dtype=X.dtype, device=DEV) for _ in range(3)]
    dp.dp_gated_ffn_forward(X, Wg, Wu, dt, M, K, F, act, *outs, ws(dp.dp_gated_ffn_forward_workspace_bytes(M, K, F, dt)))
    return outs


def backward(dH, G, U, Wg, Wu, act):
    (M, F), K, dt = dH.shape, Wg.shape[1], dp.dtype_of(dH)
    BG, BU = torch.full_like(dH, 7.0), torch.full_like(dH, 7.0)
    dX = torch.full((M, K), 7.0, dtype=dH.dtype, device=DEV)
    dp.dp_gated_ffn_backward(dH, G, U, Wg, Wu, dt, M, K, F, act, BG, BU, dX,
                             ws(dp.dp_gated_ffn_backward_workspace_bytes(M, K, F, dt)))
    return BG, BU, dX


@pytest.mark.parametrize("act", [dp.DP_ACT_SILU, dp.DP_ACT_GELU_TANH])
def test_slopes_between_the_tails(act):
    """act' where the gate comes near 1, to a few half steps u: dH = U = 1, so that BG is the slope and BU the value.

    With e = exp(-w) and p = 1 / (1 + e): w of the GELU form has 7 roundings (0.044715, three products, the sum, and
    2 sqrt(2/pi) with its product), SiLU's none, so e is off by E = 7 u |w| + 2 u (expf: one step); p by (1 - p) E, the sum
    and the quotient (2 u); q = p (1 - p) = e p^2 by |2 p - 1| E, both twice and two products (6 u), and the slope's second
    term q g w' by at most 10 u more (3 * 0.044715, six products and a sum, 2 sqrt(2/pi), its own), and the sum by u.
    Gates under the smallest normal value may be 0."""
    say("ffn slopes", act)
    u, tiny = R.U32, float(torch.finfo(torch.float32).tiny)
    G = torch.linspace(-14, 14, 2 ** 17, dtype=torch.float64).float().reshape(64, -1)
    one, W = torch.ones_like(G).to(DEV), torch.zeros((G.shape[1], 8), device=DEV)
    BG, BU, dX = backward(one, G.to(DEV), one, W, W, act)
    g = R.f64(G)
    w = g if act == dp.DP_ACT_SILU else 2 * R.C0 * (g + R.C1 * g ** 3)
    dw = np.ones_like(g) if act == dp.DP_ACT_SILU else 2 * R.C0 * (1 + 3 * R.C1 * g ** 2)
    e = np.exp(-w)
    p, q = 1 / (1 + e), e / (1 + e) / (1 + e)
    E = (0 if act == dp.DP_ACT_SILU else 7 * u) * np.abs(w) + 2 * u
    slope, ep = p + g * dw * q, (e * p) * E + 2 * u
    bound = p * ep + np.abs(g * dw) * (q * (np.abs(2 * p - 1) * E + 16 * u) + tiny) + u * np.abs(slope) + tiny
    R.within(BG, slope, 1.01 * bound, "slope")
    R.within(BU, g * p, 1.01 * np.abs(g) * (p * (ep + u) + tiny) + tiny, "value")
    assert (dX == 0).all()


# ------------------------------------------------------------------ fp32 by parts: over 64 rows

SIZES = [(70, 64, 40), (300, 264, 136), (520, 72, 1000), (300, 264, 2048)]


def inputs(M, K, F, seed=0):
    rng = np.random.default_rng(M + K + F + seed)
    t = lambda *s: torch.from_numpy(rng.standard_normal(s)).float()  # noqa: E731
    return t(M, K), t(F, K) / math.sqrt(K), t(F, K) / math.sqrt(K), t(M, F), t(M, F), t(M, F)


def bits(t):
    return t.view(torch.int32)


def check_forward(X, Wg, Wu, act):
    out = forward(X.to(DEV), Wg.to(DEV), Wu.to(DEV), act)
    want, bound = R.ffn_forward(act, R.f64(X), R.f64(Wg), R.f64(Wu), torch.float32)
    for name, g, w, b in zip("HGU", out, want, bound):
        R.within(g, w, b, name)
    return out


def check_backward(dH, G, U, Wg, Wu, act):
    BG, BU, dX = backward(dH.to(DEV), G.to(DEV), U.to(DEV), Wg.to(DEV), Wu.to(DEV), act)
    want, bound = R.ffn_backprops(act, R.f64(dH), R.f64(G), R.f64(U), torch.float32)
    for name, g, w, b in zip(("BG", "BU"), (BG, BU), want, bound):
        R.within(g, w, b, name)
    R.within(dX, *R.ffn_dx(R.f64(BG), R.f64(BU), R.f64(Wg), R.f64(Wu), torch.float32), "dX")
    return BG, BU, dX


@pytest.mark.parametrize("M,K,F", SIZES)
@pytest.mark.parametrize("value", [1e-30, 1e-36, 1e-42])
def test_f32_small_values_change_no_other_row(M, K, F, value):
    """One small value in a row or a feature: the others keep their bits."""
    say("ffn small value", M, K, F, value)
    act = dp.DP_ACT_GELU_TANH
    X, Wg, Wu, dH, G, U = inputs(M, K, F)
    out = check_forward(X, Wg, Wu, act)
    BG, BU, dX = check_backward(dH, G, U, Wg, Wu, act)
    m, f = M // 2, F // 3
    x, wg, dh = X.clone(), Wg.clone(), dH.clone()
    x[m, K // 3] = wg[f, K // 3] = dh[m, f] = value
    rows, feats = [i for i in range(M) if i != m], [i for i in range(F) if i != f]
    for a, b in zip(out, check_forward(x, Wg, Wu, act)):
        assert torch.equal(bits(a[rows]), bits(b[rows]))
    h, g, u = check_forward(X, wg, Wu, act)
    assert torch.equal(bits(h[:, feats]), bits(out[0][:, feats])) and torch.equal(bits(u), bits(out[2]))
    assert torch.equal(bits(g[:, feats]), bits(out[1][:, feats]))
    bg, bu, dx = check_backward(dh, G, U, Wg, Wu, act)
    assert torch.equal(bits(dx[rows]), bits(dX[rows]))
    cols = [i for i in range(K) if i != K // 3]
    assert torch.equal(bits(check_backward(dH, G, U, wg, Wu, act)[2][:, cols]), bits(dX[:, cols]))


@pytest.mark.parametrize("M,K,F", SIZES[1:])
@pytest.mark.parametrize("value", [math.nan, math.inf, 3e38])
def test_f32_other_tiles_keep_their_bits(M, K, F, value):
    """A value without parts turns its own tiles (128 rows, 64 features) over to the fp32 units, no others."""
    say("ffn tiles", M, K, F, value)
    act = dp.DP_ACT_SILU
    X, Wg, Wu, dH, G, U = inputs(M, K, F, 1)
    out = forward(X.to(DEV), Wg.to(DEV), Wu.to(DEV), act)
    dX = backward(dH.to(DEV), G.to(DEV), U.to(DEV), Wg.to(DEV), Wu.to(DEV), act)[2]
    m, f = 140, 70
    x, wg, dh = X.clone(), Wg.clone(), dH.clone()
    x[m, 5] = wg[f, 5] = dh[m, 5] = value
    rows, feats = [i for i in range(M) if i // 128 != m // 128], [i for i in range(F) if i // 64 != f // 64]
    for a, b in zip(out, forward(x.to(DEV), Wg.to(DEV), Wu.to(DEV), act)):
        assert torch.equal(bits(a[rows]), bits(b[rows]))
    for a, b in zip(out, forward(X.to(DEV), wg.to(DEV), Wu.to(DEV), act)):
        assert torch.equal(bits(a[:, feats]), bits(b[:, feats]))
    dx = backward(dh.to(DEV), G.to(DEV), U.to(DEV), Wg.to(DEV), Wu.to(DEV), act)[2]
    assert torch.equal(bits(dx[rows]), bits(dX[rows]))
    assert not dx[m].isfinite().any() if not math.isfinite(value) else True


@pytest.mark.parametrize("M,K,F", SIZES)
@pytest.mark.parametrize("deviation", [3.0, 12.0])
def test_f32_gelu_gates_in_the_tails(M, K, F, deviation):
    """A mean loss's gradient over gates whose slopes go down to nothing."""
    say("ffn gelu tails", M, K, F, deviation)
    X, Wg, Wu, dH, G, U = inputs(M, K, F, 2)
    BG, _, _ = check_backward(dH / 4096, G * deviation, U, Wg, Wu, dp.DP_ACT_GELU_TANH)
    assert (BG != 0).logical_and(BG.abs() < 2.0 ** -100).any() or M * F < 100000


@pytest.mark.parametrize("M,K,F", SIZES)
@pytest.mark.parametrize("value", [1e30, 1e32, 2e38, float(torch.finfo(torch.float32).max)])
def test_f32_single_large_values(M, K, F, value):
    """One large finite value with small partners, so that the sums stay finite: of parts, of parts that overflow, and of
    a magnitude that bf16 rounds to infinity."""
    say("ffn large value", M, K, F, value)
    act = dp.DP_ACT_SILU
    X, Wg, Wu, dH, G, U = inputs(M, K, F, 3)
    m, k, f = M - 1, K // 2, F - 1
    X[m, k] = value
    Wg[:, k] *= 1e-20
    Wu[:, k] *= 1e-20
    out = check_forward(X, Wg, Wu, act)
    assert all(t.isfinite().all() for t in out) and out[1][m].abs().max() > 1e-22 * value
    X, Wg, Wu, dH, G, U = inputs(M, K, F, 4)
    dH[m, f] = value                                         # BG = about -0.3 value, BU = 0.2 value
    G[m, f], U[m, f] = -1.0, -4.0
    Wg[f] *= 1e-20
    Wu[f] *= 1e-20
    if value > 1e38:
        U[m, f] = 1.0
    BG, BU, dX = check_backward(dH, G, U, Wg, Wu, act)
    assert all(t.isfinite().all() for t in (BG, BU, dX)) and BU[m, f].abs() > 0.2 * value


@pytest.mark.parametrize("M,K,F", SIZES)
def test_f32_large_sums(M, K, F):
    """Ordinary rows and weights whose products pass what the scaled parts' sums hold (2^80)."""
    say("ffn large sums", M, K, F)
    X, Wg, Wu, dH, G, U = inputs(M, K, F, 5)
    out = check_forward(X * 1e13, Wg * 1e13, Wu * 1e-13, dp.DP_ACT_SILU)
    assert all(t.isfinite().all() for t in out) and out[1].abs().max() > 2.0 ** 80
    dX = check_backward(dH * 1e13, G, U, Wg * 1e13, Wu * 1e13, dp.DP_ACT_SILU)[2]
    assert dX.isfinite().all() and dX.abs().max() > 2.0 ** 80
