"""The gated feed-forward block's forward and backward on the GPU, against the 64-bit definitions of lm_ref, against
autograd in 64 bits and against differences."""
import math
import sys

import numpy as np
import pytest
import torch

import lm_ref as R
from paper_2109_12298_amd import binding as dp

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"f32": (torch.float32, dp.DP_F32), "bf16": (torch.bfloat16, dp.DP_BF16)}


def say(*a):
    print("[case]", *a, file=sys.stderr, flush=True)


def unaligned(x, by):
    buf = torch.empty(x.numel() + 16, dtype=x.dtype, device=DEV)
    v = buf[by:by + x.numel()].view(x.shape)
    v.copy_(x)
    return v


def ws(n):
    return torch.full((max(n, 16),), 0xFF, dtype=torch.uint8, device=DEV)       # NaN in every type


def forward(X, Wg, Wu, act, save=True, outs=None):
    (M, K), F, dt = X.shape, Wg.shape[0], dp.dtype_of(X)
    if outs is None:
        outs = [torch.full((M, F), 7.0, dtype=X.dtype, device=DEV) if k == 0 or save else None for k in range(3)]
    dp.dp_gated_ffn_forward(X, Wg, Wu, dt, M, K, F, act, *outs, ws(dp.dp_gated_ffn_forward_workspace_bytes(M, K, F, dt)))
    return outs


def backward(dH, G, U, Wg, Wu, act, want_dx=True, BG=None, BU=None):
    (M, F), K, dt = dH.shape, Wg.shape[1], dp.dtype_of(dH)
    BG = torch.full_like(dH, 7.0) if BG is None else BG
    BU = torch.full_like(dH, 7.0) if BU is None else BU
    dX = torch.full((M, K), 7.0, dtype=dH.dtype, device=DEV) if want_dx else None
    dp.dp_gated_ffn_backward(dH, G, U, Wg, Wu, dt, M, K, F, act, BG, BU, dX,
                             ws(dp.dp_gated_ffn_backward_workspace_bytes(M, K, F, dt)))
    return BG, BU, dX


def weights(rng, F, K, tt):
    return [torch.from_numpy(rng.standard_normal((F, K)) / math.sqrt(K)).to(tt) for _ in range(2)]


# below, at and above the tile sizes; rows of one to many; features that are no multiple of anything
SIZES = [(1, 1, 1), (1, 64, 64), (1, 500, 77), (2, 256, 136), (3, 5, 7), (4, 8, 8), (5, 1032, 40), (8, 96, 256),
         (15, 72, 24), (16, 512, 130), (17, 40, 264), (31, 128, 128), (33, 128, 200), (48, 264, 96), (64, 64, 64),
         (65, 100, 130), (100, 192, 328), (127, 136, 72), (128, 256, 128), (129, 320, 129), (200, 77, 300),
         (256, 256, 256), (257, 136, 264), (300, 1000, 520), (520, 72, 1000), (1000, 512, 264),
         (70, 1, 2), (66, 16, 3), (90, 17, 33), (130, 33, 50), (70, 50, 17), (97, 65, 80), (260, 82, 97), (150, 140, 3000),
         (90, 2000, 70), (20, 700, 900), (64, 130, 2100)]


@pytest.mark.parametrize("M,K,F", SIZES)
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("act", [dp.DP_ACT_SILU, dp.DP_ACT_GELU_TANH])
def test_forward(M, K, F, dt, act):
    say("ffn forward", M, K, F, dt, act)
    rng = np.random.default_rng(M + 100 * K + F)
    tt, _ = DT[dt]
    X, (Wg, Wu) = torch.from_numpy(rng.standard_normal((M, K)) * 2).to(tt), weights(rng, F, K, tt)
    got = forward(X.to(DEV), Wg.to(DEV), Wu.to(DEV), act)
    want, bound = R.ffn_forward(act, R.f64(X), R.f64(Wg), R.f64(Wu), tt)
    for name, g, w, b in zip("HGU", got, want, bound):
        R.within(g, w, b, name)
    alone, _, _ = forward(X.to(DEV), Wg.to(DEV), Wu.to(DEV), act, save=False)
    assert torch.equal(alone, got[0])                          # H does not depend on what else is kept


@pytest.mark.parametrize("M,K,F", SIZES)
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("act", [dp.DP_ACT_SILU, dp.DP_ACT_GELU_TANH])
def test_backward(M, K, F, dt, act):
    say("ffn backward", M, K, F, dt, act)
    rng = np.random.default_rng(M + 100 * K + F + 1)
    tt, _ = DT[dt]
    dH, G, U = [torch.from_numpy(rng.standard_normal((M, F)) * s).to(tt) for s in (0.1, 2.0, 1.0)]
    Wg, Wu = weights(rng, F, K, tt)
    dHg, Gg, Ug, Wgg, Wug = [t.to(DEV) for t in (dH, G, U, Wg, Wu)]
    BG, BU, dX = backward(dHg, Gg, Ug, Wgg, Wug, act)
    (wg, wu), (bg, bu) = R.ffn_backprops(act, R.f64(dH), R.f64(G), R.f64(U), tt)
    R.within(BG, wg, bg, "BG")
    R.within(BU, wu, bu, "BU")
    wx, bx = R.ffn_dx(R.f64(BG), R.f64(BU), R.f64(Wg), R.f64(Wu), tt)            # from the backprops as stored
    R.within(dX, wx, bx, "dX")
    b2, u2, none = backward(dHg, Gg, Ug, Wgg, Wug, act, want_dx=False)
    assert none is None and torch.equal(b2, BG) and torch.equal(u2, BU)
    # the backprops in place of what they are formed from
    g3, u3, x3 = backward(dHg, Gg, Ug, Wgg, Wug, act, BG=Gg, BU=Ug)
    assert torch.equal(g3, BG) and torch.equal(u3, BU) and torch.equal(x3, dX)


@pytest.mark.parametrize("M,K,F", [(1, 136, 264), (7, 64, 72), (40, 200, 136), (130, 136, 264), (300, 264, 136)])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("by", [1, 2, 4])
def test_unaligned(M, K, F, dt, by):
    """Arrays that start between 16-byte boundaries, and guards beside the outputs."""
    say("ffn unaligned", M, K, F, dt, by)
    rng = np.random.default_rng(by)
    tt, ct = DT[dt]
    act = dp.DP_ACT_SILU
    X, (Wg, Wu) = torch.from_numpy(rng.standard_normal((M, K))).to(tt), weights(rng, F, K, tt)
    dH = torch.from_numpy(rng.standard_normal((M, F))).to(tt)
    bufs = [torch.full((M * F + 32,), 7.0, dtype=tt, device=DEV) for _ in range(3)]
    outs = [b[by:by + M * F].view(M, F) for b in bufs]
    forward(unaligned(X, by), unaligned(Wg, by), unaligned(Wu, by), act, outs=outs)
    want, bound = R.ffn_forward(act, R.f64(X), R.f64(Wg), R.f64(Wu), tt)
    for g, w, b in zip(outs, want, bound):
        R.within(g, w, b)
    assert all((b[:by] == 7).all() and (b[by + M * F:] == 7).all() for b in bufs)
    buf = torch.full((M * K + 32,), 7.0, dtype=tt, device=DEV)
    dX = buf[by:by + M * K].view(M, K)
    BG, BU = torch.empty_like(outs[0]), torch.empty_like(outs[0])
    dp.dp_gated_ffn_backward(unaligned(dH, by), outs[1], outs[2], unaligned(Wg, by), unaligned(Wu, by), ct, M, K, F, act, BG,
                             BU, dX, ws(dp.dp_gated_ffn_backward_workspace_bytes(M, K, F, ct)))
    wx, bx = R.ffn_dx(R.f64(BG), R.f64(BU), R.f64(Wg), R.f64(Wu), tt)
    R.within(dX, wx, bx)
    assert (buf[:by] == 7).all() and (buf[by + M * K:] == 7).all()


@pytest.mark.parametrize("M,K,F", [(2, 64, 64), (20, 136, 40), (300, 136, 264), (260, 70, 33)])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_nonfinite_rows_stay_apart(M, K, F, dt, value):
    """A NaN or infinity in one row reaches that row's outputs, all of them, and no other's (whose sums may be formed
    by another kernel then: both meet the bound)."""
    say("ffn nonfinite", M, K, F, dt, value)
    rng = np.random.default_rng(M)
    tt, _ = DT[dt]
    X, (Wg, Wu) = torch.from_numpy(rng.standard_normal((M, K))).to(tt), weights(rng, F, K, tt)
    want, bound = R.ffn_forward(dp.DP_ACT_SILU, R.f64(X), R.f64(Wg), R.f64(Wu), tt)
    Wg, Wu = Wg.to(DEV), Wu.to(DEV)
    bad = M // 2
    Xb = X.clone()
    Xb[bad, K // 3] = value
    rest = [m for m in range(M) if m != bad]
    out = forward(Xb.to(DEV), Wg, Wu, dp.DP_ACT_SILU)
    for g, w, b in zip(out, want, bound):
        R.within(g[rest], w[rest], b[rest])
    assert not out[1][bad].isfinite().any() and not out[2][bad].isfinite().any()
    _, G, U = forward(X.to(DEV), Wg, Wu, dp.DP_ACT_SILU)
    dH = torch.from_numpy(rng.standard_normal((M, F))).to(tt)
    dH[bad, F // 3] = value
    BG, BU, dX = backward(dH.to(DEV), G, U, Wg, Wu, dp.DP_ACT_SILU)
    assert not dX[bad].isfinite().any() and not BU[bad, F // 3].isfinite().any()
    wx, bx = R.ffn_dx(R.f64(BG[rest]), R.f64(BU[rest]), R.f64(Wg), R.f64(Wu), tt)
    R.within(dX[rest], wx, bx)


@pytest.mark.parametrize("value", [1e-36, 1e-31, 1e-30, 2e38])
@pytest.mark.parametrize("M,K,F", [(70, 64, 40), (300, 264, 136)])
def test_f32_values_without_parts(M, K, F, value):
    """fp32 values of the ends of the range, which the three-part product leaves to another kernel: one of them in X, in
    a weight, in a backprop."""
    say("ffn range", M, K, F, value)
    rng = np.random.default_rng(K)
    X, (Wg, Wu) = torch.from_numpy(rng.standard_normal((M, K))).float(), weights(rng, F, K, torch.float32)
    dH = torch.from_numpy(rng.standard_normal((M, F))).float()
    for where in ("X", "Wu", "dH"):
        x, wu, dh = X.clone(), Wu.clone(), dH.clone()
        if where == "X":
            x[3] = x[3] * value / x[3].abs().max() / 4
            wu, dh = wu.clone(), dh.clone()
        elif where == "Wu":
            wu[F - 1] = wu[F - 1] * value / wu[F - 1].abs().max() / (4 * K)
        else:
            dh[M - 1] = dh[M - 1] * value / dh[M - 1].abs().max() / (16 * F)
        out = forward(x.to(DEV), Wg.to(DEV), wu.to(DEV), dp.DP_ACT_SILU)
        want, bound = R.ffn_forward(dp.DP_ACT_SILU, R.f64(x), R.f64(Wg), R.f64(wu), torch.float32)
        fine = np.abs(want[0]) < 1e38                          # H = act(G) U may leave the range of fp32
        for g, w, b in zip(out, want, bound):
            R.within(g[torch.from_numpy(fine)], w[fine], b[fine])
        G, U = torch.from_numpy(want[1]).float().clamp(-8, 8), torch.from_numpy(want[2]).float().clamp(-8, 8)
        BG, BU, dX = backward(dh.to(DEV), G.to(DEV), U.to(DEV), Wg.to(DEV), wu.to(DEV), dp.DP_ACT_SILU)
        wx, bx = R.ffn_dx(R.f64(BG), R.f64(BU), R.f64(Wg), R.f64(wu), torch.float32)
        fine = np.abs(wx) + bx < 1e38
        R.within(dX[torch.from_numpy(fine)], wx[fine], bx[fine])


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("act", [dp.DP_ACT_SILU, dp.DP_ACT_GELU_TANH])
def test_large_and_small_gates(dt, act):
    """Gates far into both tails: no overflow turns into NaN, and the slopes end at 0 and 1."""
    say("ffn tails", dt, act)
    tt, _ = DT[dt]
    g = torch.tensor([0.0, -0.0, 1e-30, -1e-30, 5, -5, 30, -30, 88, -88, 105, -105, 1e4, -1e4, 1e13, -1e13, 1e30, -1e30],
                     dtype=torch.float64).to(tt)
    G = g.repeat(3, 1)
    one = torch.ones_like(G)
    F = G.shape[1]
    W = torch.zeros((F, 8), dtype=tt, device=DEV)
    BG, BU, dX = backward(one.to(DEV), G.to(DEV), one.to(DEV), W, W, act)
    (wg, wu), (bg, bu) = R.ffn_backprops(act, np.ones(G.shape), np.clip(R.f64(G), -200, 200), np.ones(G.shape), tt)
    big = np.abs(R.f64(G)) > 200
    wu = np.where(big, np.maximum(R.f64(G), 0), wu)
    bu = np.where(big, R.U32 * np.abs(wu), bu)
    R.within(BG, wg, bg)
    R.within(BU, wu, bu)
    assert (dX == 0).all()


def test_gradient_against_autograd_and_differences():
    """The chain forward -> backward in fp32 against 64-bit autograd, and along a direction against differences."""
    say("ffn autograd")
    rng = np.random.default_rng(11)
    M, K, F = 37, 48, 52
    X, (Wg, Wu) = torch.from_numpy(rng.standard_normal((M, K))).float(), weights(rng, F, K, torch.float32)
    dH = torch.from_numpy(rng.standard_normal((M, F))).float()
    for act in (dp.DP_ACT_SILU, dp.DP_ACT_GELU_TANH):
        fn = (lambda g: g * torch.sigmoid(g)) if act == dp.DP_ACT_SILU else \
            (lambda g: torch.nn.functional.gelu(g, approximate="tanh"))
        x, wg, wu = [t.double().requires_grad_(True) for t in (X, Wg, Wu)]
        (fn(x @ wg.t()) * (x @ wu.t()) * dH.double()).sum().backward()
        _, G, U = forward(X.to(DEV), Wg.to(DEV), Wu.to(DEV), act)
        BG, BU, dX = backward(dH.to(DEV), G, U, Wg.to(DEV), Wu.to(DEV), act)
        # chains of K, then 2 F, then M fp32 terms with everything of order 1 to 10: 1e-5 of the largest value is
        # over a hundred times u = 6e-8, and sqrt(K + 2 F + M) u times the condition of the sums (about 4) stays under
        for got, want in ((dX, x.grad), (BG.double().t() @ X.to(DEV).double(), wg.grad),
                          (BU.double().t() @ X.to(DEV).double(), wu.grad)):
            assert (got.cpu().double() - want).abs().max() <= 1e-5 * want.abs().max()
        # the loss sum(dH * H) along a direction of X, by central differences of the kernel's own forward in fp32: the
        # step h = 2^-7 leaves h^2 / 6 of the third derivative and 2^-24 |loss terms| / h of rounding, both under 1e-3
        # of the sum of the terms' sizes
        dirn, h = torch.from_numpy(rng.standard_normal((M, K))).float(), 2.0 ** -7
        up, down = [forward((X + s * h * dirn).to(DEV), Wg.to(DEV), Wu.to(DEV), act)[0].double().cpu() for s in (1, -1)]
        terms = dH.double() * (up - down) / (2 * h)
        assert abs(terms.sum() - (dX.cpu().double() * dirn.double()).sum()) <= 1e-3 * terms.abs().sum()


def test_empty():
    say("ffn empty")
    W = torch.zeros((4, 8), device=DEV)
    assert forward(torch.empty((0, 8), device=DEV), W, W, 0)[0].shape == (0, 4)
    e = torch.empty((0, 4), device=DEV)
    assert backward(e, e.clone(), e.clone(), W, W, 0, BG=None)[2].shape == (0, 8)


@pytest.mark.parametrize("M,K,F", [(20, 64, 2048), (300, 264, 136)])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_backprops_alone_take_no_workspace(M, K, F, dt):
    """Without dX nothing but the elementwise pass runs: no workspace, no weights."""
    say("ffn backprops alone", M, K, F, dt)
    rng = np.random.default_rng(M)
    tt, ct = DT[dt]
    dH, G, U = [torch.from_numpy(rng.standard_normal((M, F))).to(tt) for _ in range(3)]
    BG, BU = [torch.full((M, F), 7.0, dtype=tt, device=DEV) for _ in range(2)]
    dp.dp_gated_ffn_backward(dH.to(DEV), G.to(DEV), U.to(DEV), None, None, ct, M, K, F, dp.DP_ACT_SILU, BG, BU)
    (wg, wu), (bg, bu) = R.ffn_backprops(dp.DP_ACT_SILU, R.f64(dH), R.f64(G), R.f64(U), tt)
    R.within(BG, wg, bg, "BG")
    R.within(BU, wu, bu, "BU")
