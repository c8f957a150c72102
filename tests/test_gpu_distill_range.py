"""The distillation loss on the GPU at the ends of its range: large quotients of logits and temperatures, rows of the type's
lowest value, rows past what registers hold."""
import sys

import numpy as np
import pytest
import torch

from lm_ref import f64, half_step
from paper_2109_12298_amd import binding as dp
from test_gpu_distill import TT, draw, run

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def say(*a):
    print("[case]", *a, file=sys.stderr, flush=True)


def softmax(x):
    """q and log q of x [V], in 64 bits."""
    with np.errstate(invalid="ignore"):
        d = x - x.max()
    e = np.exp(d)
    return e / e.sum(), d - np.log(e.sum())


def expect(z, ids, logits, label, alpha, tau, w, dt):
    """loss and dZ of one position in 64 bits, with bounds.

    A class' exponent is a difference, whose rounding is half a step of itself, times a constant that is off by half a step (1 / tau
    and log2 e: two): 4 half steps of |z - max| / tau; exp2 takes 2 more.  A sum over V is formed by at least 64 threads at
    once, in trees over waves: V / 1024 + 8 * 16 terms (a thread of a long row; a short row's 16 pieces of 8) one after another, and
    2 half steps of rescaling, with its exponent's, at most 24 times."""
    V = len(z)
    n = V / 1024 + 8 * 20 + 16 + 48
    loss, dz, el, ed = 0.0, np.zeros(V), 0.0, np.zeros(V)

    def part(t):
        q, lq = softmax(z / t)
        far = np.where(np.isfinite(z), z.max() - z, 0.0) / t
        rel = 2 * U * (4 * far + 2 + n) + 2 * U * (4 * (q * far).sum() + 2 + n)
        return q, lq, far, rel
    used = ids >= 0
    if alpha > 0 and used.any():
        k, t = ids[used], logits[used].astype(np.float64)
        P, lP = softmax(t / tau)
        q, lq, far, rel = part(tau)
        tf = (t.max() - t) / tau
        rp = 2 * U * (4 * tf + 4 * (P * tf).sum() + 8 + len(k))
        terms = P * (lP - lq[k])
        loss += alpha * tau ** 2 * terms.sum()
        el += alpha * tau ** 2 * (np.abs(terms) * (rp + 2 * U * len(k)) + P * (
            2 * U * (4 * (tf + np.abs(lP)) + 4 * (far[k] + np.abs(lq[k])) + 8) + rp + rel[k])).sum()
        dz += alpha * tau * q
        np.add.at(dz, k, -alpha * tau * P)
        ed += alpha * tau * q * (rel + 4 * U)
        np.add.at(ed, k, alpha * tau * P * (rp + (4 + len(k)) * U))
    if label is not None and 0 <= label < V and alpha < 1:
        q, lq, far, rel = part(1.0)
        loss -= (1 - alpha) * lq[label]
        el += (1 - alpha) * (2 * U * (4 * (far[label] + abs(lq[label])) + 8) + rel[label])
        dz += (1 - alpha) * q
        ed += (1 - alpha) * q * (rel + 4 * U)
        dz[label] -= 1 - alpha
        ed[label] += (1 - alpha) * 4 * U
    h = half_step(TT[dt])
    el, ed = abs(w) * el + 4 * U * abs(w * loss), abs(w) * ed + 4 * U * np.abs(w * dz)
    return w * loss, w * dz, el + 1e-37, ed + h * (np.abs(w * dz) + ed) + 1e-37


def check(Z, ids, logits, labels, alpha, tau, weight, dt):
    loss, dz, status = run(Z, ids, logits, labels, alpha, tau, weight, dt)
    assert status == 0
    loss, dz, z = f64(loss), f64(dz), f64(Z)
    for m in range(len(z)):
        l, d, el, ed = expect(z[m], ids[m], logits[m], labels[m], alpha, tau, float(weight[m]), dt)
        assert abs(loss[m] - l) <= el, (m, loss[m], l, el)
        assert (np.abs(dz[m] - d) <= ed).all(), (m, float((np.abs(dz[m] - d) / ed).max()))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("V", [300, 5000, 33001, 170001])
@pytest.mark.parametrize("tau,spread", [(2.0 ** -20, 3000.0), (2.0 ** -20, 1.0), (2.0 ** -10, 1e7), (1.0, 1e12), (2.0 ** 20, 1e30)])
def test_large_quotients(tau, spread, V, dt):
    """Logits that are billions of temperatures large: one class has everything, or two that are alike share it."""
    say("quotients", tau, spread, V, dt)
    Z, ids, logits, labels, weight = draw(4, V, 9, dt, seed=3, spread=spread)
    Z[1] = Z[1].abs()
    Z[2] = -Z[2].abs() - spread
    Z[3, V // 2] = Z[3, V // 3] = 5 * spread
    check(Z, ids, logits, labels, 0.4, tau, weight, dt)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("V", [37, 4099, 100001, 170001])
def test_rows_of_the_lowest_value(V, dt):
    """Every class, or all but two, at the type's lowest value: the softmax is even over what is the largest."""
    say("lowest", V, dt)
    Z, ids, logits, labels, weight = draw(3, V, 5, dt, seed=4, ragged=False)
    low = float(torch.finfo(TT[dt]).min)
    labels[:], ids[1] = V // 2, np.arange(5)
    Z[:2] = low
    Z[2, 5:] = low
    ids[2], labels[2] = np.arange(5), 3
    for tau in (1.0, 0.5, 8.0):
        check(Z, ids, logits, labels, 0.5, tau, weight, dt)
    Z[0], Z[1] = -low, low
    Z[1, 7] = -low                                     # differences past the type's range
    ids[1], labels[1] = 7, 7
    check(Z, ids, logits, labels, 0.5, 1.0, weight, dt)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("V", [20011, 100001, 200003])
@pytest.mark.parametrize("spread,tau,offset", [(30.0, 0.7, 0.0), (200.0, 0.7, 0.0), (1e4, 1.0, 0.0), (1e4, 1e4, 0.0), (2.0, 1.0, 1000.0)])
def test_long_rows_keep_their_bits(spread, tau, offset, V, dt):
    """Sums that threads take from maxima of their own."""
    say("long", spread, tau, offset, V, dt)
    Z, ids, logits, labels, weight = draw(2, V, 9, dt, seed=5, spread=spread)
    Z += offset
    labels = np.abs(labels)
    check(Z, ids, logits, labels, 0.4, tau, weight, dt)


@pytest.mark.parametrize("V", [50, 9000, 100001])
def test_labels_that_have_no_share_are_looked_at(V):
    """alpha = 1: a label adds nothing to the loss, and one past the classes is flagged all the same (but not at weight 0)."""
    Z, ids, logits, labels, weight = draw(3, V, 5, "f32", ragged=False)
    labels[:] = [1, V, 2]
    loss, dz, status = run(Z, ids, logits, labels, 1.0, 2.0, weight, "f32")
    assert status == dp.DP_FLAG_BAD_INDEX
    want, dwant, none = run(Z, ids, logits, None, 1.0, 2.0, weight, "f32")
    assert none == 0 and torch.equal(loss, want) and torch.equal(dz, dwant)
    weight[1] = 0.0
    assert run(Z, ids, logits, labels, 1.0, 2.0, weight, "f32")[2] == 0


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("V", [60, 9001, 100001])
@pytest.mark.parametrize("top", [1.0, 1e9])
def test_targets_at_the_lowest_value(top, V, dt):
    """A teacher's class, or the label, that the row masks with the type's lowest value: a loss of that size, not an infinity."""
    say("target", top, V, dt)
    Z, ids, logits, labels, weight = draw(3, V, 4, dt, seed=6, ragged=False)
    Z *= top
    low = float(torch.finfo(TT[dt]).min)
    ids[:], labels[:], weight[:] = [3, 9, 20, 30], 40, 0.5
    Z[0, 9] = low
    Z[1, 40] = low
    Z[2, 3] = Z[2, 30] = Z[2, 40] = low
    check(Z, ids, logits, labels, 0.5, 1.0, weight, dt)
