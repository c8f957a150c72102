"""Attention on the GPU at the ends of its range: scores that fp32 differences no longer resolve, gradients that cancel,
padding that holds anything, lists of tiles longer than one group."""
import sys

import numpy as np
import pytest
import torch

from lm_ref import f64
from paper_2109_12298_amd import binding as dp
from test_gpu_attention import DEV, Case, ws_of

pytestmark = pytest.mark.gpu


def say(*a):
    print("[case]", *a, file=sys.stderr, flush=True)


# ---------------------------------------------------------------------------
# large scores
# ---------------------------------------------------------------------------

# One workgroup's waves, keys split over workgroups, blocks of 128 rows, row by row.  The last wave has one row: where one row's
# sums are not finite, all of a wave's are formed again.
SHAPES = {  # N, Tq, Tk, Hq, Hk, D
    "small": (20, 33, 100, 2, 2, 64), "split": (30, 1, 2000, 2, 2, 64), "blocks": (16, 65, 65, 16, 16, 64), "rows": (2, 33, 60, 2, 1, 136)}


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["plain", "slopes", "cap", "both"])
@pytest.mark.parametrize("shape", list(SHAPES))
def test_scores_past_the_resolution_of_their_differences(shape, kind, dt):
    """Scores of 2^29 to 2^37, exact in fp32: the weight belongs to the largest ones.

    Q and K are whole numbers, so that q.k is exact; scales, biases and caps are powers of two.  Scores of different keys differ by
    2^18 at the least (2^28 times a whole number, less 2^18 times a distance below 2^10), the steps' roundings are below 2^14 (some
    2^-24 of 2^37), so that all keys but the largest have weight exp(-2^17) = 0; equal ones (without biases) share it."""
    say("large", shape, kind, dt)
    N, Tq, Tk, Hq, Hk, D = SHAPES[shape]
    last = shape == "split"
    c = Case(N, Tq, Tk, Hq, Hk, D, dt, causal=True, last=last, scale=2.0 ** 28, cap=2.0 ** 59 if kind in ("cap", "both") else 0.0, seed=21)
    rng = np.random.default_rng(22)
    whole = lambda x: torch.from_numpy(rng.integers(-3, 4, x.shape)).to(c.tt)  # noqa: E731
    c.Q, c.K = whole(c.Q), whole(c.K)
    if last:                                          # the same keys for every wave of every workgroup
        c.K = c.K[:, :32].repeat(1, Tk // 32 + 1, 1, 1)[:, :Tk].contiguous()
    far = np.zeros((Tq, Tk))
    if kind in ("slopes", "both"):
        c.slopes = np.full(Hq, 2.0 ** 18, dtype=np.float32)
        far = c.mask.far[0] % 1024 * 2.0 ** 18 if Tk <= 1024 else None
        if far is None:                               # distances past 2^10: biases as small as keep them below one step of q.k
            c.slopes[:] = 2.0 ** 16
            far = c.mask.far[0] * 2.0 ** 16
    out, lse = c.run(backward=False)
    Q, K, V = f64(c.Q), f64(c.K), f64(c.V)
    for n in range(N):
        for h in range(Hq):
            kv = h // (Hq // Hk)
            s = np.where(c.mask.see[n], 2.0 ** 28 * (Q[n, :, h] @ K[n, :, kv].T) - far, -np.inf)
            top = s.max(1, keepdims=True)
            p = (s == top) / (s == top).sum(1, keepdims=True)
            want = p @ V[n, :, kv]
            # equal weights, their sum and quotient: 4 half steps of fp32 and one of each addition (Tk at most), one of the output's
            half = 2.0 ** -8 if dt == "bf16" else 2.0 ** -24
            size = p @ np.abs(V[n, :, kv])
            got = f64(out["O"][n, :, h])
            assert (np.abs(got - want) <= (4 + 2 * (s == top).sum(1, keepdims=True)) * 2.0 ** -24 * size + half * np.abs(want) + 2 * (
                half if dt == "bf16" else 0) * size).all(), (n, h)
            l = top[:, 0] + np.log((s == top).sum(1))
            # the score's steps, factors log2 e and ln 2: 16 half steps; the capped score's polynomial 10 more
            assert (np.abs(f64(lse[n, h]) - l) <= 32 * 2.0 ** -24 * (np.abs(l) + far.max())).all(), (n, h)
