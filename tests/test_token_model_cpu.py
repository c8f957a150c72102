"""Refusals of rotary positions, attention and the distillation loss on the host (nothing is enqueued; no GPU needed), and
the tests' own definitions against differences."""
import ctypes
import math

import numpy as np
import pytest
import torch

import token_model_ref as ref
from paper_2109_12298_amd import binding as dp

# addresses below are never dereferenced: every call fails validation first, or has nothing to do
FAKE = 0x10000


def code_of(fn, *a, **k):
    try:
        fn(*a, stream=0, **k)
    except dp.DPError as e:
        return e.code
    return dp.DP_OK


def test_rotary_refusals():
    def call(X=FAKE, dt=dp.DP_F32, N=2, T=3, H=2, D=8, ldx=16, pos=FAKE, sections=(2, 2), freq=FAKE, layout=0, inverse=0, Y=2 * FAKE,
             ldy=16):
        return code_of(dp.dp_rotary, X, dt, N, T, H, D, ldx, pos, list(sections), freq, layout, inverse, Y, ldy)

    assert call(dt=5) == dp.DP_EDTYPE
    for bad in (dict(N=-1), dict(T=-1), dict(H=0), dict(D=0), dict(ldx=15), dict(ldy=15), dict(sections=()), dict(sections=(1,) * 5),
                dict(sections=(3, 2)), dict(sections=(-1, 2)), dict(layout=2), dict(X=None), dict(Y=None), dict(pos=None),
                dict(freq=None), dict(X=FAKE + 2), dict(Y=FAKE + 1), dict(pos=FAKE + 4), dict(freq=FAKE + 4), dict(Y=FAKE, ldy=20)):
        assert call(**bad) == dp.DP_EINVAL, bad
    for much in (dict(N=2 ** 20, T=2 ** 11), dict(N=2 ** 62, T=4), dict(D=1025, ldx=4096, ldy=4096), dict(H=2 ** 20, ldx=2 ** 25, ldy=2 ** 25),
                 dict(ldx=2 ** 31)):
        assert call(**much) == dp.DP_EUNSUPPORTED, much
    assert call(N=0, X=None, Y=None, pos=None, freq=None) == dp.DP_OK
    L = dp.lib()
    assert L.dp_rotary(FAKE, 0, 2, 3, 2, 8, 16, FAKE, None, 1, FAKE, 0, 0, 2 * FAKE, 16, None) == dp.DP_EINVAL


GOOD = dict(dt=dp.DP_F32, N=2, Tq=3, Tk=4, Hq=4, Hk=2, D=8, scale=0.5)


def test_attention_refusals():
    L = dp.lib()

    def fwd(Q=FAKE, K=FAKE, V=FAKE, O=FAKE, lse=FAKE, ws=FAKE, n=1 << 40, a=None, **kw):
        a = dp.make_attention(**{**GOOD, **kw}) if a is None else a
        return L.dp_attention_forward(ctypes.addressof(a), Q, K, V, O, lse, ws, n, None)

    def bwd(Q=FAKE, K=FAKE, V=FAKE, O=FAKE, lse=FAKE, dO=FAKE, dQ=FAKE, dK=FAKE, dV=2 * FAKE, ws=FAKE, n=1 << 40, **kw):
        a = dp.make_attention(**{**GOOD, **kw})
        return L.dp_attention_backward(ctypes.addressof(a), Q, K, V, O, lse, dO, dQ, dK, dV, ws, n, None)

    for call in (fwd, bwd):
        assert call(dt=7) == dp.DP_EDTYPE
        for bad in (dict(N=-1), dict(Tq=-1), dict(Tk=-1), dict(Hk=0), dict(Hq=0), dict(Hq=3), dict(D=0), dict(flags=4), dict(scale=math.nan),
                    dict(scale=math.inf), dict(softcap=-1.0), dict(softcap=math.inf), dict(softcap=1e-19), dict(softcap=math.nan), dict(scale=1e19), dict(prefix=FAKE), dict(ldq=31), dict(ldk=15),
                    dict(ldv=15), dict(ldo=31), dict(slopes=FAKE + 2), dict(lens=FAKE + 1), dict(docs=FAKE + 2), dict(Q=None), dict(K=None),
                    dict(V=None), dict(O=None), dict(Q=FAKE + 2), dict(V=FAKE + 1), dict(lse=FAKE + 2)):
            assert call(**bad) == dp.DP_EINVAL, bad
        for much in (dict(D=257), dict(Tq=2 ** 24), dict(Tk=2 ** 24), dict(N=2 ** 31), dict(N=2 ** 23, Tk=33), dict(N=2 ** 22, Tq=1),
                     dict(Hq=2 ** 23, ldq=2 ** 40, ldo=2 ** 40), dict(ldq=2 ** 22), dict(ldk=2 ** 22), dict(ldv=2 ** 22), dict(ldo=2 ** 22)):
            assert call(**much) == dp.DP_EUNSUPPORTED, much
        assert call(N=0, Q=None, K=None, V=None, O=None, lse=None, ws=None, n=0) == dp.DP_OK
    for k in ("lse", "dO", "dQ", "dK", "dV"):
        assert bwd(**{k: None}) == dp.DP_EINVAL, k
    assert bwd(dV=FAKE) == dp.DP_EINVAL                                # both key gradients into one array
    assert L.dp_attention_forward(None, FAKE, FAKE, FAKE, FAKE, None, None, 0, None) == dp.DP_EINVAL
    for size, call in ((dp.dp_attention_forward_workspace_bytes, fwd), (dp.dp_attention_backward_workspace_bytes, bwd)):
        assert size(dp.make_attention(**{**GOOD, "D": 0})) == 0 and size(dp.make_attention(**{**GOOD, "N": 0})) == 0
        for kw in (dict(Tq=1, Tk=5000), dict(Tq=500, Tk=500), dict(Tq=1, Tk=5000, D=128, dt=dp.DP_BF16), dict(Tq=300, Tk=300, dt=dp.DP_BF16)):
            n = size(dp.make_attention(**{**GOOD, **kw}))
            if n > 0:
                assert call(n=n - 1, **kw) == dp.DP_EINVAL and call(ws=None, **kw) == dp.DP_EINVAL
                assert call(ws=FAKE + 8, **kw) == dp.DP_EINVAL


def test_distill_refusals():
    def call(Z=FAKE, dt=dp.DP_F32, M=2, V=9, ids=FAKE, logits=FAKE, K=3, labels=None, alpha=0.5, tau=1.0, weight=None, loss=FAKE,
             dZ=FAKE):
        return code_of(dp.dp_distill_loss, Z, dt, M, V, ids, logits, K, labels, alpha, tau, weight, loss, dZ)

    assert call(dt=2) == dp.DP_EDTYPE
    for bad in (dict(M=-1), dict(K=-1), dict(V=0), dict(alpha=-0.1), dict(alpha=1.1), dict(alpha=math.nan), dict(tau=0.0), dict(tau=-1.0),
                dict(tau=math.nan), dict(tau=math.inf), dict(tau=1e-7), dict(tau=2e6), dict(Z=None), dict(loss=None), dict(ids=None), dict(logits=None), dict(Z=FAKE + 2),
                dict(dZ=FAKE + 1), dict(ids=FAKE + 4), dict(labels=FAKE + 4), dict(weight=FAKE + 2), dict(loss=FAKE + 1)):
        assert call(**bad) == dp.DP_EINVAL, bad
    for much in (dict(M=2 ** 31), dict(V=2 ** 30), dict(K=1025)):
        assert call(**much) == dp.DP_EUNSUPPORTED, much
    assert call(M=0, Z=None, loss=None, dZ=None, ids=None, logits=None) == dp.DP_OK
    assert dp.dp_distill_loss_workspace_bytes(0, 1, 1, dp.DP_F32) == 0


class Fake:
    """Stands for a GPU tensor of [N][T][W] with given strides; only its description is read."""

    def __init__(self, dtype, shape, stride=None, device=0):
        self.dtype, self.shape, self.device = dtype, tuple(shape), device
        dense = [1]
        for s in reversed(shape[1:]):
            dense.insert(0, dense[0] * s)
        self.strides = tuple(dense if stride is None else stride)
        self.dense = self.strides == tuple(dense)

    def get_device(self):
        return self.device

    def is_contiguous(self):
        return self.dense

    def dim(self):
        return len(self.shape)

    def stride(self, k=None):
        return self.strides if k is None else self.strides[k]

    def numel(self):
        return math.prod(self.shape)

    def element_size(self):
        return self.dtype.itemsize

    def data_ptr(self):
        return FAKE


def test_tensors_are_checked_before_the_call():
    f, b = torch.float32, torch.bfloat16
    rows = lambda x, N=2, T=3, ld=40, width=16, dev=None: dp._rows("f", dev, f, ("X", x, N, T, ld, width))  # noqa: E731
    assert rows(Fake(f, (2, 3, 16), (120, 40, 1))) == (0, [FAKE])
    assert rows(Fake(f, (2, 3, 2, 8), (120, 40, 8, 1)))[0] == 0
    assert rows(Fake(f, (240,))) == (0, [FAKE]) and rows(Fake(f, (216,)))[0] == 0
    assert rows(None) == (None, [None]) and rows(FAKE) == (None, [FAKE])
    for x in (Fake(f, (215,)), Fake(f, (2, 3, 16), (120, 41, 1)), Fake(f, (2, 3, 16), (100, 40, 1)), Fake(f, (2, 3, 15), (120, 40, 1)),
              Fake(f, (2, 2, 16), (120, 40, 1)), Fake(f, (1, 3, 16), (120, 40, 1)), Fake(f, (2, 3, 16), (120, 40, 2)),
              Fake(f, (6, 16), (40, 1)), Fake(f, (2, 3, 16, 1, 4), (120, 40, 2, 1, 1)), Fake(f, (2, 3, 16), (120, 40, 1), device=-1)):
        with pytest.raises(ValueError):
            rows(x)
    with pytest.raises(TypeError):
        rows(Fake(b, (240,)))
    with pytest.raises(ValueError, match="GPU 1"):
        rows(Fake(f, (240,), device=1), dev=0)
    lens = Fake(torch.int32, (2,), device=1)
    a = dp.make_attention(**GOOD, lens=lens)
    assert a.kept[1] is lens and a.dev == 1
    x = [Fake(f, (2, 3, 32)), Fake(f, (2, 4, 16)), Fake(f, (2, 4, 16)), Fake(f, (2, 3, 32))]
    with pytest.raises(ValueError, match="GPU 0"):
        dp.dp_attention_forward(a, *x)
    with pytest.raises(ValueError, match="lse"):
        dp.dp_attention_forward(a, *x, lse=Fake(f, (24,)))
    with pytest.raises(TypeError):
        dp.make_attention(**GOOD, docs=Fake(torch.int64, (8,)))
    with pytest.raises(ValueError):
        dp.make_attention(**GOOD, docs=Fake(torch.int32, (7,)))
    with pytest.raises(ValueError, match="not on a GPU"):
        dp.dp_rotary(torch.zeros(2, 3, 16), dp.DP_F32, 2, 3, 2, 8, 16, FAKE, [4], FAKE, 0, 0, FAKE, 16)
    with pytest.raises(ValueError, match="not on a GPU"):
        dp.dp_distill_loss(torch.zeros(2, 9), dp.DP_F32, 2, 9, FAKE, FAKE, 3, None, 1.0, 1.0, None, FAKE)


def test_the_attention_definition_against_differences():
    """The formula of the gradients that the GPU tests take is the derivative of the forward definition."""
    rng = np.random.default_rng(3)
    N, T, Hq, Hk, D = 1, 6, 4, 2, 5
    x = {"Q": rng.standard_normal((N, T, Hq, D)), "K": rng.standard_normal((N, T, Hk, D)), "V": rng.standard_normal((N, T, Hk, D))}
    dO = rng.standard_normal((N, T, Hq, D))
    mask = ref.Mask(N, T, T, causal=True, prefix=np.array([2]), docs=np.array([[0, 0, 0, 0, 1, 1]]))
    slopes = rng.uniform(0.1, 1, Hq)
    value = lambda y: (ref.attention(y["Q"], y["K"], y["V"], mask, 0.7, 1.5, slopes, torch.float32)[0][0] * dO).sum()  # noqa: E731
    grads, _ = ref.attention_grads(x["Q"], x["K"], x["V"], dO, mask, 0.7, 1.5, slopes, torch.float32)
    for name, g in zip(x, grads):
        for at in np.ndindex(g.shape):
            y = {k: v.copy() for k, v in x.items()}
            y[name][at] += 1e-5
            up = value(y)
            y[name][at] -= 2e-5
            assert abs((up - value(y)) / 2e-5 - g[at]) < 1e-8 * (1 + abs(g[at]))


def test_the_distillation_definition_against_autograd():
    rng = np.random.default_rng(4)
    M, V, K = 5, 30, 4
    Z, ids, t = rng.standard_normal((M, V)), rng.integers(-1, V, (M, K)), rng.standard_normal((M, K))
    labels, w = rng.integers(-1, V, M), rng.uniform(0.5, 2, M)
    ids[1] = -1
    loss, dZ, _, _ = ref.distill(Z, ids, t, labels, 0.3, 1.7, w, torch.float32)
    z = torch.from_numpy(Z).requires_grad_(True)
    total = 0
    for m in range(M):
        used = ids[m] >= 0
        if used.any():
            P = torch.log_softmax(torch.from_numpy(t[m][used]) / 1.7, 0)
            q = torch.log_softmax(z[m] / 1.7, 0)[torch.from_numpy(ids[m][used])]
            total = total + w[m] * 0.3 * 1.7 ** 2 * (P.exp() * (P - q)).sum()
        if labels[m] >= 0:
            total = total - w[m] * 0.7 * torch.log_softmax(z[m], 0)[labels[m]]
    assert abs(float(total.detach()) - loss.sum()) < 1e-12 * (1 + abs(loss.sum()))
    assert np.abs(torch.autograd.grad(total, z)[0].numpy() - dZ).max() < 1e-13
