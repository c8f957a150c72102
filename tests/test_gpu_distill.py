"""The distillation loss and its gradient on the GPU against the definition in 64 bits."""
import sys

import numpy as np
import pytest
import torch

import token_model_ref as ref
from lm_ref import f64, within
from paper_2109_12298_amd import binding as dp

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TT = {"f32": torch.float32, "bf16": torch.bfloat16}
DT = {"f32": dp.DP_F32, "bf16": dp.DP_BF16}


def draw(M, V, K, dt, seed=0, spread=2.0, ragged=True):
    rng = np.random.default_rng(seed)
    Z = torch.from_numpy(spread * rng.standard_normal((M, V))).to(TT[dt])
    ids = rng.integers(0, V, (M, K))
    if ragged and K > 1:
        ids[np.arange(K)[None] >= rng.integers(0, K + 1, M)[:, None]] = -1
    logits = np.float32(3 * rng.standard_normal((M, K)))
    labels = rng.integers(-1, V, M)
    weight = np.float32(rng.uniform(0.2, 2.0, M))
    return Z, ids, logits, labels, weight


def run(Z, ids, logits, labels, alpha, tau, weight, dt, grad=True, offset=0, out_offset=0, inplace=False):
    M, V = Z.shape
    g = lambda x: None if x is None else torch.from_numpy(np.ascontiguousarray(x)).to(DEV)  # noqa: E731
    # behind and before the rows lie values that have to stay
    store = torch.full((M * V + offset + 9,), 3.0, dtype=TT[dt], device=DEV)
    z = store[offset:offset + M * V].view(M, V)
    z.copy_(Z)
    out = torch.full((M * V + out_offset + 9,), 3.0, dtype=TT[dt], device=DEV)
    dz = z if inplace else out[out_offset:out_offset + M * V].view(M, V)
    loss = torch.full((M,), float("nan"), device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    K = 0 if ids is None else ids.shape[1]
    dp.dp_distill_loss(z, DT[dt], M, V, g(ids), g(logits), K, g(labels), alpha, tau, g(weight), loss, dz if grad else None, status,
                       None)
    torch.cuda.synchronize()
    for buf, o in ((store, offset), (out, out_offset)):
        assert bool((buf[:o] == 3.0).all()) and bool((buf[o + M * V:] == 3.0).all())
    return loss, dz, int(status[0])


def check(M, V, K, dt, alpha=0.6, tau=1.5, seed=0, use=("soft", "labels", "weight"), **kw):
    Z, ids, logits, labels, weight = draw(M, V, K, dt, seed)
    ids, logits = (ids, logits) if "soft" in use else (None, None)
    labels, weight = labels if "labels" in use else None, weight if "weight" in use else None
    loss, dz, status = run(Z, ids, logits, labels, alpha, tau, weight, dt, **kw)
    l, d, el, ed = ref.distill(f64(Z), ids, logits, labels, alpha, tau, weight, TT[dt])
    within(loss, l, el, "loss")
    if kw.get("grad", True):
        within(dz, d, ed, "dZ")
    assert status == 0


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("M,V,K", [(1, 1, 1), (3, 2, 2), (5, 7, 3), (9, 100, 16), (4, 511, 7), (3, 2049, 64), (2, 8191, 20), (2, 10000, 16),
                                   (2, 33001, 64), (2, 70003, 5), (1, 110001, 3), (1, 150001, 8), (1, 240000, 8), (2, 300, 1024)])
def test_sizes(M, V, K, dt):
    print("[case]", M, V, K, dt, file=sys.stderr, flush=True)
    check(M, V, K, dt, seed=V)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("alpha,tau,use", [(1.0, 1.0, ("soft",)), (0.0, 2.0, ("labels",)), (0.0, 1.0, ("soft", "labels")), (1.0, 4.0, ("soft", "labels")),
                                           (0.3, 0.5, ("soft", "labels")), (0.5, 2.0, ("soft", "weight")), (0.5, 1.0, ())])
def test_parts_of_the_loss(alpha, tau, use, dt):
    print("[case]", alpha, tau, use, dt, file=sys.stderr, flush=True)
    check(12, 333, 9, dt, alpha, tau, use=use)
    check(3, 9000, 9, dt, alpha, tau, use=use, grad=False)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("V", [37, 4099, 120001, 200003])
def test_alignment_and_in_place(V, dt):
    print("[case]", V, dt, file=sys.stderr, flush=True)
    for kw in (dict(offset=1, out_offset=1), dict(offset=3, out_offset=2), dict(inplace=True), dict(inplace=True, offset=5)):
        check(2, V, 12, dt, seed=V, **kw)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_odd_values(dt):
    Z, ids, logits, labels, weight = draw(8, 500, 6, dt, ragged=False)
    ids[0] = 17                                        # one class six times
    ids[1, 3] = labels[1] = 40                         # the label among them
    Z[2, 100:] = -float("inf")                         # classes that cannot be
    ids[2], labels[2] = np.arange(6) * 10, 50
    logits[3, :] = -np.inf                             # a teacher without any
    labels[3] = -5
    weight[4] = 0.0
    Z[4, 3], logits[4, 2] = float("nan"), np.nan
    logits[5, 1] = -np.inf
    ids[6], labels[6] = -1, 7
    loss, dz, status = run(Z, ids, logits, labels, 0.5, 2.0, weight, dt)
    lg = logits.copy()
    ids3 = ids.copy()
    ids3[3] = -1                                       # as if its ids were unused
    with np.errstate(invalid="ignore"):
        l, d, el, ed = ref.distill(f64(Z), ids3, lg, labels, 0.5, 2.0, weight, TT[dt])
    within(loss, l, el, "loss")
    within(dz, d, ed, "dZ")
    assert status == 0 and float(loss[3]) == 0.0 and bool((dz[3] == 0).all()) and bool((dz[4] == 0).all())
    Z[7, 9] = float("nan")
    loss, dz, _ = run(Z, ids, logits, labels, 0.5, 2.0, weight, dt)
    assert bool(torch.isnan(loss[7])) and bool(torch.isnan(dz[7]).all()) and bool(torch.isfinite(dz[:7]).all())


def test_bad_ids_are_flagged_and_left_out():
    Z, ids, logits, labels, weight = draw(4, 50, 5, "f32", ragged=False)
    ids[1, 2], labels[2] = 50, 1 << 40
    loss, dz, status = run(Z, ids, logits, labels, 0.5, 1.0, weight, "f32")
    assert status == dp.DP_FLAG_BAD_INDEX
    l, d, el, ed = ref.distill(f64(Z), ids, logits, labels, 0.5, 1.0, weight, torch.float32)
    within(loss, l, el)
    within(dz, d, ed)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_large_logits(dt):
    """Logits of some hundreds, spread over the exponent's range."""
    Z, ids, logits, labels, weight = draw(4, 3000, 9, dt, spread=200.0)
    loss, dz, _ = run(Z, ids, logits, labels, 0.4, 0.7, weight, dt)
    l, d, el, ed = ref.distill(f64(Z), ids, logits, labels, 0.4, 0.7, weight, TT[dt])
    within(loss, l, el)
    within(dz, d, ed)


def test_gradient_against_differences():
    Z, ids, logits, labels, weight = draw(3, 21, 4, "f32", seed=5)
    _, dz, _ = run(Z, ids, logits, labels, 0.4, 1.7, weight, "f32")
    z = f64(Z)
    for m in range(3):
        for v in range(0, 21, 4):
            at = []
            for h in (1e-4, -1e-4):
                y = z.copy()
                y[m, v] += h
                at.append(ref.distill(y, ids, logits, labels, 0.4, 1.7, weight, torch.float32)[0].sum())
            # h^2 / 6 of a third derivative below 4, 2^-52 / h, and some tens of half steps
            assert abs(float(dz[m, v]) - (at[0] - at[1]) / 2e-4) < 1e-5


def test_replayed_graph_and_streams():
    M, V, K = 20, 5001, 8
    Z, ids, logits, labels, weight = draw(M, V, K, "bf16")
    g = lambda x: torch.from_numpy(np.ascontiguousarray(x)).to(DEV)  # noqa: E731
    z, i, t, lab, w = Z.to(DEV), g(ids), g(logits), g(labels), g(weight)
    outs = [(torch.empty(M, device=DEV), torch.empty_like(z)) for _ in range(2)]
    call = lambda o, **k: dp.dp_distill_loss(z, dp.DP_BF16, M, V, i, t, K, lab, 0.5, 2.0, w, o[0], o[1], **k)  # noqa: E731
    call(outs[0])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    call(outs[1], stream=s)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(*outs))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(outs[1])
    for k in range(3):
        z.copy_(torch.randn(z.shape, device=DEV))
        call(outs[0])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(*outs))
