"""A transformer layer and a loss from the library's calls, as a DP-SGD step of a token model uses them: positions, attention,
the loss with its gradient, their backward passes and the projections' per-sample gradients, against per-sample autograd in 64
bits; as a replayed graph beside an eager run, and two steps on streams of their own."""
import sys

import numpy as np
import pytest
import torch

from compare import assert_g12, assert_rel
from paper_2109_12298_amd import binding as dp

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def say(*a):
    print("[case]", *a, file=sys.stderr, flush=True)


class Step:
    """x -> fused projection qkv -> rotary (q, k) -> attention -> output layer -> distillation; run() enqueues it and the way
    back on the current stream.  Matrix products of the layers are torch's: the library's part is what lies between."""

    def __init__(self, N, T, E, Hq, Hk, D, V, K, dt, cap=0.0, docs=False):
        self.sizes, self.cap = (N, T, E, Hq, Hk, D, V, K), cap
        self.tt = torch.bfloat16 if dt == "bf16" else torch.float32
        self.dt = dp.DP_BF16 if dt == "bf16" else dp.DP_F32
        z = lambda *s, t=self.tt: torch.zeros(s, dtype=t, device=DEV)  # noqa: E731
        f, W = torch.float32, (Hq + 2 * Hk) * D
        self.x, self.Wqkv, self.Wo = z(N, T, E), z(W, E), z(V, Hq * D)
        self.qkv, self.rot, self.dqkv, self.drot = z(N, T, W), z(N, T, W), z(N, T, W), z(N, T, W)
        self.O, self.dO, self.lse = z(N, T, Hq * D), z(N, T, Hq * D), z(N, Hq, T, t=f)
        self.Z, self.dZ, self.loss, self.weight = z(N, T, V), z(N, T, V), z(N * T, t=f), z(N * T, t=f)
        self.ids, self.top, self.labels = z(N * T, K, t=torch.int64), z(N * T, K, t=f), z(N * T, t=torch.int64)
        self.pos = z(1, N, T, t=torch.int64)
        self.freq = torch.tensor(10000.0 ** (-np.arange(D // 2) / (D // 2)), device=DEV)
        self.lens = z(N, t=torch.int32)
        self.docs = z(N, T, t=torch.int32) if docs else None
        self.status = z(1, t=torch.int32)
        self.a = dp.make_attention(self.dt, N, T, T, Hq, Hk, D, D ** -0.5, dp.DP_ATTENTION_CAUSAL, cap, None, self.lens, None,
                                   self.docs, W, W, W, Hq * D)
        ws = lambda n: torch.empty(max(int(n), 16), dtype=torch.uint8, device=DEV)  # noqa: E731
        self.ws_f = ws(dp.dp_attention_forward_workspace_bytes(self.a))
        self.ws_b = ws(dp.dp_attention_backward_workspace_bytes(self.a))
        self.sq, self.norm = z(2, N, t=f), z(N, t=f)
        self.g_qkv, self.g_o = z(N, W, E, t=f), z(N, V, Hq * D, t=f)
        self.ws_l = ws(max(dp.dp_grad_sample_linear_workspace_bytes(N, T, E, W, self.dt),
                           dp.dp_grad_sample_linear_workspace_bytes(N, T, Hq * D, V, self.dt)))

    def draw(self, seed):
        N, T, E, Hq, Hk, D, V, K = self.sizes
        rng = np.random.default_rng(seed)
        put = lambda t, v: t.copy_(torch.from_numpy(np.asarray(v)).to(t.dtype))  # noqa: E731
        put(self.x, rng.standard_normal((N, T, E)))
        put(self.Wqkv, rng.standard_normal(self.Wqkv.shape) / np.sqrt(E))
        put(self.Wo, 3 * rng.standard_normal(self.Wo.shape) / np.sqrt(Hq * D))
        put(self.ids, rng.integers(0, V, (N * T, K)))
        put(self.top, rng.standard_normal((N * T, K)))
        put(self.labels, rng.integers(-1, V, N * T))
        lens = rng.integers(1, T + 1, N)
        lens[0] = T
        put(self.lens, lens)
        put(self.weight, (np.arange(T)[None] < lens[:, None]).reshape(-1) / T)          # padding has no part in the loss
        put(self.pos, rng.integers(0, 100000, (1, N, 1)) + np.arange(T))
        if self.docs is not None:
            put(self.docs, np.sort(rng.integers(0, 3, (N, T)), 1))

    def run(self):
        N, T, E, Hq, Hk, D, V, K = self.sizes
        W, H = (Hq + 2 * Hk) * D, Hq + Hk
        q, k, v = self.rot.split([Hq * D, Hk * D, Hk * D], 2)
        dq, dk, dv = self.drot.split([Hq * D, Hk * D, Hk * D], 2)
        torch.matmul(self.x, self.Wqkv.t(), out=self.qkv)
        self.rot.copy_(self.qkv)                                       # values keep their places
        dp.dp_rotary(self.qkv, self.dt, N, T, H, D, W, self.pos, [D // 2], self.freq, dp.DP_ROTARY_HALVES, False, self.rot, W)
        dp.dp_attention_forward(self.a, q, k, v, self.O, self.lse, self.ws_f)
        torch.matmul(self.O, self.Wo.t(), out=self.Z)
        dp.dp_distill_loss(self.Z, self.dt, N * T, V, self.ids, self.top, K, self.labels, 0.6, 2.0, self.weight, self.loss,
                           self.dZ, self.status)
        torch.matmul(self.dZ, self.Wo, out=self.dO)
        dp.dp_attention_backward(self.a, q, k, v, self.O, self.lse, self.dO, dq, dk, dv, self.ws_b)
        self.dqkv.copy_(self.drot)
        dp.dp_rotary(self.drot, self.dt, N, T, H, D, W, self.pos, [D // 2], self.freq, dp.DP_ROTARY_HALVES, True, self.dqkv, W)
        dp.dp_grad_sample_linear(self.x, self.dqkv, self.dt, N, T, E, W, 1.0, self.g_qkv, None, self.sq[0], self.status, self.ws_l)
        dp.dp_grad_sample_linear(self.O, self.dZ, self.dt, N, T, Hq * D, V, 1.0, self.g_o, None, self.sq[1], self.status, self.ws_l)
        dp.dp_per_sample_norms(self.sq, 2, N, self.norm, self.status)

    def outputs(self):
        return [self.O, self.lse, self.loss, self.dZ, self.dqkv, self.g_qkv, self.g_o, self.norm]


def reference(s):
    """Every sample's loss and gradients by autograd in 64 bits."""
    N, T, E, Hq, Hk, D, V, K = s.sizes
    c = lambda t: t.detach().cpu().double()  # noqa: E731
    Wqkv, Wo = c(s.Wqkv).requires_grad_(True), c(s.Wo).requires_grad_(True)
    losses, grads = [], []
    for n in range(N):
        L = int(s.lens[n])
        qkv = (c(s.x)[n, :L] @ Wqkv.t()).reshape(L, Hq + 2 * Hk, D)
        ang = c(s.pos)[0, n, :L, None] * c(s.freq)
        co, si = torch.cos(ang)[:, None], torch.sin(ang)[:, None]
        a, b = qkv[:, :Hq + Hk, :D // 2], qkv[:, :Hq + Hk, D // 2:]
        turned = torch.cat([a * co - b * si, b * co + a * si], 2)
        see = torch.ones(L, L).tril().bool()
        if s.docs is not None:
            d = s.docs[n, :L].cpu()
            see &= d[:, None] == d[None]
        heads = []
        for h in range(Hq):
            x = (turned[:, h] @ turned[:, Hq + h * Hk // Hq].t()) * D ** -0.5
            if s.cap > 0:
                x = s.cap * torch.tanh(x / s.cap)
            heads.append(torch.softmax(x.masked_fill(~see, -np.inf), 1) @ qkv[:, Hq + Hk + h * Hk // Hq])
        z = torch.cat(heads, 1) @ Wo.t()
        at = slice(n * T, n * T + L)
        P, logq = torch.log_softmax(c(s.top)[at] / 2.0, 1), torch.log_softmax(z / 2.0, 1)
        loss = 0.6 * 4.0 * (P.exp() * (P - logq.gather(1, s.ids[at].cpu()))).sum(1)
        lab = s.labels[at].cpu()
        hard = -torch.log_softmax(z, 1).gather(1, lab.clamp(min=0)[:, None])[:, 0]
        loss = (loss + torch.where(lab >= 0, 0.4 * hard, 0.0)) * c(s.weight)[at]
        grads.append([g.numpy() for g in torch.autograd.grad(loss.sum(), (Wqkv, Wo))])
        losses.append(torch.cat([loss.detach(), torch.zeros(T - L, dtype=torch.float64)]).numpy())
    return np.concatenate(losses), grads


@pytest.mark.parametrize("sizes", [(4, 40, 24, 4, 2, 16, 50, 5), (3, 70, 64, 2, 1, 64, 333, 8), (2, 1, 8, 1, 1, 8, 9, 1)])
@pytest.mark.parametrize("cap,docs", [(0.0, False), (4.0, True)])
def test_step_matches_per_sample_autograd(sizes, cap, docs):
    say(sizes, cap, docs)
    s = Step(*sizes, "f32", cap, docs)
    s.draw(1)
    s.run()
    torch.cuda.synchronize()
    loss, grads = reference(s)
    assert int(s.status[0]) == 0
    # chains of some ten fp32 calls, each within a few hundred half steps of its sums: 1e-4, as the library's other chains
    assert_g12(s.loss.cpu(), loss, 1e-4, "loss")
    for n in range(sizes[0]):
        assert_g12(s.g_qkv[n].cpu(), grads[n][0], 1e-4, "qkv %d" % n)
        assert_g12(s.g_o[n].cpu(), grads[n][1], 1e-4, "out %d" % n)
    assert_rel(s.norm.cpu(), [np.sqrt(sum((g * g).sum() for g in gs)) for gs in grads], 1e-4, "norms")


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_replayed_graphs_beside_eager_runs(dt):
    """Two steps captured into graphs of their own, replayed in turn with eager runs of the same buffers between."""
    steps = [Step(3, 90, 64, 4, 2, 32, 200, 6, dt, 5.0, True), Step(2, 200, 32, 2, 2, 64, 77, 3, dt)]
    graphs = []
    side = torch.cuda.Stream()
    for k, s in enumerate(steps):
        s.draw(k)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            s.run()
        torch.cuda.current_stream().wait_stream(side)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            s.run()
        graphs.append(g)
    for turn in range(3):
        for k, (s, g) in enumerate(zip(steps, graphs)):
            s.draw(10 * turn + k)
            s.run()
            torch.cuda.synchronize()
            want = [t.clone() for t in s.outputs()]
            for t in s.outputs():
                t.fill_(3.0)
            g.replay()
            torch.cuda.synchronize()
            for i, (a, b) in enumerate(zip(s.outputs(), want)):
                assert torch.equal(a, b), (turn, k, i)


def test_two_steps_on_streams_of_their_own():
    """Calls that overlap on one GPU: each with its own workspace, outputs as one after another."""
    steps = [Step(3, 130, 64, 4, 2, 64, 500, 6, "bf16", 5.0, True), Step(2, 300, 32, 8, 2, 32, 4000, 3, "bf16")]
    for k, s in enumerate(steps):
        s.draw(k)
        s.run()
    torch.cuda.synchronize()
    want = [[t.clone() for t in s.outputs()] for s in steps]
    for turn in range(3):
        streams = [torch.cuda.Stream() for _ in steps]
        for s in steps:
            for t in s.outputs():
                t.fill_(3.0)
        torch.cuda.synchronize()
        for s, st in zip(steps, streams):
            with torch.cuda.stream(st):
                s.run()
        torch.cuda.synchronize()
        for s, w in zip(steps, want):
            assert all(torch.equal(a, b) for a, b in zip(s.outputs(), w)), turn
