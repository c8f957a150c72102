"""The language-model operators together, as a DP-SGD step of a small token model uses them: lookup, gated feed-forward,
their backward passes, per-sample norms, clipped sums, average, and the norm of the result; eagerly against per-sample
autograd in 64 bits, as a replayed graph and on a stream of its own against the eager calls."""
import sys

import numpy as np
import pytest
import torch

from compare import assert_g12, assert_rel
from paper_2109_12298_amd import binding as dp

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
ACT = dp.DP_ACT_SILU


def say(*a):
    print("[case]", *a, file=sys.stderr, flush=True)


class Step:
    """Buffers of one step; run() enqueues it on the current stream."""

    def __init__(self, N, T, V, D, F, dt, C=3.0, bound=0.05):
        self.sizes, self.C, self.bound = (N, T, V, D, F), C, bound
        self.tt = torch.bfloat16 if dt == "bf16" else torch.float32
        self.dt = dp.DP_BF16 if dt == "bf16" else dp.DP_F32
        self.scale = D ** 0.5
        e = lambda *s, t=self.tt: torch.zeros(s, dtype=t, device=DEV)  # noqa: E731
        f = torch.float32
        self.ids = torch.zeros((N, T), dtype=torch.int64, device=DEV)
        self.E, self.Wg, self.Wu = e(V, D, t=f), e(F, D), e(F, D)
        self.dH = e(N, T, F)
        self.Y, self.H, self.G, self.U = e(N, T, D), e(N, T, F), e(N, T, F), e(N, T, F)
        self.BG, self.BU, self.dY = e(N, T, F), e(N, T, F), e(N, T, D)
        self.sq, self.norm, self.total = e(3, N, t=f), e(N, t=f), e(1, t=f)
        self.sums = [e(V, D, t=f), e(F, D, t=f), e(F, D, t=f)]
        self.status = torch.zeros(1, dtype=torch.int32, device=DEV)
        self.row_ptr, self.uniq = torch.zeros(N + 1, dtype=torch.int64, device=DEV), e(N * T, t=torch.int64)
        self.rows, self.gs = e(N * T, D, t=f), e(N, F, D, t=f)
        ws = lambda n: torch.empty(max(int(n), 16), dtype=torch.uint8, device=DEV)  # noqa: E731
        M = N * T
        self.ws_f = ws(dp.dp_gated_ffn_forward_workspace_bytes(M, D, F, self.dt))
        self.ws_b = ws(dp.dp_gated_ffn_backward_workspace_bytes(M, D, F, self.dt))
        self.ws_e = ws(dp.dp_grad_sample_embedding_workspace_bytes(N, T))
        self.ws_l = ws(dp.dp_grad_sample_linear_workspace_bytes(N, T, D, F, self.dt))
        self.ws_t = ws(dp.dp_clip_accumulate_tokens_workspace_bytes(N, T, V, D, self.dt))
        self.lin = dp.make_linear_clips([(self.Y, self.BG, T, D, F, 1.0, self.sums[1], None),
                                         (self.Y, self.BU, T, D, F, 1.0, self.sums[2], None)])
        self.ws_c = ws(dp.dp_clip_accumulate_linear_many_workspace_bytes(self.lin, 2, self.dt, N))
        self.items = dp.make_grad_tensors([(s, s, s.numel(), dp.DP_F32) for s in self.sums])
        self.ws_n = ws(dp.dp_clip_global_norm_many_workspace_bytes(self.items, 3))

    def draw(self, seed):
        N, T, V, D, F = self.sizes
        rng = np.random.default_rng(seed)
        put = lambda t, x: t.copy_(torch.from_numpy(np.asarray(x)).to(t.dtype))  # noqa: E731
        put(self.ids, np.minimum((np.exp(rng.random((N, T)) * np.log(V + 1.0)) - 1).astype(np.int64), V - 1))
        put(self.E, rng.standard_normal((V, D)) / np.sqrt(D))
        put(self.Wg, rng.standard_normal((F, D)) / np.sqrt(D))
        put(self.Wu, rng.standard_normal((F, D)) / np.sqrt(D))
        put(self.dH, rng.standard_normal((N, T, F)) * rng.uniform(0.1, 1.0, (N, 1, 1)) / T)

    def run(self):
        N, T, V, D, F = self.sizes
        M, dt = N * T, self.dt
        dp.dp_embedding_lookup(self.ids, self.E, dp.DP_F32, N, T, V, D, self.scale, self.Y, dt, self.status)
        dp.dp_gated_ffn_forward(self.Y, self.Wg, self.Wu, dt, M, D, F, ACT, self.H, self.G, self.U, self.ws_f)
        dp.dp_gated_ffn_backward(self.dH, self.G, self.U, self.Wg, self.Wu, dt, M, D, F, ACT, self.BG, self.BU, self.dY,
                                 self.ws_b)
        dp.dp_grad_sample_embedding(self.ids, self.dY, dt, N, T, V, D, self.scale, self.row_ptr, self.uniq, self.rows, M,
                                    self.sq[0], self.status, self.ws_e)
        for k, B in ((1, self.BG), (2, self.BU)):
            dp.dp_grad_sample_linear(self.Y, B, dt, N, T, D, F, 1.0, self.gs, None, self.sq[k], self.status, self.ws_l)
        dp.dp_per_sample_norms(self.sq, 3, N, self.norm, self.status)
        dp.dp_clip_accumulate_tokens(self.ids, self.dY, dt, N, T, V, D, self.scale, self.norm, self.C, self.sums[0],
                                     self.status, self.ws_t)
        dp.dp_clip_accumulate_linear_many(self.lin, 2, dt, N, self.norm, self.C, self.status, self.ws_c)
        for k, s in enumerate(self.sums):
            dp.dp_add_noise(s, s, s.numel(), 0, 0, k, 0.0, self.C, float(N), self.status)
        dp.dp_clip_global_norm_many(self.items, 3, self.bound, self.total, self.status, self.ws_n)

    def outputs(self):
        return [self.Y, self.H, self.BG, self.BU, self.dY, self.norm, self.total] + self.sums


def reference(s):
    """The same step by autograd of each sample's own loss in 64 bits."""
    N, T, V, D, F = s.sizes
    E, Wg, Wu = [t.detach().cpu().double().requires_grad_(True) for t in (s.E, s.Wg, s.Wu)]
    ids, dH = s.ids.cpu(), s.dH.cpu().double()
    norms, sums = [], [torch.zeros_like(p) for p in (E, Wg, Wu)]
    for n in range(N):
        x = s.scale * E[ids[n]]
        g = x @ Wg.t()
        loss = (g * torch.sigmoid(g) * (x @ Wu.t()) * dH[n]).sum()
        grads = torch.autograd.grad(loss, (E, Wg, Wu))
        norm = torch.sqrt(sum((q * q).sum() for q in grads))
        norms.append(float(norm))
        c = min(1.0, s.C / (float(norm) + 1e-6))
        for a, q in zip(sums, grads):
            a += c * q
    sums = [(a / N).numpy() for a in sums]
    total = np.sqrt(sum((a * a).sum() for a in sums))
    return np.array(norms), total, [a * min(1.0, s.bound / (total + 1e-6)) for a in sums]


@pytest.mark.parametrize("N,T,V,D,F", [(5, 9, 40, 24, 36), (6, 32, 200, 64, 96), (3, 1, 7, 8, 8)])
def test_step_matches_per_sample_autograd(N, T, V, D, F):
    """fp32 throughout: every stage is off by its sums' roundings, under 1e-5 of the result's size at these lengths, and the
    five stages in a row by less than the 1e-4 that the library's fp32 results are held to."""
    say("lm step", N, T, V, D, F)
    s = Step(N, T, V, D, F, "f32")
    s.draw(N)
    s.C = float(np.median(reference(s)[0]))          # some samples are clipped, some are not
    norms, total, sums = reference(s)
    s.run()
    assert s.status.item() == 0
    assert_rel(s.norm.cpu().numpy(), norms, 1e-4, "norms")
    assert_rel(s.total.cpu().numpy(), [total], 1e-4, "total")
    for got, want in zip(s.sums, sums):
        assert_g12(got.cpu().numpy(), want, 1e-4)


@pytest.mark.parametrize("sizes", [(4, 16, 300, 64, 128), (20, 150, 5000, 136, 200), (1, 1, 50, 64, 64)])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_replayed_graph_and_other_stream_equal_eager_calls(sizes, dt):
    """Three replays on new inputs, with eager work between them, bit for bit; then the same calls on a stream of their own."""
    say("lm step graph", sizes, dt)
    s, e = Step(*sizes, dt), Step(*sizes, dt)
    s.draw(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s.run()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.run()
    for seed in (1, 2, 3):
        s.draw(seed)
        graph.replay()
        e.draw(seed)
        e.run()
        torch.cuda.synchronize()
        for a, b in zip(s.outputs(), e.outputs()):
            assert torch.equal(a, b) and a.isfinite().all()
    s.draw(4)
    e.draw(4)
    e.run()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        s.run()
    side.synchronize()
    for a, b in zip(s.outputs(), e.outputs()):
        assert torch.equal(a, b)
    assert s.status.item() == 0


def test_two_steps_at_once_on_two_streams():
    """Disjoint outputs and workspaces: calls on two streams may overlap."""
    say("lm step two streams")
    sizes = (8, 300, 3000, 128, 192)
    a, b, ra, rb = [Step(*sizes, "bf16") for _ in range(4)]
    for s, seed in ((a, 1), (ra, 1), (b, 2), (rb, 2)):
        s.draw(seed)
    ra.run()
    rb.run()
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        with torch.cuda.stream(s1):
            a.run()
        with torch.cuda.stream(s2):
            b.run()
    torch.cuda.synchronize()
    for x, r in ((a, ra), (b, rb)):
        for p, q in zip(x.outputs(), r.outputs()):
            assert torch.equal(p, q)
