"""Attention forward and backward on the GPU against the definition in 64 bits: head layouts, masks, lengths, strides."""
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


def say(*a):
    print("[case]", *a, file=sys.stderr, flush=True)


def ws_of(n):
    return torch.full((max(int(n), 16),), 0xA5, dtype=torch.uint8, device=DEV)


class Case:
    """Inputs, the call and the reference.  With gap > 0 the positions of every array are `gap` values apart, and those values
    have to stay as they were."""

    def __init__(self, N, Tq, Tk, Hq, Hk, D, dt="f32", causal=False, last=False, lens=None, prefix=None, docs=None, cap=0.0,
                 slopes=False, gap=0, seed=0, scale=None, size=1.0):
        rng = np.random.default_rng(seed)
        self.sizes, self.dt, self.tt = (N, Tq, Tk, Hq, Hk, D), dt, TT[dt]
        self.cap, self.gap = cap, gap
        self.scale = float(np.float32(D ** -0.5 if scale is None else scale))
        draw = lambda T, H: torch.from_numpy(size * rng.standard_normal((N, T, H, D))).to(self.tt)  # noqa: E731
        self.Q, self.K, self.V, self.dO = draw(Tq, Hq), draw(Tk, Hk), draw(Tk, Hk), draw(Tq, Hq)
        self.slopes = np.float32(2.0 ** -rng.uniform(1, 8, Hq)) if slopes else None
        self.lens, self.prefix, self.docs = [None if x is None else np.asarray(x, dtype=np.int32) for x in (lens, prefix, docs)]
        self.causal, self.last = causal, last
        self.mask = ref.Mask(N, Tq, Tk, causal, last, self.lens, self.prefix, self.docs)

    def put(self, x, fill=None):
        """[N][T][H][D] on the GPU, its positions ld values apart."""
        N, T, H, D = x.shape
        ld = H * D + self.gap
        buf = torch.full((N, T, ld), -7.0, dtype=self.tt, device=DEV)
        view = buf[:, :, :H * D]
        view.copy_(x.reshape(N, T, H * D)) if fill is None else view.fill_(fill)
        return buf, view, ld

    def attention(self, ld):
        N, Tq, Tk, Hq, Hk, D = self.sizes
        g = lambda x: None if x is None else torch.from_numpy(x).to(DEV)  # noqa: E731
        flags = (dp.DP_ATTENTION_CAUSAL if self.causal else 0) | (dp.DP_ATTENTION_LAST if self.last else 0)
        return dp.make_attention(DT[self.dt], *self.sizes, self.scale, flags, self.cap, g(self.slopes), g(self.lens),
                                 g(self.prefix), g(self.docs), *ld)

    def run(self, backward=True):
        N, Tq, Tk, Hq, Hk, D = self.sizes
        bufs = {k: self.put(getattr(self, k)) for k in ("Q", "K", "V", "dO")}
        bufs["O"] = self.put(self.Q, float("nan"))
        for k, like in (("dQ", self.Q), ("dK", self.K), ("dV", self.V)):
            bufs[k] = self.put(like, float("nan"))
        a = self.attention([bufs[k][2] for k in ("Q", "K", "V", "O")])
        v = {k: b[1] for k, b in bufs.items()}
        lse = torch.full((N, Hq, Tq), float("nan"), device=DEV)
        dp.dp_attention_forward(a, v["Q"], v["K"], v["V"], v["O"], lse, ws_of(dp.dp_attention_forward_workspace_bytes(a)))
        names = ["O"]
        if backward:
            dp.dp_attention_backward(a, v["Q"], v["K"], v["V"], v["O"], lse, v["dO"], v["dQ"], v["dK"], v["dV"],
                                     ws_of(dp.dp_attention_backward_workspace_bytes(a)))
            names += ["dQ", "dK", "dV"]
        torch.cuda.synchronize()
        if self.gap:
            for k in names:
                assert bool((bufs[k][0][:, :, -self.gap:] == -7.0).all()), k
        shape = lambda k: {"O": self.Q, "dQ": self.Q, "dK": self.K, "dV": self.V}[k].shape  # noqa: E731
        return {k: v[k].reshape(shape(k)) for k in names}, lse

    def check(self, backward=True):
        out, lse = self.run(backward)
        Q, K, V, dO = [f64(x) for x in (self.Q, self.K, self.V, self.dO)]
        args = (self.mask, self.scale, self.cap, self.slopes, self.tt)
        (O, l), (eO, el) = ref.attention(Q, K, V, *args)
        within(out["O"], O, eO, "O")
        within(lse, l, el, "lse")
        if backward:
            grads, errs = ref.attention_grads(Q, K, V, dO, *args)
            for k, g, e in zip(("dQ", "dK", "dV"), grads, errs):
                within(out[k], g, e, k)
        again, lse2 = self.run(backward)
        bits = lambda x: x.contiguous().view(torch.int16 if x.dtype == torch.bfloat16 else torch.int32)  # noqa: E731
        for k in out:
            assert torch.equal(bits(out[k]), bits(again[k])), k
        assert torch.equal(bits(lse), bits(lse2))
        return out, lse


SIZES = [  # N, Tq, Tk, Hq, Hk, D
    (1, 1, 1, 1, 1, 1), (2, 3, 3, 2, 1, 2), (2, 31, 31, 3, 3, 8), (1, 32, 32, 4, 2, 16), (2, 33, 65, 2, 2, 20), (1, 64, 64, 2, 1, 32),
    (1, 63, 129, 5, 1, 48), (2, 65, 65, 2, 1, 64), (1, 130, 130, 4, 2, 64), (1, 127, 64, 2, 2, 80), (1, 128, 128, 1, 1, 96),
    (1, 200, 257, 3, 1, 100), (2, 129, 129, 2, 1, 128), (1, 257, 257, 4, 1, 128), (1, 40, 70, 2, 1, 130), (1, 33, 40, 2, 1, 256)]


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("sizes", SIZES)
def test_sizes(sizes, causal, dt):
    say("sizes", sizes, causal, dt)
    Case(*sizes, dt=dt, causal=causal, seed=sum(sizes)).check()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("D", [24, 64, 128])
@pytest.mark.parametrize("kind", ["cap", "slopes", "both", "lens", "prefix", "docs", "docs_prefix", "all", "last", "bidir_docs"])
def test_scores_and_masks(kind, D, dt):
    say("masks", kind, D, dt)
    N, T, Hq, Hk = 3, 150, 4, 2
    rng = np.random.default_rng(5)
    docs = np.sort(rng.integers(0, 4, (N, T)), 1)
    docs[1] = rng.integers(0, 3, T)                    # not in runs
    docs[2, -20:] = -1
    kw = {"cap": dict(cap=3.0), "slopes": dict(slopes=True), "both": dict(cap=5.0, slopes=True),
          "lens": dict(lens=[150, 0, 71]), "prefix": dict(prefix=[0, 70, 150]), "docs": dict(docs=docs),
          "docs_prefix": dict(docs=docs, prefix=[60, 10, 500]),
          "all": dict(docs=docs, prefix=[60, -3, 9], lens=[149, 1, 200], cap=4.0, slopes=True),
          "last": dict(lens=[3, 150, 64], last=True, slopes=True),
          "bidir_docs": dict(docs=docs, lens=[100, 150, 140], causal=False, slopes=True)}[kind]
    Case(N, T, T, Hq, Hk, D, dt=dt, **{"causal": True, **kw}, seed=7).check()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("Tq,Tk,Hq,Hk,D", [(1, 1, 4, 1, 64), (1, 700, 8, 2, 128), (1, 2000, 3, 3, 48), (2, 1500, 16, 2, 64),
                                           (5, 300, 2, 1, 128), (1, 4097, 32, 1, 16), (7, 999, 40, 2, 80), (1, 5000, 4, 4, 256)])
def test_few_queries_over_a_cache(Tq, Tk, Hq, Hk, D, dt):
    say("cache", Tq, Tk, Hq, Hk, D, dt)
    N = 3
    kw = dict(causal=True, last=True, seed=11)
    Case(N, Tq, Tk, Hq, Hk, D, dt=dt, **kw).check(backward=False)
    Case(N, Tq, Tk, Hq, Hk, D, dt=dt, lens=[Tk, max(1, Tk // 3), 0], cap=2.0, slopes=True, **kw).check()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("gap,D", [(8, 64), (1, 64), (3, 33), (40, 128), (2, 48)])
def test_positions_apart_and_unaligned(gap, D, dt):
    say("gap", gap, D, dt)
    Case(2, 70, 90, 4, 2, D, dt=dt, gap=gap, seed=3).check()
    Case(2, 1, 333, 4, 2, D, dt=dt, gap=gap, causal=True, last=True, seed=3).check(backward=False)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("D", [40, 64, 128])
def test_values_in_hidden_places_have_no_part(D, dt):
    """NaN and infinities behind a sample's keys, in padding queries, and in other documents."""
    say("hidden", D, dt)
    N, T = 2, 140
    docs = np.repeat(np.array([[0, 1]]), N, 0).repeat(70, 1)
    c = Case(N, T, T, 4, 2, D, dt=dt, causal=True, lens=[140, 120], docs=docs, cap=6.0, seed=9)
    bad = torch.tensor([float("nan"), float("inf"), -float("inf")]).to(c.tt)
    for x in (c.K, c.V, c.Q, c.dO):
        x[1, 120:] = bad[torch.arange(20 * x.shape[2] * D).reshape(20, x.shape[2], D) % 3]       # sample 1: padding
    out, _ = c.check()
    assert all(bool(torch.isfinite(v).all()) for v in out.values())
    c = Case(N, T, T, 4, 2, D, dt=dt, causal=True, docs=docs, seed=9)
    c.K[0, 100], c.V[0, 101, 0, 3], c.Q[1, 75], c.dO[1, 76, 0, 0] = bad[0], bad[1], bad[0], bad[0]  # seen within document 1
    out, _ = c.check()
    for v in out.values():
        assert bool(torch.isfinite(v[:, :70]).all())
    assert bool(torch.isnan(out["O"][0, 100:]).any())
    c = Case(1, 100, 100, 2, 1, D, dt=dt, causal=True, seed=2)                                      # later keys
    c.K[0, 90], c.V[0, 80] = bad[0], bad[1]
    out, _ = c.check()
    assert bool(torch.isfinite(out["O"][:, :80]).all())


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("cap", [1e-5, 0.3, 2e4, 1e9])
def test_caps_of_all_sizes(cap, dt):
    """A cap far below the scores, about them, and so far above that its polynomial's coefficients vanish; hidden pairs in all."""
    say("cap", cap, dt)
    docs = np.repeat(np.array([[0, 1]]), 2, 0).repeat(45, 1)
    Case(2, 90, 90, 2, 1, 64, dt=dt, causal=True, cap=float(np.float32(cap)), lens=[90, 75], docs=docs, seed=13).check()
    Case(1, 1, 500, 4, 2, 64, dt=dt, causal=True, last=True, lens=[333], cap=float(np.float32(cap)), seed=13).check(backward=False)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_rows_that_see_nothing(dt):
    c = Case(2, 50, 50, 2, 1, 64, dt=dt, docs=np.full((2, 50), -1), seed=1)
    out, lse = c.check()
    assert all(bool((v == 0).all()) for v in out.values()) and bool((lse == -float("inf")).all())
    Case(2, 40, 40, 2, 1, 64, dt=dt, lens=[0, 0], seed=1).check()
    c = Case(2, 6, 0, 2, 1, 64, dt=dt, seed=1)
    out, lse = c.run()
    assert bool((out["O"] == 0).all()) and bool((out["dQ"] == 0).all()) and bool((lse == -float("inf")).all())
    c = Case(2, 0, 6, 2, 1, 64, dt=dt, seed=1)
    out, _ = c.run()
    assert bool((out["dK"] == 0).all()) and bool((out["dV"] == 0).all())


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("scale,size", [(1.0, 6.0), (0.001, 1.0), (-0.2, 1.0)])
def test_large_and_small_scores(scale, size, dt):
    """Scores of some hundreds: one key has all the weight."""
    say("scores", scale, size, dt)
    Case(1, 100, 140, 2, 1, 64, dt=dt, scale=scale, size=size, seed=4).check()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("G,causal", [(1, True), (2, False)])
def test_many_blocks_of_documents(G, causal, dt):
    """Blocks enough to be run in the order of their work: documents of different lengths, in runs and mixed, padded samples."""
    say("blocks", G, causal, dt)
    N, T, Hk = 2, 1100, 16
    docs = np.repeat(np.arange(5), [100, 500, 30, 300, 170])[None].repeat(N, 0)
    docs[1] = np.repeat([3, -1, 3, 9, 0], [50, 20, 400, 600, 30])
    Case(N, T, T, Hk * G, Hk, 16, dt=dt, causal=causal, docs=docs, lens=[1100, 1071], prefix=[200, 0] if causal else None, seed=12).check()


def test_gradients_against_differences():
    """The fp32 kernels' gradients against central differences of the forward definition in 64 bits."""
    c = Case(1, 9, 9, 4, 2, 12, causal=True, cap=2.0, slopes=True, docs=np.array([[0] * 4 + [1] * 5]), seed=8)
    out, _ = c.run()
    base = {k: f64(getattr(c, k)) for k in ("Q", "K", "V")}

    def value(k, at, x):
        b = dict(base)
        b[k] = base[k].copy()
        b[k][at] += x
        (O, _), _ = ref.attention(b["Q"], b["K"], b["V"], c.mask, c.scale, c.cap, c.slopes, torch.float32)
        return float((O * f64(c.dO)).sum())

    rng = np.random.default_rng(0)
    for k in base:
        for _ in range(12):
            at = tuple(rng.integers(0, s) for s in base[k].shape)
            want = (value(k, at, 1e-4) - value(k, at, -1e-4)) / 2e-4
            # differences: h^2 / 6 of a third derivative (some tens) and 2^-52 / h; the kernel: some hundred half steps
            assert abs(float(out["d" + k][at]) - want) < 2e-5 * (1 + abs(want)), (k, at)


def test_graph_replays_match_eager():
    for kw in (dict(sizes=(2, 150, 150, 4, 2, 64), causal=True, cap=8.0), dict(sizes=(2, 1, 3000, 8, 2, 128), causal=True, last=True)):
        sizes = kw.pop("sizes")
        for dt in ("bf16", "f32"):
            c = Case(*sizes, dt=dt, lens=[sizes[2], sizes[2] // 2], seed=6, **kw)
            a = c.attention([sizes[3] * sizes[5], sizes[4] * sizes[5], sizes[4] * sizes[5], sizes[3] * sizes[5]])
            x = {k: getattr(c, k).to(DEV) for k in ("Q", "K", "V", "dO")}
            o = {k: torch.zeros_like(x[l]) for k, l in (("O", "Q"), ("dQ", "Q"), ("dK", "K"), ("dV", "V"))}
            lse = torch.zeros((sizes[0], sizes[3], sizes[1]), device=DEV)
            w1, w2 = ws_of(dp.dp_attention_forward_workspace_bytes(a)), ws_of(dp.dp_attention_backward_workspace_bytes(a))

            def go():
                dp.dp_attention_forward(a, x["Q"], x["K"], x["V"], o["O"], lse, w1)
                dp.dp_attention_backward(a, x["Q"], x["K"], x["V"], o["O"], lse, x["dO"], o["dQ"], o["dK"], o["dV"], w2)

            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                go()
            torch.cuda.current_stream().wait_stream(side)
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                go()
            for k in range(3):
                for t in x.values():
                    t.copy_(torch.randn(t.shape, generator=torch.Generator().manual_seed(k)).to(t.dtype))
                go()
                torch.cuda.synchronize()
                want = {n: t.clone() for n, t in o.items()}
                for t in o.values():
                    t.fill_(5.0)
                graph.replay()
                torch.cuda.synchronize()
                for n, t in o.items():
                    assert torch.equal(t, want[n]), (n, k)


@pytest.mark.parametrize("N", [3, 300])
def test_key_gradients_where_dS_cancels(N):
    """Values that differ little: dO.V - dO.O is a small difference, and O is rounded to bf16 before the call."""
    T, D = 8, 32
    say("test_key_gradients_where_dS_cancels", N)
    case = Case(N, T, T, 1, 1, D, "bf16", scale=2.0 ** -5, seed=11)
    common = torch.from_numpy(np.random.default_rng(12).standard_normal((N, 1, 1, D)))
    case.V = (common + case.V.double() / 16).to(torch.bfloat16)
    Q, K, V, dO = (f64(getattr(case, k))[:, :, 0] for k in ("Q", "K", "V", "dO"))
    s = case.scale * (Q @ K.transpose(0, 2, 1))
    p = np.exp(s - s.max(-1, keepdims=True))
    p /= p.sum(-1, keepdims=True)
    dP = dO @ V.transpose(0, 2, 1)
    e = p * (dP - (p * dP).sum(-1, keepdims=True))
    want = case.scale * (e.transpose(0, 2, 1) @ Q)
    # dK is rounded once (2^-8); e goes into its product as two bf16 values (2^-16) and has p's error (2^-18: scores of size 1 at
    # most some units, fp32 sums of 32 products; 2^-14 in all covers both); dO.V and the corrected dO.O are fp32 sums of D and of
    # D + T products in any order, the latter off by what sum p lacks of 1 as well (2^-18 = 64 * 2^-24)
    size = (np.abs(dO) @ np.abs(V).transpose(0, 2, 1)).max(-1, keepdims=True)
    near = p * (2 * (D + T + 8) + 64) * 2.0 ** -24 * size + np.abs(e) * 2.0 ** -14
    bound = 2.0 ** -8 * np.abs(want) + case.scale * (near.transpose(0, 2, 1) @ np.abs(Q)) + 2.0 ** -126
    # (with dO.O from the rounded O alone the bound would not hold)
    rounded = (p @ V).astype(np.float32)
    O = f64(torch.from_numpy(rounded).to(torch.bfloat16))
    off = case.scale * ((p * (dP - (dO * O).sum(-1, keepdims=True))).transpose(0, 2, 1) @ Q)
    assert (np.abs(off - want) > bound).any()
    got = f64(case.run()[0]["dK"]).reshape(N, T, D)
    assert (np.abs(got - want) <= bound).all(), float((np.abs(got - want) / bound).max())
