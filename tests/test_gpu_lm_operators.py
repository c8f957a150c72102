"""Embedding lookup, its clipped gradient by sorted tokens, and the global gradient norm on the GPU, against the
64-bit definitions of lm_ref."""
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


def unaligned(x, by=1):
    """x's values on the GPU, `by` elements behind a 16-byte boundary."""
    buf = torch.empty(x.numel() + 16, dtype=x.dtype, device=DEV)
    v = buf[by:by + x.numel()].view(x.shape)
    v.copy_(x)
    return v


def status():
    return torch.zeros(1, dtype=torch.int32, device=DEV)


def ws(n):
    return torch.full((max(n, 1),), 0xA5, dtype=torch.uint8, device=DEV)


# ------------------------------------------------------------------ lookup

@pytest.mark.parametrize("N,T,V,D", [(1, 1, 1, 1), (1, 1, 100, 2048), (3, 7, 50, 100), (2, 33, 10, 533), (5, 64, 300, 64),
                                     (1, 4, 9, 4104), (2, 1000, 77, 8), (1, 3, 5, 257)])
@pytest.mark.parametrize("te,ty", [("f32", "f32"), ("f32", "bf16"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("shift", [0, 1])
def test_lookup(N, T, V, D, te, ty, shift):
    say("lookup", N, T, V, D, te, ty, shift)
    rng = np.random.default_rng(N * 1000 + T + D)
    (tt, ct), (yt, cy) = DT[te], DT[ty]
    E = torch.from_numpy(rng.standard_normal((V, D))).to(tt)
    ids = rng.integers(0, V, (N, T))
    scale = math.sqrt(D) / 3
    Eg = unaligned(E, shift)
    buf = torch.full((N * T * D + 64,), 7.0, dtype=yt, device=DEV)
    Y = buf[shift:shift + N * T * D].view(N, T, D)
    st = status()
    dp.dp_embedding_lookup(torch.from_numpy(ids).to(DEV), Eg, ct, N, T, V, D, scale, Y, cy, st)
    want = R.lookup(ids, R.f64(E), float(np.float32(scale)))
    # one product in fp32, one rounding to the output's type (none more for fp32)
    h = R.half_step(yt) + (R.U32 if ty == "bf16" else 0.0)
    R.within(Y, want, h * (1 + R.U32) * np.abs(want))
    assert st.item() == 0
    assert (buf[:shift] == 7).all() and (buf[shift + N * T * D:] == 7).all()       # nothing beside the output


@pytest.mark.parametrize("te,ty", [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16")])
def test_lookup_large_output(te, ty):
    """Outputs stored past the caches."""
    say("lookup large", te, ty)
    (tt, ct), (yt, cy) = DT[te], DT[ty]
    N, T, V, D = 7, 3700, 900, 2056
    g = torch.Generator(device=DEV).manual_seed(3)
    E = torch.randn((V, D), generator=g, device=DEV).to(tt)
    ids = torch.randint(0, V, (N, T), generator=g, device=DEV)
    Y = torch.full((N, T, D), 7.0, dtype=yt, device=DEV)
    assert Y.numel() * Y.element_size() > 96 << 20
    dp.dp_embedding_lookup(ids, E, ct, N, T, V, D, 1.5, Y, cy)
    assert torch.equal(Y, (E.float() * 1.5).to(yt)[ids])               # one product, one rounding: the same bits


@pytest.mark.parametrize("te,ty", [("f32", "f32"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("D", [2056, 2060])
def test_lookup_large_output_between_boundaries(te, ty, D):
    """Outputs stored past the caches, from 16 bytes behind a 32-byte boundary."""
    say("lookup large between boundaries", te, ty, D)
    (tt, ct), (yt, cy) = DT[te], DT[ty]
    N, T, V = 7, 3700, 900
    g = torch.Generator(device=DEV).manual_seed(3)
    E = torch.randn((V, D), generator=g, device=DEV).to(tt)
    ids = torch.randint(0, V, (N, T), generator=g, device=DEV)
    by = 16 // torch.empty((), dtype=yt).element_size()
    buf = torch.full((N * T * D + 64,), 7.0, dtype=yt, device=DEV)
    Y = buf[by:by + N * T * D].view(N, T, D)
    assert Y.data_ptr() % 32 == 16 and Y.numel() * Y.element_size() > 96 << 20
    dp.dp_embedding_lookup(ids, E, ct, N, T, V, D, 1.5, Y, cy)
    assert torch.equal(Y, (E.float() * 1.5).to(yt)[ids])
    assert (buf[:by] == 7).all() and (buf[by + N * T * D:] == 7).all()


def test_lookup_bad_ids_and_empty():
    say("lookup bad ids")
    V, D = 6, 40
    E = torch.full((V, D), float("inf"), device=DEV)
    E[1:5] = torch.arange(4.0, device=DEV)[:, None] + 1
    ids = torch.tensor([[1, -1, 4], [6, 2 ** 40, 3]], device=DEV)
    Y, st = torch.full((2, 3, D), 7.0, device=DEV), status()
    dp.dp_embedding_lookup(ids, E, dp.DP_F32, 2, 3, V, D, 2.0, Y, dp.DP_F32, st)
    assert st.item() == dp.DP_FLAG_BAD_INDEX
    assert Y[..., 0].tolist() == [[2.0, 0.0, 8.0], [0.0, 0.0, 6.0]] and (Y == Y[..., :1]).all()
    Y.fill_(7.0)
    for N, T in ((0, 3), (2, 0)):
        dp.dp_embedding_lookup(ids, E, dp.DP_F32, N, T, V, D, 2.0, Y, dp.DP_F32)
    assert (Y == 7).all()


# ------------------------------------------------------------------ gradient by sorted tokens

def run_tokens(ids, B, dt, V, scale, norm, C, out=None, st=None, space=None):
    N, T, D = B.shape
    out = torch.full((V, D), 7.0, device=DEV) if out is None else out
    if space is None:
        space = ws(dp.dp_clip_accumulate_tokens_workspace_bytes(N, T, V, D, dt))
    dp.dp_clip_accumulate_tokens(ids, B, dt, N, T, V, D, scale, norm, C, out, st, space)
    return out


def token_ids(rng, kind, N, T, V):
    if kind == "skewed":
        return np.minimum((np.exp(rng.random((N, T)) * math.log(V + 1.0)) - 1).astype(np.int64), V - 1)
    if kind == "same":
        return np.full((N, T), V // 2)
    if kind == "distinct":
        return rng.permutation(max(V, N * T))[:N * T].reshape(N, T) % V
    return rng.integers(0, V, (N, T))


# one launch up to 2048 positions, sorted in one up to 16384 where the ids have 10 bits, 64 tiles of 8192 at 524288
SIZES = [(1, 1, 1, 1), (1, 2, 3, 5), (2, 8, 512, 64), (1, 17, 511, 257), (3, 100, 9000, 200), (16, 128, 300, 100),
         (3, 683, 513, 12), (1, 2049, 40, 100), (2, 4096, 100, 8), (8193, 1, 1000, 6), (33, 300, 70000, 16),
         (5, 2011, 600, 533), (64, 256, 1000, 100), (1, 16385, 500, 40), (4, 5000, 90000, 20), (4, 4096, 512, 8), (16384, 1, 513, 4), (37, 63, 700, 130), (41, 65, 511, 24),
         (150, 100, 130000, 40)]


@pytest.mark.parametrize("N,T,V,D", SIZES)
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["skewed", "same", "distinct"])
def test_tokens(N, T, V, D, dt, kind):
    say("tokens", N, T, V, D, dt, kind)
    rng = np.random.default_rng(N + 10 * T + V)
    tt, ct = DT[dt]
    ids = token_ids(rng, kind, N, T, V)
    B = torch.from_numpy(rng.standard_normal((N, T, D))).to(tt)
    norm = np.exp(rng.standard_normal(N)).astype(np.float32)
    st = status()
    idg, Bg, ng = torch.from_numpy(ids).to(DEV), B.to(DEV), torch.from_numpy(norm).to(DEV)
    got = run_tokens(idg, Bg, ct, V, 1.5, ng, 0.75, st=st)
    want, bound = R.tokens(ids, R.f64(B), V, 1.5, norm, 0.75)
    R.within(got, want, bound)
    assert st.item() == 0
    again = run_tokens(idg, Bg, ct, V, 1.5, ng, 0.75)
    assert torch.equal(got.view(torch.int32), again.view(torch.int32))             # the same bits
    plain = run_tokens(idg, Bg, ct, V, 1.5, None, 0.0)                             # no norms: no clipping, C unused
    want, bound = R.tokens(ids, R.f64(B), V, 1.5, None, 0.0)
    R.within(plain, want, bound)


@pytest.mark.parametrize("M,D", [(140000, 3), (530000, 2)])
def test_tokens_many_positions(M, D):
    """Eight positions per thread, and counts scanned by a launch of their own."""
    say("tokens many", M, D)
    rng = np.random.default_rng(M)
    V = 300000
    ids = token_ids(rng, "skewed", 1, M, V)
    ids[0, ::3] = rng.integers(0, V, ids[0, ::3].shape)
    B = torch.from_numpy(rng.standard_normal((1, M, D))).float()
    got = run_tokens(torch.from_numpy(ids).to(DEV), B.to(DEV), dp.DP_F32, V, 1.0, None, 1.0)
    want, bound = R.tokens(ids, R.f64(B), V, 1.0, None, 1.0)
    R.within(got, want, bound)


@pytest.mark.parametrize("M", [1, 300, 3000, 20000])
def test_tokens_large_vocabulary(M):
    """Ids of 27 bits: three digits."""
    say("tokens vocabulary", M)
    rng = np.random.default_rng(M)
    V, D = 70_000_000, 1
    ids = rng.integers(0, V, (1, M))
    ids[0, M // 2:] = ids[0, :M - M // 2]
    ids[0, 0] = V - 1
    B = torch.from_numpy(rng.standard_normal((1, M, D))).float()
    got = run_tokens(torch.from_numpy(ids).to(DEV), B.to(DEV), dp.DP_F32, V, 1.0, None, 1.0)
    uniq, at = np.unique(ids[0], return_inverse=True)
    want, bound = R.tokens(at.reshape(1, M), R.f64(B), len(uniq), 1.0, None, 1.0)
    R.within(got[torch.from_numpy(uniq).to(DEV)], want, bound)
    got[torch.from_numpy(uniq).to(DEV)] = 0.0
    assert (got == 0).all()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 520])
def test_tokens_large_table(dt, D):
    """A table over 128 MB: only rows without a token are zeroed, by their flags."""
    say("tokens large table", dt, D)
    rng = np.random.default_rng(D)
    tt, ct = DT[dt]
    M, V = 20000, 40_000_000 // D
    assert 4 * V * D > 128 << 20
    ids = token_ids(rng, "skewed", 4, M // 4, V)
    ids[1] = rng.integers(0, V, M // 4)
    ids[2, :100] = -1                                                              # left out: no row of their own
    B = torch.from_numpy(rng.standard_normal((4, M // 4, D))).to(tt)
    st = status()
    got = run_tokens(torch.from_numpy(ids).to(DEV), B.to(DEV), ct, V, 1.0, None, 1.0, st=st)
    uniq, at = np.unique(ids, return_inverse=True)
    want, bound = R.tokens(at.reshape(ids.shape) - 1, R.f64(B), len(uniq) - 1, 1.0, None, 1.0)
    rows = torch.from_numpy(uniq[1:]).to(DEV)
    R.within(got[rows], want, bound)
    got[rows] = 0.0
    assert (got == 0).all() and st.item() == dp.DP_FLAG_BAD_INDEX


@pytest.mark.parametrize("T", [9, 700, 3000, 5000])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("V", [64, 5000])
def test_tokens_left_out(V, T, dt):
    """Padding rows are not looked at, bad ids are flagged, a broken norm poisons its sample's ids alone."""
    say("tokens left out", V, T, dt)
    rng = np.random.default_rng(T)
    tt, ct = DT[dt]
    N, D = 5, 24
    ids = rng.integers(0, V // 2, (N, T))
    ids[3] = V - 1 - rng.integers(0, 3, T)                                         # ids of the broken sample alone
    B = rng.standard_normal((N, T, D)).astype(np.float32)
    norm = np.array([0.5, -1.0, 2.0, math.inf, 1.0], dtype=np.float32)
    ids[1], B[1] = rng.integers(-2 ** 40, 2 ** 40, T), math.nan                    # behind the active batch
    Bt = torch.from_numpy(B).to(tt)
    st = status()
    got = run_tokens(torch.from_numpy(ids).to(DEV), Bt.to(DEV), ct, V, 1.0, torch.from_numpy(norm).to(DEV), 1.0, st=st)
    want, bound = R.tokens(ids, R.f64(Bt), V, 1.0, norm, 1.0)
    assert np.isnan(want).any() and np.isfinite(want[:V // 2]).all()
    R.within(got, want, bound)
    assert st.item() == 0
    bad = ids.copy()
    bad[0, ::2], bad[4, -1] = V, -3
    got = run_tokens(torch.from_numpy(bad).to(DEV), Bt.to(DEV), ct, V, 1.0, torch.from_numpy(norm).to(DEV), 1.0, st=st)
    want, bound = R.tokens(bad, R.f64(Bt), V, 1.0, norm, 1.0)
    R.within(got, want, bound)
    assert st.item() == dp.DP_FLAG_BAD_INDEX


@pytest.mark.parametrize("N,T", [(0, 5), (4, 0), (2, 3), (1, 9000), (1, 17000)])
@pytest.mark.parametrize("V", [33, 900])
def test_tokens_nothing_left(V, N, T):
    """No positions, or none that counts: zeros."""
    say("tokens nothing", N, T)
    ids = torch.full((N, T), -1, device=DEV)
    B = torch.full((N, T, 20), math.nan, device=DEV)
    st = status()
    assert (run_tokens(ids, B, dp.DP_F32, V, 1.0, None, 1.0, st=st) == 0).all()
    assert st.item() == (dp.DP_FLAG_BAD_INDEX if N * T else 0)
    st = status()
    norm = torch.full((N,), -1.0, device=DEV)
    assert (run_tokens(ids, B, dp.DP_F32, V, 1.0, norm, 1.0, st=st) == 0).all()
    assert st.item() == 0


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("D", [8, 96, 200])
@pytest.mark.parametrize("M", [50, 9001])
def test_tokens_unaligned(dt, D, M):
    say("tokens unaligned", dt, D, M)
    rng = np.random.default_rng(D + M)
    tt, ct = DT[dt]
    ids = token_ids(rng, "skewed", 1, M, 90)
    B = torch.from_numpy(rng.standard_normal((1, M, D))).to(tt)
    want, bound = R.tokens(ids, R.f64(B), 90, 1.0, None, 1.0)
    for by in (1, 2, 4):
        buf = torch.full((90 * D + 64,), 7.0, device=DEV)
        out = buf[by:by + 90 * D].view(90, D)
        R.within(run_tokens(torch.from_numpy(ids).to(DEV), unaligned(B, by), ct, 90, 1.0, None, 1.0, out=out), want, bound)
        assert (buf[:by] == 7).all() and (buf[by + 90 * D:] == 7).all()


def test_tokens_equal_the_csr_path():
    """The same sums as dp_grad_sample_embedding + dp_clip_accumulate_embedding, from whose norms they are clipped."""
    say("tokens csr")
    rng = np.random.default_rng(4)
    N, T, V, D = 16, 80, 500, 36
    ids = token_ids(rng, "skewed", N, T, V)
    B = torch.from_numpy(rng.standard_normal((N, T, D)).astype(np.float32)).to(DEV)
    idg = torch.from_numpy(ids).to(DEV)
    row_ptr, uniq = torch.empty(N + 1, dtype=torch.int64, device=DEV), torch.empty(N * T, dtype=torch.int64, device=DEV)
    rows, sq, norm = torch.empty(N * T, D, device=DEV), torch.empty(1, N, device=DEV), torch.empty(N, device=DEV)
    dp.dp_grad_sample_embedding(idg, B, dp.DP_F32, N, T, V, D, 1.25, row_ptr, uniq, rows, N * T, sq, None,
                                ws(dp.dp_grad_sample_embedding_workspace_bytes(N, T)))
    dp.dp_per_sample_norms(sq, 1, N, norm)
    C = float(norm.median())
    a = torch.empty(V, D, device=DEV)
    dp.dp_clip_accumulate_embedding(row_ptr, uniq, rows, N * T, norm, C, N, V, D, a, None,
                                    ws(dp.dp_clip_accumulate_embedding_workspace_bytes(N, V)))
    b = run_tokens(idg, B, dp.DP_F32, V, 1.25, norm, C)
    _, bound = R.tokens(ids, R.f64(B), V, 1.25, norm.cpu().numpy(), C)
    R.within(b, R.f64(a), 2 * bound)


# ------------------------------------------------------------------ global norm

def run_norm(ents, C, st=None):
    """ents: (g, out or None) tensors; returns the norm."""
    items = dp.make_grad_tensors([(g, o, g.numel(), dp.dtype_of(g)) for g, o in ents])
    norm = torch.full((1,), 7.0, device=DEV)
    dp.dp_clip_global_norm_many(items, len(ents), C, norm, st, ws(dp.dp_clip_global_norm_many_workspace_bytes(items, len(ents))))
    return norm


def check_norm(gs, outs, norm, C):
    """norm and outs for the gradients gs (host tensors)."""
    n64 = R.global_norm([R.f64(g) for g in gs])
    # squares and sums in 64 bits: one rounding to fp32 (and far less before it)
    assert abs(norm.item() - n64) <= (R.U32 + 1e-12) * n64
    c = float(R.clip_factors([n64], C)[0])
    for g, o in zip(gs, outs):
        if o is not None:
            want = c * R.f64(g)
            # the norm, the sum, the quotient and the product: four roundings in fp32, one to the type
            R.within(o, want, (5 * R.U32 + (R.half_step(o.dtype) if o.dtype == torch.bfloat16 else 0)) * np.abs(want) * 1.01
                     + float(torch.finfo(o.dtype).tiny))


COUNTS = [[1], [5, 0, 7], [64 * 16, 16], [4096], [4097, 8191, 3], [26010, 1, 255], [100] * 97, [3] * 200,
          [3_000_001, 17], [700_000, 900_001, 1_100_000, 5]]


@pytest.mark.parametrize("numels", COUNTS, ids=lambda v: "%dx%d" % (len(v), max(v)))
@pytest.mark.parametrize("mix", ["f32", "bf16", "mixed"])
@pytest.mark.parametrize("C", [0.5, 1e9])
def test_global_norm(numels, mix, C):
    say("norm", len(numels), max(numels), mix, C)
    rng = np.random.default_rng(sum(numels))
    tt = [torch.bfloat16 if mix == "bf16" or (mix == "mixed" and k % 2) else torch.float32 for k in range(len(numels))]
    gs = [torch.from_numpy(rng.standard_normal(n) * 0.3).to(t) for n, t in zip(numels, tt)]
    gg = [g.to(DEV) for g in gs]
    outs = [torch.full_like(g, 7.0) for g in gg]
    st = status()
    norm = run_norm(list(zip(gg, outs)), C, st)
    check_norm(gs, outs, norm, C)
    assert st.item() == 0
    assert all(torch.equal(a.cpu(), b) for a, b in zip(gg, gs))                     # the inputs stay
    if C > 1e8:
        assert all(torch.equal(a, b) for a, b in zip(gg, outs))                     # a factor of 1 changes no bit
    only = run_norm([(g, None) for g in gg], C)                                     # the norm alone
    assert abs(only.item() - norm.item()) <= R.U32 * 2 * norm.item()
    inplace = run_norm([(g, g) for g in gg], C)
    assert inplace.item() == norm.item()
    assert all(torch.equal(a, b) for a, b in zip(gg, outs))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_global_norm_unaligned(dt):
    say("norm unaligned", dt)
    rng = np.random.default_rng(8)
    tt, _ = DT[dt]
    gs = [torch.from_numpy(rng.standard_normal(n)).to(tt) for n in (1, 3, 9, 1000, 4096, 8203, 20000)]
    for by, to in ((1, 1), (3, 3), (1, 0), (0, 5), (2, 7)):
        gg = [unaligned(g, by) for g in gs]
        bufs = [torch.full((g.numel() + 32,), 7.0, dtype=tt, device=DEV) for g in gs]
        outs = [b[to:to + g.numel()] for b, g in zip(bufs, gs)]
        check_norm(gs, outs, run_norm(list(zip(gg, outs)), 1.0), 1.0)
        assert all((b[:to] == 7).all() and (b[to + g.numel():] == 7).all() for b, g in zip(bufs, gs))


@pytest.mark.parametrize("value", [1e30, 3e38, 1e-30, 1e-38, 0.0])
def test_global_norm_range(value):
    """Squares beyond fp32's range, and a norm that only fp32 itself bounds."""
    say("norm range", value)
    g = torch.full((300,), value, device=DEV)
    g[::2] *= -1
    out, st = torch.full_like(g, 7.0), status()
    norm = run_norm([(g, out)], 1e-3, st)
    n64 = math.sqrt(300) * float(np.float32(value))
    if n64 > 3.4e38:
        assert math.isinf(norm.item()) and out.isnan().all() and st.item() == dp.DP_FLAG_NONFINITE
    else:
        check_norm([g.cpu()], [out], norm, 1e-3)
        assert st.item() == 0


@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("n", [50, 3_000_000])
def test_global_norm_nonfinite(value, n):
    say("norm nonfinite", value, n)
    g, h = torch.ones(n, device=DEV), torch.ones(77, device=DEV, dtype=torch.bfloat16)
    g[n // 3] = value
    st = status()
    norm = run_norm([(h, h), (g, g)], 1.0, st)
    assert not math.isfinite(norm.item()) and st.item() == dp.DP_FLAG_NONFINITE
    assert g.isnan().all() and h.isnan().all()


def test_global_norm_empty_and_infinite_c():
    say("norm empty")
    assert run_norm([], 1.0).item() == 0.0
    e = torch.empty(0, device=DEV)
    assert run_norm([(e, e)], 1.0).item() == 0.0
    g = torch.full((10,), 100.0, device=DEV)
    o = torch.zeros_like(g)
    run_norm([(g, o)], math.inf)
    assert torch.equal(g, o)
