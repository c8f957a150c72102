"""Attention on the GPU at the ends of its range: scores that fp32 differences no longer resolve, gradients that cancel,
padding that holds anything, lists of tiles longer than one group."""
import sys

import numpy as np
import pytest
import torch

import token_model_ref as ref
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


# ---------------------------------------------------------------------------
# gradients that cancel
# ---------------------------------------------------------------------------

CANCEL = {  # N, Tq, Tk, Hq, Hk, D: few rows, a workgroup's waves, keys with their queries split, blocks of 128 rows, row by row
    "few": (3, 8, 8, 1, 1, 32), "small": (2, 200, 200, 2, 1, 64), "split": (1, 300, 40, 8, 2, 80), "small128": (1, 257, 257, 2, 2, 128),
    "blocks": (16, 150, 150, 16, 16, 128), "blocks64": (8, 260, 260, 32, 16, 64), "blocks96": (16, 97, 97, 16, 16, 96),
    "rows": (2, 70, 70, 2, 1, 160)}


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("shape", list(CANCEL))
def test_gradients_where_keys_and_values_differ_little(shape, causal):
    """Keys and values with a common part: dS sums to 0 over a row and what is left of dQ is small, so that dO.O has to be that of
    O before it was rounded to bf16."""
    say("cancel", shape, causal)
    N, Tq, Tk, Hq, Hk, D = CANCEL[shape]
    c = Case(*CANCEL[shape], "bf16", causal=causal, scale=2.0 ** -5, seed=31)
    rng = np.random.default_rng(32)
    for name, part in (("K", 0.25), ("V", 1 / 16)):
        common = torch.from_numpy(rng.standard_normal((N, 1, Hk, D)))
        setattr(c, name, (common + part * getattr(c, name).double()).to(torch.bfloat16))
    out, _ = c.run()
    Q, K, V, dO = [f64(getattr(c, k)) for k in ("Q", "K", "V", "dO")]
    G, U = Hq // Hk, 2.0 ** -24
    want = {k: np.zeros(x.shape) for k, x in (("dQ", Q), ("dK", K))}
    off, bound = ({k: np.zeros(x.shape) for k, x in want.items()} for _ in range(2))
    for n in range(N):
        see = c.mask.see[n]
        rows = see.any(1)
        for h in range(Hq):
            q, k, v, d = Q[n, :, h], K[n, :, h // G], V[n, :, h // G], dO[n, :, h]
            s = np.where(see, c.scale * (q @ k.T), -np.inf)
            top = np.where(rows, s.max(1), 0.0)[:, None]
            w = np.exp(s - top)
            tot = np.where(rows, w.sum(1), 1.0)[:, None]
            p, lse = w / tot, top + np.log(tot)
            dP = d @ v.T
            e = p * (dP - (p * dP).sum(1, keepdims=True))
            # a weight: its score's sum of D products, the scale, lse and their difference; a weight is off by some of itself
            ep = 2 * U * ((D + 4) * c.scale * (np.abs(q) @ np.abs(k).T) + 8 * (1 + np.abs(lse)))
            size = np.where(see, np.abs(d) @ np.abs(v).T, 0.0).max(1, keepdims=True)
            # dO.V and dO.O are fp32 sums of D and of D + Tk products, the latter corrected by what it lacks (the sum of p (dO.V - dO.O),
            # 2^-8 of the size at the most, off by p's error); dS goes into its products as two bf16 values (2^-16)
            ee = np.abs(e) * (ep + 2.0 ** -16 + 4 * U) + p * size * (2 * U * (2 * D + Tk + 8) + 2.0 ** -8 * ep.max(1, keepdims=True))
            rounded = f64(torch.from_numpy((p @ v).astype(np.float32)).to(torch.bfloat16))
            eo = p * (dP - (d * rounded).sum(1, keepdims=True))
            for x, y, z in ((want, e, False), (off, eo, False), (bound, ee + 2 * U * (Tk + Tq * G) * np.abs(e), True)):
                a, b = (np.abs(k), np.abs(q)) if z else (k, q)
                x["dQ"][n, :, h] = c.scale * (y @ a)
                x["dK"][n, :, h // G] += c.scale * (y.T @ b)
    for k in ("dQ", "dK"):
        b = bound[k] + 2.0 ** -8 * (np.abs(want[k]) + bound[k]) + 2.0 ** -126
        # (with dO.O from the rounded O dQ's bound would not hold; dK's sum over many queries may hide it)
        assert k == "dK" or (np.abs(off[k] - want[k]) > 4 * b).any()
        wrong = np.abs(f64(out[k]) - want[k]) / b
        assert (wrong <= 1).all(), (k, float(wrong.max()), float((wrong > 1).mean()))


# ---------------------------------------------------------------------------
# padding
# ---------------------------------------------------------------------------

PADDED = {  # N, Tq, Tk, Hq, Hk, D: a workgroup's waves, queries split, blocks of 128 rows and keys, unaligned heads
    "small": (3, 90, 90, 4, 2, 64), "split": (3, 300, 40, 4, 2, 80), "blocks": (16, 150, 150, 16, 16, 64), "blocks128": (9, 260, 260, 32, 32, 128),
    "odd": (3, 70, 70, 4, 2, 33)}


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["plain", "cap", "causal", "last"])
@pytest.mark.parametrize("shape", list(PADDED))
def test_padding_holds_anything_at_no_cost(shape, kind, dt):
    """What lies in padding (queries, their dO, keys, values) changes no bit: sums that it reached would not be finite, and would be
    formed again in another order and at another speed."""
    say("padding", shape, kind, dt)
    N, Tq, Tk, Hq, Hk, D = PADDED[shape]
    last = kind == "last"
    lens = np.random.default_rng(41).integers(0, Tk + 1, N)
    lens[0], lens[1] = Tk // 2 + 1, Tk
    c = Case(N, Tq, Tk, Hq, Hk, D, dt, causal=kind in ("causal", "last"), last=last, lens=lens, cap=5.0 if kind == "cap" else 0.0, seed=42)
    outs = []
    for fill in (0.0, float("nan"), float("inf"), float(torch.finfo(c.tt).max)):
        for n in range(N):
            L = int(c.mask.L[n])
            c.K[n, L:], c.V[n, L:] = fill, fill
            pad = slice(0, max(0, Tq - L)) if last else slice(min(L, Tq), Tq)
            c.Q[n, pad], c.dO[n, pad] = fill, fill
        out, lse = c.run()
        outs.append([lse, *out.values()])
    bits = lambda x: x.contiguous().view(torch.int16 if x.dtype == torch.bfloat16 else torch.int32)  # noqa: E731
    for other in outs[1:]:
        for k, a, b in zip(("lse", "O", "dQ", "dK", "dV"), outs[0], other):
            assert bool(torch.isfinite(b if k != "lse" else b.nan_to_num(neginf=0.0)).all()), k
            assert torch.equal(bits(a), bits(b)), k


# ---------------------------------------------------------------------------
# documents over more tiles than one list holds (1024 of 32 or 64 keys)
# ---------------------------------------------------------------------------

def documents(rng, T, lengths, again):
    """[T]: documents of `lengths` in turn, every `again`-th one under an earlier one's number, some places without a document."""
    row, k = np.empty(T, dtype=np.int64), 0
    at = 0
    while at < T:
        n = int(rng.integers(*lengths))
        row[at:at + n] = k if again == 0 or k % again else k // 2
        at, k = at + n, k + 1
    row[rng.integers(0, T, 20)] = -1
    return row.astype(np.int32)


def part_mask(see):
    m = ref.Mask(1, *see.shape)
    m.see = [see]
    return m


def compare(got, want, bound, what):
    wrong = np.abs(f64(got) - want) > bound
    assert not wrong.any(), (what, int(wrong.sum()))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_documents_in_several_lists_single_tokens(dt):
    """One query a sample over 33500 keys, by a workgroup that is not split: 1047 tiles of 32."""
    say("lists", "single", dt)
    N, Tk, H, D, tt = 16, 33500, 64, 8, {"f32": torch.float32, "bf16": torch.bfloat16}[dt]
    rng = np.random.default_rng(51)
    g = torch.Generator(device=DEV)
    g.manual_seed(52)
    Q, K, V = [torch.randn((N, T, H * D), generator=g, device=DEV, dtype=tt) for T in (1, Tk, Tk)]
    lens = rng.integers(32700, Tk + 1, N).astype(np.int32)
    lens[0], lens[1], lens[2] = Tk, 500, 32768
    docs = np.stack([documents(rng, Tk, (10, 900), 3) for _ in range(N)])
    for n in range(N):                                 # the last query's document: at its end, about the first list's, and at the start
        p = int(lens[n]) - 1
        docs[n, p - 40 - 10 * n:p + 1] = 7
        docs[n, 5:60:7] = 7
        docs[n, 32768 - 20:32768 + 20] = 7
    dev = lambda x: torch.from_numpy(x).to(DEV)  # noqa: E731
    a = dp.make_attention(dp.DP_F32 if dt == "f32" else dp.DP_BF16, N, 1, Tk, H, H, D, D ** -0.5,
                          dp.DP_ATTENTION_CAUSAL | dp.DP_ATTENTION_LAST, lens=dev(lens), docs=dev(docs))
    assert dp.dp_attention_forward_workspace_bytes(a) == 0
    O, lse = torch.full_like(Q, float("nan")), torch.full((N, H, 1), float("nan"), device=DEV)
    dp.dp_attention_forward(a, Q, K, V, O, lse)
    for n in range(N):
        L = int(lens[n])
        at = torch.from_numpy(np.flatnonzero((docs[n, :L] == 7) & (docs[n, L - 1] == 7))).to(DEV)
        part = lambda x: f64(x.reshape(1, -1, H, D))  # noqa: E731
        (o, l), (eo, el) = ref.attention(part(Q[n]), part(K[n, at]), part(V[n, at]), part_mask(np.ones((1, len(at)), dtype=bool)),
                                         float(np.float32(D ** -0.5)), dt=tt)
        compare(O[n].reshape(1, 1, H, D), o, eo, ("O", n))
        compare(lse[n:n + 1], l, el, ("lse", n))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("Tq,Tk,Hq,Hk", [(66100, 66100, 1, 1), (3, 33500, 4, 2), (200, 70000, 2, 2)])
def test_documents_in_several_lists(Tq, Tk, Hq, Hk, dt):
    """Forward and backward: all queries of a sample of 66100, and few over more keys than a list has."""
    say("lists", Tq, Tk, Hq, Hk, dt)
    last, D = Tq < Tk, 16
    rng = np.random.default_rng(53)
    docs = documents(rng, Tk, (50, 400), 5)
    docs[32760:32780], docs[65500:65700] = docs[32759], docs[min(65499, Tk - 1)]      # across the lists' ends
    if last:                                           # the queries' documents start and end all over the keys
        ids = docs[Tk - Tq:][docs[Tk - Tq:] >= 0]
        for k in np.unique(ids):
            s = rng.integers(0, Tk - 60, 12)
            for b in s:
                docs[b:b + rng.integers(1, 50)] = k
    tt = {"f32": torch.float32, "bf16": torch.bfloat16}[dt]
    x = {k: torch.from_numpy(rng.standard_normal((1, T, H, D))).to(tt) for k, T, H in (("Q", Tq, Hq), ("K", Tk, Hk), ("V", Tk, Hk), ("dO", Tq, Hq))}
    flags = dp.DP_ATTENTION_CAUSAL | (dp.DP_ATTENTION_LAST if last else 0)
    a = dp.make_attention(dp.DP_F32 if dt == "f32" else dp.DP_BF16, 1, Tq, Tk, Hq, Hk, D, 0.25, flags,
                          docs=torch.from_numpy(docs[None].copy()).to(DEV))
    d = {k: v.reshape(1, v.shape[1], -1).to(DEV) for k, v in x.items()}
    o = {k: torch.full_like(d[l], float("nan")) for k, l in (("O", "Q"), ("dQ", "Q"), ("dK", "K"), ("dV", "V"))}
    lse = torch.full((1, Hq, Tq), float("nan"), device=DEV)
    dp.dp_attention_forward(a, d["Q"], d["K"], d["V"], o["O"], lse, ws_of(dp.dp_attention_forward_workspace_bytes(a)))
    dp.dp_attention_backward(a, d["Q"], d["K"], d["V"], o["O"], lse, d["dO"], o["dQ"], o["dK"], o["dV"],
                             ws_of(dp.dp_attention_backward_workspace_bytes(a)))
    got = {k: f64(v).reshape(1, v.shape[1], -1, D) for k, v in o.items()}
    X = {k: f64(v) for k, v in x.items()}
    first = Tk - Tq if last else 0
    keys_left = np.ones(Tk, dtype=bool)
    for k in np.unique(docs[docs >= 0]):
        j = np.flatnonzero(docs == k)
        i = j[j >= first] - first
        if len(i) == 0:
            continue
        keys_left[j] = False
        see = j[None, :] <= (i + first)[:, None]
        args = (part_mask(see), 0.25, 0.0, None, tt)
        q, kk, v, do = X["Q"][:, i], X["K"][:, j], X["V"][:, j], X["dO"][:, i]
        (O, l), (eO, el) = ref.attention(q, kk, v, *args)
        compare(torch.from_numpy(got["O"][:, i]), O, eO, ("O", k))
        compare(lse[:, :, torch.from_numpy(i).to(DEV)], l, el, ("lse", k))
        grads, errs = ref.attention_grads(q, kk, v, do, *args)
        for name, at, want, err in zip(("dQ", "dK", "dV"), (i, j, j), grads, errs):
            compare(torch.from_numpy(got[name][:, at]), want, err, (name, k))
    none = docs[first:first + Tq] < 0
    assert (got["O"][:, none] == 0).all() and (got["dQ"][:, none] == 0).all()
    assert (got["dK"][:, keys_left] == 0).all() and (got["dV"][:, keys_left] == 0).all()


# ---------------------------------------------------------------------------
# scores far past their cap
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["cap", "both"])
@pytest.mark.parametrize("shape", ["small", "blocks", "rows", "odd"])
def test_gradients_of_scores_far_past_their_cap(shape, kind, dt):
    """All scores 5 to 9 caps large, of either sign: 1 - tanh^2 is 2e-4 to 6e-8, and has to be right by itself, not as a difference."""
    say("saturated", shape, kind, dt)
    N, T, Hq, Hk, D = {"small": (2, 90, 2, 1, 64), "blocks": (16, 150, 16, 16, 64), "rows": (1, 50, 2, 2, 136), "odd": (2, 60, 2, 1, 33)}[shape]
    c = Case(N, T, T, Hq, Hk, D, dt, causal=kind == "both", cap=1.0, slopes=kind == "both", scale=1.0, seed=61)
    rng = np.random.default_rng(62)
    u = rng.standard_normal(D)
    u /= np.sqrt(u @ u)
    put = lambda x: torch.from_numpy(x).to(c.tt)  # noqa: E731
    c.Q = put(np.sqrt(7) * u + 0.03 * rng.standard_normal(c.Q.shape))
    c.K = put(rng.choice([-1.0, 1.0], (N, T, Hk, 1)) * np.sqrt(7) * u + 0.03 * rng.standard_normal(c.K.shape))
    out, _ = c.run()
    Q, K, V, dO = [f64(getattr(c, k)) for k in ("Q", "K", "V", "dO")]
    G, U, bf16 = Hq // Hk, 2.0 ** -24, dt == "bf16"
    want = {k: np.zeros(x.shape) for k, x in (("dQ", Q), ("dK", K))}
    bound = {k: np.zeros(x.shape) for k, x in want.items()}
    for n in range(N):
        see = c.mask.see[n]
        for h in range(Hq):
            q, k, v, d = Q[n, :, h], K[n, :, h // G], V[n, :, h // G], dO[n, :, h]
            y = q @ k.T
            assert np.abs(y).min() > 5 and np.abs(y).max() < 9
            s = np.where(see, np.tanh(y) - (0.0 if c.slopes is None else c.slopes[h]) * c.mask.far[n], -np.inf)
            w = np.exp(s - s.max(1, keepdims=True))
            p = w / w.sum(1, keepdims=True)
            r = 1 / (1 + np.exp(2 * np.abs(y)))
            bend = 4 * r * (1 - r)
            dP = d @ v.T
            e = p * (dP - (p * dP).sum(1, keepdims=True)) * bend
            # bend's logarithm has slope 2 at most: twice the score's error, a sum of D products; the exponential's argument, the quotient
            # and the product 16 half steps in all.  p: the capped score, bias, lse and exp2, 64 half steps of sizes below 40
            ey = U * (D + 8) * (np.abs(q) @ np.abs(k).T)
            ep = 64 * 40 * U
            size = np.where(see, np.abs(d) @ np.abs(v).T, 0.0).max(1, keepdims=True)
            ee = np.abs(e) * (2 * ey * 1.01 + 16 * U + 36 * U + ep + (2.0 ** -16 if bf16 else 0)) + p * bend * size * (
                2 * U * (2 * D + T + 8) + (2.0 ** -8 * ep if bf16 else 0))
            ee += 2 * U * (T + T * G) * np.abs(e)
            for x, z, kk, qq in ((want, e, k, q), (bound, ee, np.abs(k), np.abs(q))):
                x["dQ"][n, :, h] = z @ kk
                x["dK"][n, :, h // G] += z.T @ qq
    half = 2.0 ** -8 if bf16 else U
    for k in ("dQ", "dK"):
        b = bound[k] + half * (np.abs(want[k]) + bound[k]) + 2.0 ** -126
        wrong = np.abs(f64(out[k]) - want[k]) / b
        assert (wrong <= 1).all(), (k, float(wrong.max()), float((wrong > 1).mean()))
