"""The language-model operators where element offsets pass 32 bits: tables, sums, activations and tensors of more than
2^31 elements."""
import math
import sys

import pytest
import torch

from paper_2109_12298_amd import binding as dp

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def say(*a):
    print("[case]", *a, file=sys.stderr, flush=True)


def ws(n):
    return torch.empty(max(int(n), 16), dtype=torch.uint8, device=DEV)


@pytest.fixture(autouse=True)
def free():
    yield
    torch.cuda.empty_cache()


def test_lookup_and_tokens_of_a_large_table():
    say("large table")
    V, D, T = 2_200_000, 1024, 3000                                   # 2.25e9 elements
    E = torch.empty((V, D), dtype=torch.bfloat16, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(1)
    ids = torch.randint(V - 50, V, (1, T), generator=g, device=DEV)
    ids[0, :4] = torch.tensor([0, V - 1, 2 ** 21, V // 2], device=DEV)
    uniq = torch.unique(ids)
    E[uniq] = torch.randn((len(uniq), D), generator=g, device=DEV).to(torch.bfloat16)
    Y = torch.empty((1, T, D), dtype=torch.bfloat16, device=DEV)
    dp.dp_embedding_lookup(ids, E, dp.DP_BF16, 1, T, V, D, 2.0, Y, dp.DP_BF16)
    assert torch.equal(Y[0], (E[ids[0]].float() * 2.0).to(torch.bfloat16))
    del E
    for n in (T, 500):                                                # both paths of the gradient
        S = torch.full((V, D), 7.0, device=DEV)                       # 9 GB
        B = Y[:, :n].contiguous()
        dp.dp_clip_accumulate_tokens(ids[:, :n].contiguous(), B, dp.DP_BF16, 1, n, V, D, 1.0, None, 1.0, S, None,
                                     ws(dp.dp_clip_accumulate_tokens_workspace_bytes(1, n, V, D, dp.DP_BF16)))
        want = torch.zeros((60, D), dtype=torch.float64, device=DEV)
        tail = ids[0, :n] >= V - 60
        want.index_add_(0, ids[0, :n][tail] - (V - 60), B[0][tail].double())
        # at most n fp32 additions of values of order 10: n 2^-23 of the sum of the terms, under n / 2^23 * 10 n / 50
        assert (S[V - 60:].double() - want).abs().max() <= n * 2.0 ** -23 * 10 * (n / 40)
        for i, v in enumerate((0, None, 2 ** 21, V // 2)):
            if v is not None:
                assert torch.equal(S[v], B[0, i].float())
        assert S[1:V // 2].abs().max() == 0
        assert float(S.abs().sum(1).ne(0).sum()) == len(torch.unique(ids[0, :n]))
        del S


@pytest.mark.parametrize("M,K,F", [(280_000, 64, 8192)])
def test_ffn_of_many_positions(M, K, F):
    say("large ffn", M, K, F)
    g = torch.Generator(device=DEV).manual_seed(2)
    bf = torch.bfloat16
    X = torch.randn((M, K), generator=g, device=DEV).to(bf)
    Wg, Wu = [(torch.randn((F, K), generator=g, device=DEV) / math.sqrt(K)).to(bf) for _ in range(2)]
    H, G, U = [torch.full((M, F), 7.0, dtype=bf, device=DEV) for _ in range(3)]
    assert H.numel() > 2 ** 31
    dp.dp_gated_ffn_forward(X, Wg, Wu, dp.DP_BF16, M, K, F, dp.DP_ACT_SILU, H, G, U,
                            ws(dp.dp_gated_ffn_forward_workspace_bytes(M, K, F, dp.DP_BF16)))
    some = torch.tensor([0, 1, 255, 256, M // 2, 262143, 262144, M - 257, M - 1], device=DEV)
    g64, u64 = X[some].double() @ Wg.double().t(), X[some].double() @ Wu.double().t()
    # one rounding to bf16, and sums of 64 terms in fp32 of values of order 1
    tol = lambda w: 2.0 ** -8 * w.abs() * 1.01 + 1e-4  # noqa: E731
    for got, want in ((G, g64), (U, u64), (H, g64 * torch.sigmoid(g64) * u64)):
        assert ((got[some].double() - want).abs() <= tol(want)).all()
    dX = torch.full((M, K), 7.0, dtype=bf, device=DEV)
    rows = [G[some].double(), U[some].double(), H[some].double()]
    dp.dp_gated_ffn_backward(H, G, U, Wg, Wu, dp.DP_BF16, M, K, F, dp.DP_ACT_SILU, G, U, dX,
                             ws(dp.dp_gated_ffn_backward_workspace_bytes(M, K, F, dp.DP_BF16)))     # BG in G, BU in U
    p = torch.sigmoid(rows[0])
    for got, want in ((G, rows[2] * rows[1] * (p + rows[0] * p * (1 - p))), (U, rows[2] * rows[0] * p)):
        assert ((got[some].double() - want).abs() <= tol(want)).all()
    want = G[some].double() @ Wg.double() + U[some].double() @ Wu.double()
    size = G[some].double().abs() @ Wg.double().abs() + U[some].double().abs() @ Wu.double().abs()
    assert ((dX[some].double() - want).abs() <= 2.0 ** -8 * want.abs() + 2 * (2 * F + 1) * 2.0 ** -24 * size).all()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_ffn_of_long_sums(dt):
    """Rows of more than 2^21 values on either side of the block."""
    say("long sums", dt)
    tt, ct = (torch.float32, dp.DP_F32) if dt == "f32" else (torch.bfloat16, dp.DP_BF16)
    g = torch.Generator(device=DEV).manual_seed(4)
    n, M, few = 2 ** 21 + 8, 66, 3
    # additions in any order (six products to a term in fp32), each rounded to 2^-24 of a partial sum, which stays under
    # 5 standard deviations: sqrt(n) forward, under 3 sqrt(n) backward (2 n terms of deviation under 2); and the result's
    eps = 2.0 ** -24 if dt == "f32" else 2.0 ** -8
    randn = lambda *s: torch.randn(s, generator=g, device=DEV).to(tt)  # noqa: E731
    X, Wg, Wu = randn(M, n), randn(few, n), randn(few, n)
    H, G, U = [torch.full((M, few), 7.0, dtype=tt, device=DEV) for _ in range(3)]
    dp.dp_gated_ffn_forward(X, Wg, Wu, ct, M, n, few, dp.DP_ACT_SILU, H, G, U,
                            ws(dp.dp_gated_ffn_forward_workspace_bytes(M, n, few, ct)))
    for got, W in ((G, Wg), (U, Wu)):
        want = X.double() @ W.double().t()
        assert ((got.double() - want).abs() <= eps * want.abs() + 6 * n * 2.0 ** -24 * 5 * math.sqrt(n)).all()
    del X, Wg, Wu
    dH, G, U = randn(M, n), randn(M, n), randn(M, n)
    Wg, Wu = randn(n, few), randn(n, few)
    dX = torch.full((M, few), 7.0, dtype=tt, device=DEV)
    dp.dp_gated_ffn_backward(dH, G, U, Wg, Wu, ct, M, few, n, dp.DP_ACT_SILU, G, U, dX,
                             ws(dp.dp_gated_ffn_backward_workspace_bytes(M, few, n, ct)))
    want = G.double() @ Wg.double() + U.double() @ Wu.double()
    assert G.isfinite().all() and U.isfinite().all() and want.abs().min() > 0
    assert ((dX.double() - want).abs() <= eps * want.abs() + 12 * n * 2.0 ** -24 * 15 * math.sqrt(n)).all()


@pytest.mark.parametrize("M", [66, 40, 9])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_ffn_of_long_sums_exactly(M, dt):
    """The same lengths on whole numbers small enough that every sum is exact in fp32 in any order (|partial sums| under
    2^24: forward at most 4 n = 2^23, backward 300 standard deviations of sqrt(n (0.9 + 32^2 * 1.4)) = 5.5e4): the
    outputs are the exact sums, rounded once."""
    say("long sums exactly", M, dt)
    tt, ct = (torch.float32, dp.DP_F32) if dt == "f32" else (torch.bfloat16, dp.DP_BF16)
    g = torch.Generator(device=DEV).manual_seed(6)
    n, few = 2 ** 21 + 8, 3
    ints = lambda top, *s: torch.randint(-top, top + 1, s, generator=g, device=DEV).to(tt)  # noqa: E731
    X, Wg, Wu = ints(2, M, n), ints(2, few, n), ints(2, few, n)
    H, G, U = [torch.full((M, few), 7.0, dtype=tt, device=DEV) for _ in range(3)]
    dp.dp_gated_ffn_forward(X, Wg, Wu, ct, M, n, few, dp.DP_ACT_SILU, H, G, U,
                            ws(dp.dp_gated_ffn_forward_workspace_bytes(M, n, few, ct)))
    g64, u64 = X.double() @ Wg.double().t(), X.double() @ Wu.double().t()
    assert g64.abs().mean() > 1000 and u64.abs().mean() > 1000
    assert torch.equal(G, g64.to(tt)) and torch.equal(U, u64.to(tt))
    h64 = g64 * torch.sigmoid(g64) * u64
    # expf, the sum, the quotient and two products in fp32 (8 half steps), and the rounding to bf16; gates under the
    # smallest normal value may be 0
    eps = 8 * 2.0 ** -24 if dt == "f32" else 1.01 * 2.0 ** -8
    assert ((H.double() - h64).abs() <= eps * h64.abs() + 1e-30).all()
    del X, Wg, Wu
    dH, U = ints(1, M, n), ints(1, M, n)
    G = torch.full((M, n), 32.0, dtype=tt, device=DEV)                # act(32) = 32, act'(32) = 1 in fp32
    Wg, Wu = ints(2, n, few), ints(2, n, few)
    BG, BU = torch.full_like(G, 7.0), torch.full_like(G, 7.0)
    dX = torch.full((M, few), 7.0, dtype=tt, device=DEV)
    dp.dp_gated_ffn_backward(dH, G, U, Wg, Wu, ct, M, few, n, dp.DP_ACT_SILU, BG, BU, dX,
                             ws(dp.dp_gated_ffn_backward_workspace_bytes(M, few, n, ct)))
    assert torch.equal(BG, dH * U) and torch.equal(BU, 32 * dH)
    want = BG.double() @ Wg.double() + BU.double() @ Wu.double()
    assert want.abs().mean() > 10000
    assert torch.equal(dX, want.to(tt))


def test_norm_of_a_large_tensor():
    say("large norm")
    n = 2 ** 31 + 12345
    g = torch.full((n,), 0.5, dtype=torch.bfloat16, device=DEV)
    g[-7:] = 3.0
    out = torch.zeros_like(g)
    norm = torch.zeros(1, device=DEV)
    items = dp.make_grad_tensors([(g, out, n, dp.DP_BF16)])
    dp.dp_clip_global_norm_many(items, 1, 1.0, norm, None, ws(dp.dp_clip_global_norm_many_workspace_bytes(items, 1)))
    want = math.sqrt((n - 7) * 0.25 + 63.0)
    assert abs(norm.item() - want) <= 2.0 ** -24 * want * 1.01
    c = 1.0 / (want + 1e-6)
    for at, v in ((0, 0.5), (2 ** 31 - 1, 0.5), (2 ** 31, 0.5), (n - 8, 0.5), (n - 7, 3.0), (n - 1, 3.0)):
        assert abs(out[at].item() - c * v) <= (2.0 ** -8 + 2.0 ** -21) * c * v
    assert out[:-7].min() == out[:-7].max()
