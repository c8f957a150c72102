"""Refusals of the language-model operators on the host (nothing is enqueued; no GPU needed)."""
import math

import pytest
import torch

from paper_2109_12298_amd import binding as dp

# addresses below are never dereferenced: every call fails validation first, or has nothing to do
FAKE = 0x10000


def code_of(fn, *a, **k):
    try:
        fn(*a, stream=0, **k)
    except dp.DPError as e:
        return e.code
    return dp.DP_OK


def test_lookup_refusals():
    f = dp.dp_embedding_lookup
    ok = dict(ids=FAKE, E=FAKE, dt=dp.DP_F32, N=2, T=3, V=10, D=4, scale=1.0, Y=FAKE, dt_y=dp.DP_BF16)
    call = lambda **k: code_of(f, **{**ok, **k})  # noqa: E731
    assert call(dt=7) == dp.DP_EDTYPE and call(dt_y=-1) == dp.DP_EDTYPE
    for bad in (dict(N=-1), dict(T=-1), dict(V=0), dict(D=0), dict(V=2 ** 31), dict(ids=None), dict(E=None), dict(Y=None)):
        assert call(**bad) == dp.DP_EINVAL, bad
    for much in (dict(N=2 ** 20, T=2 ** 11), dict(N=2 ** 62, T=2 ** 62), dict(D=2 ** 23)):
        assert call(**much) == dp.DP_EUNSUPPORTED, much
    assert call(N=0, ids=None, E=None, Y=None) == dp.DP_OK
    assert call(T=0, ids=None, E=None, Y=None) == dp.DP_OK


def test_tokens_refusals():
    f = dp.dp_clip_accumulate_tokens
    lib = dp.lib().dp_clip_accumulate_tokens
    need = dp.dp_clip_accumulate_tokens_workspace_bytes(2, 3, 10, 4, dp.DP_F32)
    assert need > 0

    def call(ids=FAKE, B=FAKE, dt=dp.DP_F32, N=2, T=3, V=10, D=4, norm=FAKE, C=1.0, sum=FAKE, ws=FAKE, ws_bytes=need):
        return lib(ids, B, dt, N, T, V, D, 1.0, norm, C, sum, None, ws, ws_bytes, None)

    assert call(dt=3) == dp.DP_EDTYPE
    for bad in (dict(N=-1), dict(T=-2), dict(V=0), dict(D=0), dict(V=2 ** 31), dict(ids=None), dict(B=None), dict(sum=None),
                dict(C=0.0), dict(C=-1.0), dict(C=math.nan), dict(ws=None), dict(ws=FAKE + 4), dict(ws_bytes=need - 1)):
        assert call(**bad) == dp.DP_EINVAL, bad
    for much in (dict(N=2 ** 15, T=2 ** 15), dict(N=2 ** 40, T=2 ** 40), dict(D=2 ** 22),
                 dict(N=2 ** 14, T=2 ** 14, D=2 ** 10), dict(V=2 ** 30, D=2 ** 10)):
        assert call(**much) == dp.DP_EUNSUPPORTED, much
    w = dp.dp_clip_accumulate_tokens_workspace_bytes
    assert w(0, 3, 10, 4, 0) == 0 and w(3, 0, 10, 4, 0) == 0 and w(-1, 3, 10, 4, 0) == 0 and w(2, 3, 10, 4, 9) == 0
    assert code_of(f, FAKE, FAKE, dp.DP_F32, 2, 3, 10, 4, 1.0, None, 1.0, FAKE) == dp.DP_EINVAL       # no workspace


def test_tokens_workspace_covers_every_alignment():
    """The columns per lane follow the arrays' alignment; the size asked for does not."""
    w = dp.dp_clip_accumulate_tokens_workspace_bytes
    for N, T, V, D in ((1, 1, 1, 1), (4, 700, 100, 64), (64, 256, 10000, 100), (16, 4096, 50000, 2048), (1, 9000, 7, 533)):
        for dt in (dp.DP_F32, dp.DP_BF16):
            assert w(N, T, V, D, dt) >= 8 * N * T + 2 * 4 * D


def test_ffn_refusals():
    L = dp.lib()
    fneed = dp.dp_gated_ffn_forward_workspace_bytes
    bneed = dp.dp_gated_ffn_backward_workspace_bytes

    def fwd(X=FAKE, Wg=FAKE, Wu=FAKE, dt=dp.DP_F32, M=4, D=8, F=16, act=0, H=FAKE, G=FAKE, U=FAKE, ws=FAKE, n=None):
        return L.dp_gated_ffn_forward(X, Wg, Wu, dt, M, D, F, act, H, G, U, ws, fneed(M, D, F, dt) if n is None else n, None)

    def bwd(dH=FAKE, G=FAKE, U=FAKE, Wg=FAKE, Wu=FAKE, dt=dp.DP_F32, M=4, D=8, F=16, act=0, BG=FAKE, BU=2 * FAKE, dX=FAKE,
            ws=FAKE, n=None):
        return L.dp_gated_ffn_backward(dH, G, U, Wg, Wu, dt, M, D, F, act, BG, BU, dX, ws,
                                       bneed(M, D, F, dt) if n is None else n, None)

    for call, outs in ((fwd, ("X", "Wg", "Wu", "H")), (bwd, ("dH", "G", "U", "Wg", "Wu", "BG", "BU"))):
        assert call(dt=2) == dp.DP_EDTYPE
        for bad in [dict(M=-1), dict(D=0), dict(F=0), dict(act=2), dict(act=-1)] + [{k: None} for k in outs]:
            assert call(**bad) == dp.DP_EINVAL, bad
        for much in (dict(M=2 ** 31), dict(F=2 ** 27), dict(D=2 ** 27), dict(M=2 ** 20, F=2 ** 16), dict(D=2 ** 18, F=2 ** 18),
                     dict(M=2 ** 62, D=2 ** 62)):
            assert call(**much) == dp.DP_EUNSUPPORTED, much
        assert call(M=0) == dp.DP_OK
    assert fwd(G=None) == dp.DP_EINVAL and fwd(U=None) == dp.DP_EINVAL
    assert bwd(BU=FAKE) == dp.DP_EINVAL                                      # both backprops into one array
    assert fwd(M=0, X=None, Wg=None, Wu=None, H=None, G=None, U=None, ws=None) == dp.DP_OK
    for need, call in ((fneed, fwd), (bneed, bwd)):
        assert need(0, 8, 16, 0) == 0 and need(4, 0, 16, 0) == 0 and need(4, 8, 16, 5) == 0
        for M, D, F in ((1, 4096, 11008), (7, 100, 130), (512, 768, 2048), (4096, 500, 1333)):
            for dt in (dp.DP_F32, dp.DP_BF16):
                n = need(M, D, F, dt)
                if n > 0:
                    assert call(M=M, D=D, F=F, dt=dt, n=n - 1) == dp.DP_EINVAL
                    assert call(M=M, D=D, F=F, dt=dt, ws=None) == dp.DP_EINVAL
                    assert call(M=M, D=D, F=F, dt=dt, ws=FAKE + 2) == dp.DP_EINVAL


def test_global_norm_refusals():
    L = dp.lib()
    size = dp.dp_clip_global_norm_many_workspace_bytes
    mk = dp.make_grad_tensors
    good = mk([(FAKE, FAKE, 100, dp.DP_F32), (FAKE, None, 5000, dp.DP_BF16), (None, None, 0, dp.DP_F32)])
    need = size(good, 3)
    assert need >= 16 + 8 * 3

    def call(items=good, count=3, C=1.0, norm=FAKE, ws=FAKE, n=need):
        return L.dp_clip_global_norm_many(items, count, C, norm, None, ws, n, None)

    for bad in (dict(count=-1), dict(count=65537), dict(items=None), dict(C=0.0), dict(C=-2.0), dict(C=math.nan),
                dict(norm=None), dict(ws=None), dict(ws=FAKE + 8), dict(n=need - 1)):
        assert call(**bad) == dp.DP_EINVAL, bad
    for ent, code in (((FAKE, FAKE, 4, 7), dp.DP_EDTYPE), ((FAKE, FAKE, -1, 0), dp.DP_EINVAL),
                      ((None, FAKE, 4, 0), dp.DP_EINVAL), ((FAKE + 2, FAKE, 4, 0), dp.DP_EINVAL),
                      ((FAKE, FAKE + 1, 4, 1), dp.DP_EINVAL), ((FAKE, FAKE, 2 ** 40, 0), dp.DP_EUNSUPPORTED)):
        items = mk([(FAKE, FAKE, 100, dp.DP_F32), ent])
        assert call(items=items, count=2) == code, ent
        assert size(items, 2) == 0


def test_tensors_are_checked_before_the_call():
    """A host tensor, a view with strides, a wrong type or a short buffer never reaches the GPU."""
    ids, E, Y = torch.zeros(6, dtype=torch.int64), torch.zeros(10, 4), torch.zeros(6, 4)
    with pytest.raises(ValueError, match="not on a GPU"):
        dp.dp_embedding_lookup(ids, E, dp.DP_F32, 2, 3, 10, 4, 1.0, Y, dp.DP_F32, stream=0)
    with pytest.raises(ValueError, match="not on a GPU"):
        dp.make_grad_tensors([(E, E, 40, dp.DP_F32)])

    class Fake:                                      # stands for a GPU tensor; only its description is read
        def __init__(self, dtype, n, dense=True, device=0):
            self.dtype, self.n, self.dense, self.device = dtype, n, dense, device

        def get_device(self):
            return self.device

        def is_contiguous(self):
            return self.dense

        def numel(self):
            return self.n

        def data_ptr(self):
            return FAKE

    def ptr(*xs):
        return dp._tensors("f", *[("x", x, torch.float32, 40) for x in xs])

    assert ptr(Fake(torch.float32, 40), None, FAKE) == (0, [FAKE, None, FAKE])
    assert ptr(None, FAKE) == (None, [None, FAKE])
    with pytest.raises(TypeError, match="not torch.float32"):
        ptr(Fake(torch.bfloat16, 40))
    with pytest.raises(ValueError, match="not contiguous"):
        ptr(Fake(torch.float32, 40, dense=False))
    with pytest.raises(ValueError, match="40 are needed"):
        ptr(Fake(torch.float32, 39))
    with pytest.raises(ValueError, match="other arguments on GPU 0"):
        ptr(Fake(torch.float32, 40), Fake(torch.float32, 40, device=1))

    items = dp.make_grad_tensors([(Fake(torch.float32, 40, device=1), None, 40, dp.DP_F32)])
    with pytest.raises(ValueError, match="on GPU 0, the tensors on GPU 1"):
        dp.dp_clip_global_norm_many(items, 1, 1.0, Fake(torch.float32, 1), None, FAKE, stream=0)
    for call in (dp.dp_clip_global_norm_many_workspace_bytes,
                 lambda items, n: dp.dp_clip_global_norm_many(items, n, 1.0, FAKE, None, FAKE, stream=0)):
        for few, n in ((items, 2), (None, 1)):       # more tensors than the array holds
            with pytest.raises(ValueError, match="tensors of an array of"):
                call(few, n)
    assert dp.dp_clip_global_norm_many_workspace_bytes(None, 0) == dp.dp_clip_global_norm_many_workspace_bytes(items, 0)


def test_item_lists_keep_their_tensors():
    """A list of items holds addresses: the tensors behind them live as long as the list."""
    import gc
    import weakref

    class Fake:                                      # stands for a GPU tensor
        dtype = torch.float32

        def get_device(self):
            return 0

        def is_contiguous(self):
            return True

        def numel(self):
            return 40

        def data_ptr(self):
            return FAKE

    def tensors(n):
        return [Fake() for _ in range(n)]

    for make, entry in ((dp.make_grad_tensors, lambda a, b, c, d: (a, b, 40, dp.DP_F32)),
                        (dp.make_params, lambda a, b, c, d: (a, b, c, 40, 0, d)),
                        (dp.make_linear_clips, lambda a, b, c, d: (a, b, 1, 4, 4, 1.0, c, d)),
                        (dp.make_layer_grads, lambda a, b, c, d: dp.linear_grad_item(a, b, 1, 4, 4, 1.0, c, d)),
                        (dp.make_ghost_layers, lambda a, b, c, d: (a, b, 1, 4, 4, 1.0, False, c)),
                        (dp.make_layernorm_layers, lambda a, b, c, d: (a, b, 1, 4, 1.0, c, d, None))):
        xs = tensors(4)
        used = {dp.make_grad_tensors: 2, dp.make_ghost_layers: 3}.get(make, 4)
        refs = [weakref.ref(x) for x in xs[:used]]
        items = make([entry(*xs)])
        del xs
        gc.collect()
        assert all(r() is not None for r in refs), make.__name__
        del items
        gc.collect()
        assert all(r() is None for r in refs), make.__name__


def test_a_stream_of_another_gpu_is_refused():
    """The kernels would run there, on addresses of this one."""
    class Fake:                                      # stands for a GPU tensor
        def __init__(self, dtype, n):
            self.dtype, self.n = dtype, n

        def get_device(self):
            return 0

        def is_contiguous(self):
            return True

        def numel(self):
            return self.n

        def data_ptr(self):
            return FAKE

        def element_size(self):
            return 4

    class Stream:
        device_index, cuda_stream = 1, FAKE

    f = lambda n: Fake(torch.float32, n)  # noqa: E731
    with pytest.raises(ValueError, match="stream is on GPU 1, the tensors on GPU 0"):
        dp.dp_embedding_lookup(Fake(torch.int64, 6), f(40), dp.DP_F32, 2, 3, 10, 4, 1.0, f(24), dp.DP_F32, stream=Stream())
    items = dp.make_grad_tensors([(f(40), None, 40, dp.DP_F32)])
    with pytest.raises(ValueError, match="stream is on GPU 1, the tensors on GPU 0"):
        dp.dp_clip_global_norm_many(items, 1, 1.0, FAKE, None, Fake(torch.uint8, 400), stream=Stream())
