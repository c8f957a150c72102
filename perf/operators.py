"""Cases of the language-model operators around the DP-SGD step, on one GPU.

Four operators, five kinds of case: the token embedding's lookup with scaling
(``lookup``) and its clipped gradient by sorted tokens (``tokens``), the gated
feed-forward block's forward (``ffn``) and backward pass (``ffn_grad``), and
the global gradient norm over many tensors with clipping (``clip``).

``listed()`` names representative cases, ``draw(rng)`` draws further ones over
the same ranges, ``prepare(case, seed)`` makes inputs and buffers on the GPU,
``run(state)`` is one pass, ``work(case)`` the bytes and operations a pass
cannot do without, and ``exact(case, seed)`` the same outputs in 64 bits.
With ``own`` set, ``run`` calls the library's entry points
(``paper_2109_12298_amd.binding``); otherwise it computes the same from
elementary torch operations in 32 bits.

Sizes are those of the repository's workloads (the Opacus paper's MNIST and
IMDb networks, a transformer block's batch and width) or generic.
"""
import math

import torch

own = False

SILU, GELU_TANH = "silu", "gelu_tanh"
MNIST = "16x1x8x8,16,32x16x4x4,32,32x512,32,10x32,10"
BLOCK = "768x768,768x768,768x768,768x768,2048x768,2048x768,768x2048,768,768"
DECODER = "32000x1024," + ",".join(["1024x1024,1024x1024,1024x1024,1024x1024,2752x1024,2752x1024,1024x2752,1024,1024"] * 24)
ALIGN = 64            # elements between the starts of two tensors of a flat gradient buffer


def listed():
    return [
        # one token of one sequence, as a decoding step looks it up: launch latency
        dict(name="lookup_token_bf16", kind="lookup", table="bf16", out="bf16", N=1, T=1, V=32000, D=2048, uniform=False),
        # a batch of long sequences from an fp32 master table into bf16 activations, scaled by sqrt(D)
        dict(name="lookup_long_mixed", kind="lookup", table="f32", out="bf16", N=16, T=4096, V=100000, D=4096,
             uniform=False),
        # the text model's embedding at its own batch, clipped per sample
        dict(name="tokens_text_f32", kind="tokens", dtype="f32", N=64, T=256, V=10000, D=100, clip=True, uniform=False),
        # a language model's embedding over a batch of long sequences, with hot tokens
        dict(name="tokens_long_bf16", kind="tokens", dtype="bf16", N=16, T=4096, V=50000, D=2048, clip=True,
             uniform=False),
        # the feed-forward block of one decoded token: the weights are read once
        dict(name="ffn_token_bf16", kind="ffn", dtype="bf16", act=SILU, M=1, d_in=4096, d_ff=11008, save=False),
        # fp32 training on sizes that fit no tile
        dict(name="ffn_ragged_f32", kind="ffn", dtype="f32", act=GELU_TANH, M=1000, d_in=500, d_ff=1333, save=True),
        # a large model's block over a batch of sequences, with what the backward pass needs kept
        dict(name="ffn_large_bf16", kind="ffn", dtype="bf16", act=SILU, M=8192, d_in=4096, d_ff=11008, save=True),
        # the backward pass at the transformer block's batch and width (32 x 128 positions, 768 features)
        dict(name="ffn_grad_block_bf16", kind="ffn_grad", dtype="bf16", act=GELU_TANH, M=4096, d_in=768, d_ff=2048),
        # the large model's backward pass
        dict(name="ffn_grad_large_bf16", kind="ffn_grad", dtype="bf16", act=SILU, M=8192, d_in=4096, d_ff=11008),
        # the MNIST network's eight tensors, 26 010 values: launch latency
        dict(name="clip_mnist_f32", kind="clip", dtype="f32", params=MNIST),
        # a transformer block's gradients in bf16, its norms' gains in fp32
        dict(name="clip_block_mixed", kind="clip", dtype="mixed", params=BLOCK),
        # every tensor of a 24-layer decoder, 217 tensors in fp32 (as noised averages are)
        dict(name="clip_decoder_f32", kind="clip", dtype="f32", params=DECODER),
    ]


# --------------------------------------------------------------------------
# drawn cases
# --------------------------------------------------------------------------

def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _feature(rng, lo, hi):
    """A feature size: mostly a multiple of 64, sometimes of 8, sometimes anything."""
    d, r = _log(rng, lo, hi), rng.random()
    return d if r < 0.2 else max(8, d // 8 * 8) if r < 0.4 else max(64, d // 64 * 64)


def _draw_once(rng):
    kind = rng.choice(["lookup", "tokens", "tokens", "ffn", "ffn", "ffn_grad", "ffn_grad", "clip"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind == "lookup":
        return dict(kind=kind, table=rng.choice(["f32", "bf16"]), out=rng.choice(["bf16", "bf16", "f32"]),
                    N=_log(rng, 1, 64), T=_log(rng, 1, 4096), V=_log(rng, 100, 100000), D=_feature(rng, 16, 4096),
                    uniform=rng.random() < 0.3)
    if kind == "tokens":
        return dict(kind=kind, dtype=dtype, N=_log(rng, 1, 64), T=_log(rng, 1, 4096), V=_log(rng, 50, 100000),
                    D=_feature(rng, 16, 4096), clip=rng.random() < 0.7, uniform=rng.random() < 0.3)
    if kind == "ffn":
        return dict(kind=kind, dtype=dtype, act=rng.choice([SILU, GELU_TANH]), M=_log(rng, 1, 8192),
                    d_in=_feature(rng, 16, 4096), d_ff=_feature(rng, 16, 11008), save=rng.random() < 0.6)
    if kind == "ffn_grad":
        return dict(kind=kind, dtype=dtype, act=rng.choice([SILU, GELU_TANH]), M=_log(rng, 1, 8192),
                    d_in=_feature(rng, 16, 4096), d_ff=_feature(rng, 16, 11008))
    d, ff, n = _feature(rng, 16, 2048), _feature(rng, 16, 4096), _log(rng, 1, 24)
    layer = "%dx%d,%dx%d,%dx%d,%d" % (d, d, ff, d, d, ff, d)
    return dict(kind=kind, dtype=rng.choice(["f32", "bf16", "mixed"]), params=",".join([layer] * n))


def draw(rng):
    """A drawn case moves or computes no more than the largest listed one of its kind."""
    while True:
        case = _draw_once(rng)
        w = work(case)
        top = [work(c) for c in listed() if c["kind"] == case["kind"]]
        if w["bytes"] > max(t["bytes"] for t in top):
            continue
        if w["flops"] * (8 if case.get("dtype") == "f32" else 1) <= max(t["flops"] for t in top):
            return case


# --------------------------------------------------------------------------
# sizes
# --------------------------------------------------------------------------

def _size(dt):
    return 2 if dt == "bf16" else 4


def _expected_distinct(V, M, uniform):
    """Expected distinct ids of M tokens; the skewed ids have P(id) = ln((id + 2) / (id + 1)) / ln(V + 1)."""
    if uniform:
        return V * -math.expm1(M * math.log1p(-1.0 / V)) if V > 1 else 1.0
    total, k, top = 0.0, 0, math.log(V + 1.0)
    while k < V:                                   # runs of ids of about the same probability
        n = min(V - k, max(1, k // 64))
        p = math.log((k + n + 1.0) / (k + 1.0)) / top / n
        total += n * -math.expm1(M * math.log1p(-p)) if p < 1 else n
        k += n
    return total


def _numels(case):
    return [math.prod(int(v) for v in t.split("x")) for t in case["params"].split(",")]


def _tensor_dtypes(case):
    """Per tensor: bf16 or fp32; mixed keeps vectors in fp32."""
    if case["dtype"] != "mixed":
        return [case["dtype"]] * len(case["params"].split(","))
    return ["bf16" if "x" in t else "f32" for t in case["params"].split(",")]


def _layout(case):
    """Per tensor (dtype, first element in that dtype's flat buffer, numel), and the buffers' sizes."""
    at, top = [], {"f32": 0, "bf16": 0}
    for dt, n in zip(_tensor_dtypes(case), _numels(case)):
        at.append((dt, top[dt], n))
        top[dt] += -(-n // ALIGN) * ALIGN
    return at, {dt: n for dt, n in top.items() if n}


def work(case):
    k = case["kind"]
    if k == "lookup":
        M, D = case["N"] * case["T"], case["D"]
        rows = _expected_distinct(case["V"], M, case["uniform"])
        return dict(bytes=8.0 * M + rows * D * _size(case["table"]) + M * D * _size(case["out"]), flops=1.0 * M * D)
    if k == "tokens":
        M, D = case["N"] * case["T"], case["D"]
        return dict(bytes=8.0 * M + 4 * case["N"] + M * D * _size(case["dtype"]) + 4.0 * case["V"] * D, flops=2.0 * M * D)
    if k == "clip":
        n = sum(n * _size(dt) for dt, n in zip(_tensor_dtypes(case), _numels(case)))
        return dict(bytes=2.0 * n + 4, flops=3.0 * sum(_numels(case)))
    M, d, f, e = case["M"], case["d_in"], case["d_ff"], _size(case["dtype"])
    if k == "ffn":
        return dict(bytes=e * (M * d + 2.0 * d * f + M * f * (3 if case["save"] else 1)), flops=4.0 * M * d * f)
    return dict(bytes=e * (5.0 * M * f + 2.0 * d * f + M * d), flops=4.0 * M * d * f)


# --------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------

def _dt(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _normal(g, *shape, dt="f32", scale=1.0):
    """N(0, scale^2), drawn in the type that it is kept in (bf16 draws are rounded once)."""
    return torch.randn(shape, generator=g, device="cuda", dtype=_dt(dt)).mul_(scale)


def _ids(g, case):
    """Token ids: uniform, or skewed as words are (the probability of an id falls with its rank)."""
    u = torch.rand((case["N"], case["T"]), generator=g, device="cuda", dtype=torch.float64)
    V = case["V"]
    x = u * V if case["uniform"] else torch.exp(u * math.log(V + 1.0)) - 1.0
    return x.to(torch.int64).clamp_(0, V - 1)


def _inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    k = case["kind"]
    if k == "lookup":
        return dict(ids=_ids(g, case), E=_normal(g, case["V"], case["D"], dt=case["table"], scale=case["D"] ** -0.5))
    if k == "tokens":
        N = case["N"]
        # backprops of a mean loss whose size differs from sample to sample, and the samples' gradient norms,
        # about half of them over the clipping threshold 1
        B = _normal(g, N, case["T"], case["D"], dt=case["dtype"], scale=1.0 / N)
        return dict(ids=_ids(g, case), B=B, norm=torch.exp(_normal(g, N)) if case["clip"] else None)
    if k == "clip":
        at, top = _layout(case)
        flat = {}
        for dt, n in top.items():
            x = _normal(g, n, dt=dt, scale=0.02)
            keep = torch.zeros(n, dtype=torch.bool, device="cuda")
            for d, first, m in at:
                if d == dt:
                    keep[first:first + m] = True
            flat[dt] = x.mul_(keep)               # the gaps between tensors hold zeros
        return dict(g=flat)
    M, d, f, dt = case["M"], case["d_in"], case["d_ff"], case["dtype"]
    Wg, Wu = _normal(g, f, d, dt=dt, scale=d ** -0.5), _normal(g, f, d, dt=dt, scale=d ** -0.5)
    if k == "ffn":
        return dict(X=_normal(g, M, d, dt=dt), Wg=Wg, Wu=Wu)
    return dict(dH=_normal(g, M, f, dt=dt, scale=1.0 / M), G=_normal(g, M, f, dt=dt), U=_normal(g, M, f, dt=dt),
                Wg=Wg, Wu=Wu)


def prepare(case, seed):
    """The inputs and, as a program that calls the library keeps them, output buffers, workspace and item list."""
    s = dict(_inputs(case, seed), case=case)
    k = case["kind"]
    empty = lambda *shape, dt="f32": torch.empty(shape, device="cuda", dtype=_dt(dt))  # noqa: E731
    if k == "lookup":
        s["Y"] = empty(case["N"], case["T"], case["D"], dt=case["out"])
    elif k == "tokens":
        s["sum"] = empty(case["V"], case["D"])
    elif k == "ffn":
        s["H"], s["G"], s["U"] = [empty(case["M"], case["d_ff"], dt=case["dtype"]) if keep else None
                                  for keep in (True, case["save"], case["save"])]
    elif k == "ffn_grad":
        s["BG"], s["BU"] = [empty(case["M"], case["d_ff"], dt=case["dtype"]) for _ in range(2)]
        s["dX"] = empty(case["M"], case["d_in"], dt=case["dtype"])
    else:
        s["out"] = {dt: torch.zeros_like(x) for dt, x in s["g"].items()}
        s["norm"] = empty(1)
    if own:
        s.update(_plan(case, s))
    return s


def _plan(case, s):
    from paper_2109_12298_amd import binding as dp
    k = case["kind"]
    plan = dict(dp=dp, status=torch.zeros(1, dtype=torch.int32, device="cuda"))
    code = {"f32": dp.DP_F32, "bf16": dp.DP_BF16}
    need = 0
    if k == "lookup":
        plan.update(dt=code[case["table"]], dt_y=code[case["out"]])
    elif k == "tokens":
        plan["dt"] = code[case["dtype"]]
        need = dp.dp_clip_accumulate_tokens_workspace_bytes(case["N"], case["T"], case["V"], case["D"], plan["dt"])
    elif k == "clip":
        at, _ = _layout(case)
        plan["items"] = dp.make_grad_tensors([(s["g"][dt][first:], s["out"][dt][first:], n, code[dt])
                                              for dt, first, n in at])
        plan["count"] = len(at)
        need = dp.dp_clip_global_norm_many_workspace_bytes(plan["items"], plan["count"])
    else:
        plan.update(dt=code[case["dtype"]], act=dp.DP_ACT_SILU if case["act"] == SILU else dp.DP_ACT_GELU_TANH)
        size = dp.dp_gated_ffn_forward_workspace_bytes if k == "ffn" else dp.dp_gated_ffn_backward_workspace_bytes
        need = size(case["M"], case["d_in"], case["d_ff"], plan["dt"])
    plan["ws"] = torch.empty(max(int(need), 256), dtype=torch.uint8, device="cuda")
    return plan


# --------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------

def _scale(case):
    """Embeddings scaled by sqrt(D)."""
    return math.sqrt(case["D"])


def run(s):
    return _run_own(s) if own else PLAIN[s["case"]["kind"]](s["case"], s)


def _run_own(s):
    c, dp = s["case"], s["dp"]
    k = c["kind"]
    if k == "lookup":
        dp.dp_embedding_lookup(s["ids"], s["E"], s["dt"], c["N"], c["T"], c["V"], c["D"], _scale(c), s["Y"], s["dt_y"],
                               s["status"])
        return s["Y"]
    if k == "tokens":
        dp.dp_clip_accumulate_tokens(s["ids"], s["B"], s["dt"], c["N"], c["T"], c["V"], c["D"], _scale(c), s["norm"], 1.0,
                                     s["sum"], s["status"], s["ws"])
        return s["sum"]
    if k == "ffn":
        dp.dp_gated_ffn_forward(s["X"], s["Wg"], s["Wu"], s["dt"], c["M"], c["d_in"], c["d_ff"], s["act"], s["H"],
                                s["G"], s["U"], s["ws"])
        return dict(H=s["H"], G=s["G"], U=s["U"])
    if k == "ffn_grad":
        dp.dp_gated_ffn_backward(s["dH"], s["G"], s["U"], s["Wg"], s["Wu"], s["dt"], c["M"], c["d_in"], c["d_ff"],
                                 s["act"], s["BG"], s["BU"], s["dX"], s["ws"])
        return dict(BG=s["BG"], BU=s["BU"], dX=s["dX"])
    dp.dp_clip_global_norm_many(s["items"], s["count"], 1.0, s["norm"], s["status"], s["ws"])
    return dict(norm=s["norm"], grads=s["out"])


def _plain_lookup(c, s):
    return (s["E"][s["ids"]].float() * _scale(c)).to(_dt(c["out"]))


def _plain_tokens(c, s):
    B = s["B"].float()
    if c["clip"]:
        B = B * (1.0 / (s["norm"] + 1e-6)).clamp(max=1.0)[:, None, None]
    out = torch.zeros((c["V"], c["D"]), device="cuda")
    return out.index_add_(0, s["ids"].reshape(-1), B.reshape(-1, c["D"])).mul_(_scale(c))


def _act(c, g):
    if c["act"] == SILU:
        return g * torch.sigmoid(g)
    return 0.5 * g * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (g + 0.044715 * g * g * g)))


def _act_slope(c, g):
    if c["act"] == SILU:
        p = torch.sigmoid(g)
        return p * (1.0 + g * (1.0 - p))
    k = math.sqrt(2.0 / math.pi)
    t = torch.tanh(k * (g + 0.044715 * g * g * g))
    return 0.5 * (1.0 + t) + 0.5 * g * (1.0 - t * t) * k * (1.0 + 3 * 0.044715 * g * g)


def _plain_ffn(c, s):
    X, dt = s["X"].float(), _dt(c["dtype"])
    g, u = X @ s["Wg"].float().t(), X @ s["Wu"].float().t()
    H = (_act(c, g) * u).to(dt)
    return dict(H=H, G=g.to(dt) if c["save"] else None, U=u.to(dt) if c["save"] else None)


def _plain_ffn_grad(c, s):
    dt = _dt(c["dtype"])
    dH, g, u = s["dH"].float(), s["G"].float(), s["U"].float()
    BG, BU = (dH * u * _act_slope(c, g)).to(dt), (dH * _act(c, g)).to(dt)
    # dX is the gradient of the two backprops as they are stored
    dX = BG.float() @ s["Wg"].float() + BU.float() @ s["Wu"].float()
    return dict(BG=BG, BU=BU, dX=dX.to(dt))


def _plain_clip(c, s):
    flat = s["g"]
    norm = torch.stack([x.float().square().sum() for x in flat.values()]).sum().sqrt().reshape(1)
    f = (1.0 / (norm + 1e-6)).clamp(max=1.0)
    return dict(norm=norm, grads={dt: (x.float() * f).to(x.dtype) for dt, x in flat.items()})


PLAIN = dict(lookup=_plain_lookup, tokens=_plain_tokens, ffn=_plain_ffn, ffn_grad=_plain_ffn_grad, clip=_plain_clip)


# --------------------------------------------------------------------------
# the same outputs in 64 bits
# --------------------------------------------------------------------------

def exact(case, seed):
    s, k = _inputs(case, seed), case["kind"]
    if k == "lookup":
        return torch.index_select(s["E"], 0, s["ids"].reshape(-1)).double().mul_(_scale(case)).reshape(
            case["N"], case["T"], case["D"])
    if k == "tokens":
        # tokens sorted by id; each id's sum is the difference of two running sums
        order = torch.sort(s["ids"].reshape(-1), stable=True).indices
        rows = s["B"].reshape(-1, case["D"])[order].double()
        if case["clip"]:
            f = torch.minimum(torch.ones(()).double().cuda(), 1.0 / (s["norm"].double() + 1e-6))
            rows.mul_(f[order // case["T"]][:, None])
        run_ = torch.cat([torch.zeros((1, case["D"]), dtype=torch.float64, device="cuda"), rows.cumsum(0)])
        ends = torch.bincount(s["ids"].reshape(-1), minlength=case["V"]).cumsum(0)
        starts = torch.cat([ends.new_zeros(1), ends[:-1]])
        return (run_[ends] - run_[starts]) * _scale(case)
    if k == "clip":
        n2 = sum(float(torch.dot(x.double(), x.double())) for x in s["g"].values())
        f = min(1.0, 1.0 / (math.sqrt(n2) + 1e-6))
        return dict(norm=torch.full((1,), math.sqrt(n2), dtype=torch.float64),
                    grads={dt: x.double() * f for dt, x in s["g"].items()})
    c = math.sqrt(2.0 / math.pi)
    if k == "ffn":
        X = s["X"].double()
        g, u = torch.mm(X, s["Wg"].double().t()), torch.mm(X, s["Wu"].double().t())
        gate = 1.0 / (1.0 + torch.exp(-g)) if case["act"] == SILU else 1.0 / (1.0 + torch.exp(-2 * c * (g + 0.044715 * g ** 3)))
        return dict(H=g * gate * u, G=g if case["save"] else None, U=u if case["save"] else None)
    g, u, dH = s["G"].double(), s["U"].double(), s["dH"].double()
    if case["act"] == SILU:
        gate = 1.0 / (1.0 + torch.exp(-g))
        slope = gate + g * gate * (1.0 - gate)
    else:                                  # (1 + tanh z) / 2 = sigmoid(2 z)
        gate = 1.0 / (1.0 + torch.exp(-2 * c * (g + 0.044715 * g ** 3)))
        slope = gate + g * gate * (1.0 - gate) * 2 * c * (1.0 + 3 * 0.044715 * g ** 2)
    BG, BU = dH * u * slope, dH * g * gate
    stored = _dt(case["dtype"])
    dX = torch.mm(BG.to(stored).double(), s["Wg"].double()) + torch.mm(BU.to(stored).double(), s["Wu"].double())
    return dict(BG=BG, BU=BU, dX=dX)
