"""Cases of a token model's operators between its weight layers, on one GPU.

Three operators, four kinds of case: rotary positions over one or several axes
(``rotary``), attention forward (``attention``: prompts and single tokens) and
as a training step does it, forward and backward (``train``), and the loss that
distils a teacher's top logits, with its gradient (``distill``).

``listed()`` names representative cases, ``draw(rng)`` draws further ones over
the same ranges, ``prepare(case, seed)`` makes inputs and buffers on the GPU,
``run(state)`` is one pass, ``work(case)`` the bytes and operations a pass
cannot do without, and ``exact(case, seed)`` the same outputs in 64 bits.
With ``own`` set, ``run`` calls the library's entry points
(``paper_2109_12298_amd.binding``); otherwise it computes the same from
elementary torch operations in 32 bits.

Sizes are those of the repository's workloads (a transformer block's batch and
width, the text model's vocabulary and length) or generic.
"""
import math

import torch

own = False

ADJACENT_BELOW = 64       # heads narrower than this pair adjacent values, wider ones their halves


def _attn(name, kind, dtype, N, Tq, Tk, Hq, Hk, D, causal=True, last=False, ragged=False, docs=0, prefix=False,
          softcap=0.0, slopes=False):
    """ragged: samples of different lengths; docs: documents packed in a sample; prefix: the first keys are seen by all."""
    return dict(name=name, kind=kind, dtype=dtype, N=N, Tq=Tq, Tk=Tk, Hq=Hq, Hk=Hk, D=D, causal=causal, last=last,
                ragged=ragged, docs=docs, prefix=prefix, softcap=softcap, slopes=slopes)


def listed():
    return [
        # queries and keys of one decoded token: launch latency
        dict(name="rotary_token_bf16", kind="rotary", dtype="bf16", N=1, T=1, H=40, Hv=8, D=128, R=128, axes=1, inverse=False),
        # a batch of video tokens (time, height, width), rotated out of the fused projection's output
        dict(name="rotary_video_bf16", kind="rotary", dtype="bf16", N=4, T=4096, H=40, Hv=8, D=128, R=128, axes=3, inverse=False),
        # one new token over a cache of 4096
        _attn("attn_token_bf16", "attention", "bf16", 1, 1, 4096, 32, 8, 128, last=True),
        # a batch of decoded tokens whose caches differ in length, with capped scores
        _attn("attn_decode_ragged_bf16", "attention", "bf16", 32, 1, 8192, 32, 8, 128, last=True, ragged=True, softcap=30.0),
        # two prompts
        _attn("attn_prompt_bf16", "attention", "bf16", 2, 4096, 4096, 32, 8, 128),
        # fp32, sizes that fit no tile, a padded batch, prefixes that all positions see, a bias by distance
        _attn("attn_prefix_ragged_f32", "attention", "f32", 3, 777, 777, 10, 5, 80, ragged=True, prefix=True, slopes=True),
        # the transformer block at its own batch, length and width: an encoder's attention over padded samples
        _attn("train_block_bf16", "train", "bf16", 32, 128, 128, 12, 12, 64, causal=False, ragged=True),
        # fp32 training on odd sizes with shared heads
        _attn("train_odd_f32", "train", "f32", 3, 500, 500, 6, 2, 48, prefix=True, slopes=True),
        # long samples, each packed of four documents, with capped scores and shared heads
        _attn("train_docs_bf16", "train", "bf16", 2, 8192, 8192, 32, 8, 128, docs=4, softcap=50.0),
        # one sample of the text model's length over its vocabulary
        dict(name="distill_text_f32", kind="distill", dtype="f32", M=256, V=10000, K=16, labels=False, ragged=False, tau=1.0),
        # odd sizes, labels mixed in, teachers that keep fewer logits at some positions
        dict(name="distill_mixed_bf16", kind="distill", dtype="bf16", M=1001, V=32001, K=20, labels=True, ragged=True, tau=1.5),
        # a batch of long sequences over a large vocabulary
        dict(name="distill_large_bf16", kind="distill", dtype="bf16", M=8192, V=100000, K=64, labels=False, ragged=False, tau=2.0),
    ]


# --------------------------------------------------------------------------
# drawn cases
# --------------------------------------------------------------------------

def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _head(rng, lo, hi):
    """Values of a head: mostly 64 or 128, sometimes a multiple of 8, sometimes anything even."""
    r = rng.random()
    if r < 0.5:
        return rng.choice([64, 128])
    d = rng.randint(lo, hi)
    return max(8, d // 8 * 8) if r < 0.8 else max(2, d // 2 * 2)


def _draw_once(rng):
    kind = rng.choice(["rotary", "attention", "attention", "attention", "train", "train", "train", "distill", "distill"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind == "rotary":
        D, axes = _head(rng, 16, 128), rng.choice([1, 1, 2, 3])
        R = D if rng.random() < 0.7 or D < 32 else D // 4 * 2
        return dict(kind=kind, dtype=dtype, N=_log(rng, 1, 16), T=_log(rng, 1, 4096), H=rng.randint(1, 40),
                    Hv=rng.choice([0, 0, 1, 8]), D=D, R=R, axes=axes, inverse=rng.random() < 0.4)
    if kind == "distill":
        V = _log(rng, 100, 100000)
        return dict(kind=kind, dtype=dtype, M=_log(rng, 1, 8192), V=V, K=min(V, _log(rng, 1, 64)), labels=rng.random() < 0.5,
                    ragged=rng.random() < 0.5, tau=rng.choice([1.0, 1.0, 1.5, 2.0, 4.0]))
    Hk, group, D = rng.choice([1, 2, 5, 8, 12]), rng.choice([1, 1, 2, 4]), _head(rng, 16, 128)
    pick = lambda p: rng.random() < p  # noqa: E731
    if kind == "train":
        T = _log(rng, 1, 8192)
        c = _attn("", kind, dtype, _log(rng, 1, 32), T, T, Hk * group, Hk, D)
        c.update(causal=pick(0.7), docs=rng.randint(2, 5) if T >= 16 and pick(0.3) else 0)
    elif pick(0.5):                                   # a prompt
        T = _log(rng, 1, 4096)
        c = _attn("", kind, dtype, _log(rng, 1, 8), T, T, Hk * group, Hk, D)
        c.update(causal=pick(0.8), docs=rng.randint(2, 5) if T >= 16 and pick(0.3) else 0)
    else:                                             # one or a few new tokens over a cache
        Tq = rng.choice([1, 1, 1, 2, 5])
        c = _attn("", kind, dtype, _log(rng, 1, 32), Tq, _log(rng, 16, 8192), Hk * group, Hk, D, last=True)
    c.update(ragged=pick(0.4), prefix=c["causal"] and not (c["last"] or c["docs"]) and pick(0.3),
             softcap=rng.choice([0.0, 0.0, 30.0, 50.0]), slopes=pick(0.25))
    del c["name"]
    return c


def draw(rng):
    """A drawn case moves or computes no more than the largest listed one of its kind."""
    while True:
        case = _draw_once(rng)
        w = work(case)
        top = [work(c) for c in listed() if c["kind"] == case["kind"]]
        if w["bytes"] > max(t["bytes"] for t in top):
            continue
        if w["flops"] * (8 if case["dtype"] == "f32" else 1) <= max(t["flops"] for t in top):
            return case


# --------------------------------------------------------------------------
# sizes
# --------------------------------------------------------------------------

def _lengths(case):
    """Keys of each sample (in an order that prepare shuffles): from about an eighth of Tk to all of it."""
    N, T = case["N"], case["Tk"]
    if not case["ragged"]:
        return [T] * N
    return [max(1, T // 8 + (T - T // 8) * (n + 1) // N) for n in range(N)]


def _doc_lengths(case, length):
    """Lengths of a sample's documents, unequal: 1 : 2 : ... parts of the sample."""
    k = case["docs"]
    ends = [length * (i + 1) * (i + 2) // (k * (k + 1)) for i in range(k)]
    return [b - a for a, b in zip([0] + ends[:-1], ends)]


def _prefix_length(case, length):
    return length // 3


def _pairs(case):
    """Visible pairs of a query and a key of all samples."""
    total = 0
    for L in _lengths(case):
        queries = min(case["Tq"], L)
        if not case["causal"]:
            total += sum(d * d for d in _doc_lengths(case, L)) if case["docs"] else queries * L
        elif case["last"]:
            total += queries * L - queries * (queries - 1) // 2
        else:
            for d in _doc_lengths(case, L) if case["docs"] else [L]:
                total += d * (d + 1) // 2
            if case["prefix"] and not case["docs"]:
                p = _prefix_length(case, L)
                total += p * (p - 1) // 2
    return total


def _size(dt):
    return 2 if dt == "bf16" else 4


def work(case):
    k, e = case["kind"], _size(case["dtype"])
    if k == "rotary":
        M = case["N"] * case["T"]
        return dict(bytes=8.0 * M * case["axes"] + 2.0 * e * M * case["H"] * case["D"], flops=3.0 * M * case["H"] * case["R"])
    if k == "distill":
        M, V, K = case["M"], case["V"], case["K"]
        return dict(bytes=2.0 * e * M * V + 12.0 * M * K + M * (16.0 if case["labels"] else 8.0), flops=6.0 * M * V)
    keys, q = sum(_lengths(case)), case["N"] * case["Tq"]
    D, Hq, Hk = case["D"], case["Hq"], case["Hk"]
    if k == "attention":
        return dict(bytes=e * D * (2.0 * Hk * keys + 2.0 * Hq * q), flops=4.0 * D * Hq * _pairs(case))
    return dict(bytes=e * D * (4.0 * Hk * keys + 4.0 * Hq * q), flops=14.0 * D * Hq * _pairs(case))


# --------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------

def _dt(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _normal(g, *shape, dt="f32", scale=1.0):
    """N(0, scale^2), drawn in the type that it is kept in (bf16 draws are rounded once)."""
    return torch.randn(shape, generator=g, device="cuda", dtype=_dt(dt)).mul_(scale)


def _sections(case):
    """Pairs of each axis: one axis has all; of three, time has a quarter, height and width share the rest."""
    P = case["R"] // 2
    if case["axes"] == 1:
        return [P]
    if case["axes"] == 2:
        return [P // 2, P - P // 2]
    return [P // 4, (P - P // 4) // 2, P - P // 4 - (P - P // 4) // 2]


def _positions(g, case):
    """[axes][N][T]: consecutive from a far start; with several axes a grid that its last axis runs through first."""
    N, T, axes = case["N"], case["T"], case["axes"]
    i = torch.arange(T, device="cuda").expand(N, T)
    start = torch.randint(0, 1 << 20, (N, 1), generator=g, device="cuda")
    if axes == 1:
        return (i + start)[None].contiguous()
    w = max(1, int(round(T ** (1.0 / axes))))
    grid = [i // w ** (axes - 1) + start] + [i // w ** k % w for k in range(axes - 2, -1, -1)]
    return torch.stack(grid).contiguous()


def _softmax_scale(case):
    return case["D"] ** -0.5


def _inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    k, dt = case["kind"], case["dtype"]
    if k == "rotary":
        P = case["R"] // 2
        freq = 10000.0 ** (-torch.arange(P, dtype=torch.float64, device="cuda") / max(P, 1))
        X = _normal(g, case["N"], case["T"], (case["H"] + case["Hv"]) * case["D"], dt=dt)
        return dict(X=X, pos=_positions(g, case), freq=freq)
    if k == "distill":
        M, V, K = case["M"], case["V"], case["K"]
        Z = _normal(g, M, V, dt=dt, scale=2.0)
        # K different ids a row; the teacher's logits fall from its best on
        u = torch.rand((2, M, 1), generator=g, device="cuda", dtype=torch.float64)
        step = 1 + (u[1] * (V // K)).to(torch.int64).clamp_(max=max(V // K - 1, 0))
        at = torch.arange(K, device="cuda")
        ids = ((u[0] * V).to(torch.int64) + at * step) % V
        top = 9.0 + _normal(g, M, 1) - torch.cumsum(-torch.log1p(-torch.rand((M, K), generator=g, device="cuda")) * 0.5, 1)
        if case["ragged"]:                            # the teacher kept 1 to K
            kept = torch.randint(1, K + 1, (M, 1), generator=g, device="cuda")
            ids = torch.where(at < kept, ids, -1)
        labels = None
        if case["labels"]:                            # a tenth of the positions has none
            labels = torch.randint(0, V, (M,), generator=g, device="cuda")
            labels[torch.rand(M, generator=g, device="cuda") < 0.1] = -1
        weight = torch.rand(M, generator=g, device="cuda") + 0.5
        return dict(Z=Z, ids=ids.contiguous(), top=top.contiguous(), labels=labels, weight=weight)
    N, Tq, Tk, Hq, Hk, D = [case[x] for x in ("N", "Tq", "Tk", "Hq", "Hk", "D")]
    s = {}
    if k == "train":
        s["qkv"] = _normal(g, N, Tq, (Hq + 2 * Hk) * D, dt=dt)     # the fused projection's output
        s["Q"], s["K"], s["V"] = s["qkv"].split([Hq * D, Hk * D, Hk * D], dim=2)
        s["dO"] = _normal(g, N, Tq, Hq * D, dt=dt, scale=1.0 / Tq)
    else:
        s["Q"], s["K"], s["V"] = [_normal(g, N, T, H * D, dt=dt) for T, H in ((Tq, Hq), (Tk, Hk), (Tk, Hk))]
    order = torch.randperm(N, generator=g, device="cuda").tolist()
    lengths = [_lengths(case)[n] for n in order]
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    s["lens"] = ints(lengths) if case["ragged"] else None
    s["prefix"] = ints([_prefix_length(case, L) for L in lengths]) if case["prefix"] else None
    s["docs"] = None
    if case["docs"]:
        rows = []
        for L in lengths:
            parts = _doc_lengths(case, L)
            turn = torch.randperm(len(parts), generator=g, device="cuda").tolist()
            row = [d for d, j in enumerate(turn) for _ in range(parts[j])]
            rows.append(row + [-1] * (Tk - L))
        s["docs"] = ints(rows)
    s["slopes"] = torch.pow(2.0, -8.0 * torch.arange(1, Hq + 1, device="cuda") / Hq) if case["slopes"] else None
    return s


def prepare(case, seed):
    """The inputs and, as a program that calls the library keeps them, output buffers, workspace and call description."""
    s = dict(_inputs(case, seed), case=case)
    k, dt = case["kind"], _dt(case["dtype"])
    if k == "rotary":
        s["Y"] = torch.empty((case["N"], case["T"], case["H"] * case["D"]), device="cuda", dtype=dt)
    elif k == "distill":
        s["loss"], s["dZ"] = torch.empty(case["M"], device="cuda"), torch.empty_like(s["Z"])
    else:
        s["O"] = torch.empty((case["N"], case["Tq"], case["Hq"] * case["D"]), device="cuda", dtype=dt)
        if k == "train":
            D, Hq, Hk = case["D"], case["Hq"], case["Hk"]
            s["lse"] = torch.empty((case["N"], Hq, case["Tq"]), device="cuda")
            s["dqkv"] = torch.empty_like(s["qkv"])
            s["dQ"], s["dK"], s["dV"] = s["dqkv"].split([Hq * D, Hk * D, Hk * D], dim=2)
    if own:
        s.update(_plan(case, s))
    return s


def _plan(case, s):
    from paper_2109_12298_amd import binding as dp
    k = case["kind"]
    plan = dict(dp=dp, dt=dp.DP_F32 if case["dtype"] == "f32" else dp.DP_BF16,
                status=torch.zeros(1, dtype=torch.int32, device="cuda"))
    need = 0
    if k == "rotary":
        plan["layout"] = dp.DP_ROTARY_ADJACENT if case["D"] < ADJACENT_BELOW else dp.DP_ROTARY_HALVES
    elif k == "distill":
        need = dp.dp_distill_loss_workspace_bytes(case["M"], case["V"], case["K"], plan["dt"])
    else:
        flags = (dp.DP_ATTENTION_CAUSAL if case["causal"] else 0) | (dp.DP_ATTENTION_LAST if case["last"] else 0)
        ld = dict(ldq=s["Q"].stride(1), ldk=s["K"].stride(1), ldv=s["V"].stride(1))
        plan["a"] = dp.make_attention(plan["dt"], *[case[x] for x in ("N", "Tq", "Tk", "Hq", "Hk", "D")],
                                      scale=_softmax_scale(case), flags=flags, softcap=case["softcap"], slopes=s["slopes"],
                                      lens=s["lens"], prefix=s["prefix"], docs=s["docs"], **ld)
        need = dp.dp_attention_forward_workspace_bytes(plan["a"])
        if k == "train":
            need = max(need, dp.dp_attention_backward_workspace_bytes(plan["a"]))
    plan["ws"] = torch.empty(max(int(need), 256), dtype=torch.uint8, device="cuda")
    return plan


# --------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------

ALPHA = 0.7               # the teacher's share of a loss with labels


def run(s):
    return _run_own(s) if own else PLAIN[s["case"]["kind"]](s["case"], s)


def _run_own(s):
    c, dp = s["case"], s["dp"]
    k = c["kind"]
    if k == "rotary":
        dp.dp_rotary(s["X"], s["dt"], c["N"], c["T"], c["H"], c["D"], s["X"].stride(1), s["pos"], _sections(c), s["freq"],
                     s["layout"], c["inverse"], s["Y"], c["H"] * c["D"])
        return s["Y"]
    if k == "distill":
        dp.dp_distill_loss(s["Z"], s["dt"], c["M"], c["V"], s["ids"], s["top"], c["K"], s["labels"],
                           ALPHA if c["labels"] else 1.0, c["tau"], s["weight"], s["loss"], s["dZ"], s["status"], s["ws"])
        return dict(loss=s["loss"], dZ=s["dZ"])
    if k == "attention":
        dp.dp_attention_forward(s["a"], s["Q"], s["K"], s["V"], s["O"], None, s["ws"])
        return s["O"]
    dp.dp_attention_forward(s["a"], s["Q"], s["K"], s["V"], s["O"], s["lse"], s["ws"])
    dp.dp_attention_backward(s["a"], s["Q"], s["K"], s["V"], s["O"], s["lse"], s["dO"], s["dQ"], s["dK"], s["dV"], s["ws"])
    return dict(O=s["O"], dqkv=s["dqkv"])


def _plain_rotary(c, s):
    D, R, P = c["D"], c["R"], c["R"] // 2
    x = s["X"][..., :c["H"] * D].reshape(c["N"], c["T"], c["H"], D).float()
    # angles of far positions in 64 bits; axis of each pair by its section
    axis = torch.repeat_interleave(torch.arange(c["axes"], device="cuda"), torch.tensor(_sections(c), device="cuda"))
    turn = s["pos"][axis].permute(1, 2, 0).double() * s["freq"]
    cos, sin = torch.cos(turn).float()[:, :, None], torch.sin(turn).float()[:, :, None]
    if c["inverse"]:
        sin = -sin
    if D < ADJACENT_BELOW:
        a, b = x[..., 0:R:2], x[..., 1:R:2]
        y = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
    else:
        a, b = x[..., :P], x[..., P:R]
        y = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
    return torch.cat([y, x[..., R:]], dim=-1).reshape(c["N"], c["T"], c["H"] * D).to(_dt(c["dtype"]))


def _plain_distill(c, s):
    z, tau, w = s["Z"].float(), c["tau"], s["weight"][:, None]
    alpha = ALPHA if c["labels"] else 1.0
    used = s["ids"] >= 0
    ids = s["ids"].clamp(min=0)
    t = (s["top"] / tau).masked_fill(~used, -math.inf)
    e = torch.exp(t - t.amax(1, keepdim=True))
    p = e / e.sum(1, keepdim=True)
    zt = z / tau
    top = zt.amax(1, keepdim=True)
    q = torch.exp(zt - top)
    total = q.sum(1, keepdim=True)
    logq = torch.gather(zt, 1, ids) - top - torch.log(total)
    loss = alpha * tau * tau * torch.where(p > 0, p * (torch.log(p) - logq), torch.zeros_like(p)).sum(1, keepdim=True)
    d = q.div_(total).mul_(alpha * tau).scatter_add_(1, ids, -alpha * tau * p)
    if c["labels"]:
        has, label = (s["labels"] >= 0)[:, None], s["labels"].clamp(min=0)[:, None]
        top = z.amax(1, keepdim=True)
        q = torch.exp(z - top)
        total = q.sum(1, keepdim=True)
        hard = -(torch.gather(z, 1, label) - top - torch.log(total))
        share = (1.0 - alpha) * has
        loss = loss + torch.where(has, share * hard, torch.zeros_like(hard))
        d = d.add_(q.div_(total).mul_(share)).scatter_add_(1, label, -share)
    return dict(loss=(loss * w).reshape(-1), dZ=d.mul_(w).to(_dt(c["dtype"])))


def _visible(c, s, n):
    """[len(n)][Tq][Tk]: which keys the queries of samples n (a slice) see; and the distances between them."""
    Tq, Tk = c["Tq"], c["Tk"]
    count = len(range(c["N"])[n])
    lens = s["lens"][n].long() if s["lens"] is not None else torch.full((count,), Tk, device="cuda")
    j = torch.arange(Tk, device="cuda")[None, None]
    i = torch.arange(Tq, device="cuda")[None, :, None] + (lens - Tq if c["last"] else torch.zeros_like(lens))[:, None, None]
    inside = (i >= 0) & (i < lens[:, None, None])
    see = (j < lens[:, None, None]) & inside
    if c["causal"]:
        seen = j <= i
        if s["prefix"] is not None:
            seen = seen | (j < s["prefix"][n].long()[:, None, None])
        see = see & seen
    if s["docs"] is not None:
        docs = s["docs"][n]
        of_query = torch.gather(docs, 1, i.squeeze(2).clamp(0, Tk - 1).expand(count, Tq))
        see = see & (of_query[:, :, None] == docs[:, None, :]) & (of_query >= 0)[:, :, None]
    return see, (i - j).abs()


def _plain_attention(c, s):
    N, Tq, Tk, Hq, Hk, D = [c[x] for x in ("N", "Tq", "Tk", "Hq", "Hk", "D")]
    G, cap, dt, scale = Hq // Hk, c["softcap"], _dt(c["dtype"]), _softmax_scale(c)
    step = max(1, min(N, (1 << 31) // max(1, Hq * Tq * Tk)))
    outs = []
    for n0 in range(0, N, step):
        n = slice(n0, min(N, n0 + step))
        m = n.stop - n0
        heads = lambda x, T, H: x[n].float().reshape(m, T, H, D).transpose(1, 2).contiguous()  # noqa: E731
        q = heads(s["Q"], Tq, Hq).reshape(m, Hk, G * Tq, D)
        k, v = heads(s["K"], Tk, Hk), heads(s["V"], Tk, Hk)
        see, far = _visible(c, s, n)
        shape = (m, Hk, G, Tq, Tk)
        x = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(scale).reshape(shape)
        bend = None
        if cap > 0:
            bend = torch.tanh(x / cap)
            x = bend * cap
        if s["slopes"] is not None:
            x = x - s["slopes"].reshape(1, Hk, G, 1, 1) * far[:, None, None].float()
        x = x.masked_fill(~see[:, None, None], -math.inf)
        top = x.amax(-1, keepdim=True)
        p = torch.exp(x - torch.where(torch.isinf(top), torch.zeros_like(top), top))
        del x
        total = p.sum(-1, keepdim=True)
        p = p / torch.where(total > 0, total, torch.ones_like(total))
        flat = (m, Hk, G * Tq, Tk)
        o = torch.matmul(p.reshape(flat), v)
        back = lambda y, T, H: y.reshape(m, H, T, D).transpose(1, 2).reshape(m, T, H * D).to(dt)  # noqa: E731
        if c["kind"] == "attention":
            outs.append((back(o, Tq, Hq),))
            continue
        do = heads(s["dO"], Tq, Hq).reshape(m, Hk, G * Tq, D)
        dv = torch.matmul(p.reshape(flat).transpose(2, 3).contiguous(), do)
        dp = torch.matmul(do, v.transpose(2, 3).contiguous()).reshape(shape)
        ds = p * (dp - (do * o).sum(-1).reshape(m, Hk, G, Tq, 1))
        del dp, p
        if cap > 0:
            ds = ds * (1.0 - bend * bend)
        ds = ds.mul_(scale).reshape(flat)
        dq = torch.matmul(ds, k)
        dk = torch.matmul(ds.transpose(2, 3).contiguous(), q)
        outs.append((back(o, Tq, Hq), torch.cat([back(dq, Tq, Hq), back(dk, Tk, Hk), back(dv, Tk, Hk)], dim=2)))
    outs = [torch.cat(x) if len(x) > 1 else x[0] for x in zip(*outs)]
    return outs[0] if c["kind"] == "attention" else dict(O=outs[0], dqkv=outs[1])


PLAIN = dict(rotary=_plain_rotary, distill=_plain_distill, attention=_plain_attention, train=_plain_attention)


# --------------------------------------------------------------------------
# the same outputs in 64 bits
# --------------------------------------------------------------------------

def exact(case, seed):
    s, k = _inputs(case, seed), case["kind"]
    if k == "rotary":
        # a rotation is a product of complex numbers
        D, R = case["D"], case["R"]
        x = s["X"][..., :case["H"] * D].double().reshape(case["N"], case["T"], case["H"], D)
        first, ang = 0, []
        for a, m in enumerate(_sections(case)):
            ang.append(s["pos"][a][..., None] * s["freq"][first:first + m])
            first += m
        ang = torch.cat(ang, dim=-1)[:, :, None]
        turn = torch.polar(torch.ones_like(ang), -ang if case["inverse"] else ang)
        out = x.clone()
        at = (slice(0, R, 2), slice(1, R, 2)) if D < ADJACENT_BELOW else (slice(0, R // 2), slice(R // 2, R))
        y = torch.complex(x[..., at[0]], x[..., at[1]]) * turn
        out[..., at[0]], out[..., at[1]] = y.real, y.imag
        return out.reshape(case["N"], case["T"], -1)
    if k == "distill":
        tau, alpha = case["tau"], ALPHA if case["labels"] else 1.0
        loss = torch.empty(case["M"], dtype=torch.float64, device="cuda")
        dZ = torch.empty_like(s["Z"], dtype=torch.float64)
        for m0 in range(0, case["M"], 1024):          # by autograd of the definition, some positions at a time
            m = slice(m0, m0 + 1024)
            z = s["Z"][m].double().requires_grad_(True)
            used = s["ids"][m] >= 0
            logp = torch.log_softmax((s["top"][m].double() / tau).masked_fill(~used, -1e300), 1)
            logq = torch.log_softmax(z / tau, 1).gather(1, s["ids"][m].clamp(min=0))
            part = torch.where(used, logp.exp() * (logp - logq), 0.0).sum(1) * (alpha * tau * tau)
            if case["labels"]:
                has = s["labels"][m] >= 0
                hard = -torch.log_softmax(z, 1).gather(1, s["labels"][m].clamp(min=0)[:, None])[:, 0]
                part = part + torch.where(has, (1.0 - alpha) * hard, 0.0)
            part = part * s["weight"][m].double()
            dZ[m] = torch.autograd.grad(part.sum(), z)[0]
            loss[m] = part.detach()
        return dict(loss=loss, dZ=dZ)
    N, Tq, Tk, Hq, Hk, D = [case[x] for x in ("N", "Tq", "Tk", "Hq", "Hk", "D")]
    train, cap = k == "train", case["softcap"]
    new = lambda T, H: torch.zeros((N, T, H, D), dtype=torch.float64, device="cuda")  # noqa: E731
    O, dq, dk, dv = new(Tq, Hq), new(Tq, Hq), new(Tk, Hk), new(Tk, Hk)
    for n in range(N):
        L = int(s["lens"][n]) if s["lens"] is not None else Tk
        first = L - Tq if case["last"] else 0
        lo, hi = max(0, -first), min(Tq, L - first)   # this sample's queries
        if hi <= lo:
            continue
        i = torch.arange(first + lo, first + hi, device="cuda")[:, None]
        j = torch.arange(L, device="cuda")[None, :]
        hide = torch.zeros((hi - lo, L), dtype=torch.bool, device="cuda")
        if case["causal"]:
            hide |= j > torch.maximum(i, (s["prefix"][n] - 1).long()) if s["prefix"] is not None else j > i
        if s["docs"] is not None:
            hide |= s["docs"][n][i] != s["docs"][n][j]
        for h in range(Hq):
            kv = h * Hk // Hq
            cut = lambda x, a, b, g: x[n, a:b, g * D:(g + 1) * D].double()  # noqa: E731
            leaves = [cut(s["Q"], lo, hi, h), cut(s["K"], 0, L, kv), cut(s["V"], 0, L, kv)]
            if train:
                leaves = [x.requires_grad_(True) for x in leaves]
            x = (leaves[0] @ leaves[1].t()) * _softmax_scale(case)
            if cap > 0:                               # tanh y = 1 - 2 / (1 + exp(2 y))
                x = cap * (1.0 - 2.0 / (1.0 + torch.exp(2.0 / cap * x)))
            if s["slopes"] is not None:
                x = x - float(s["slopes"][h]) * (i - j).abs()
            o = torch.softmax(x.masked_fill(hide, -math.inf), 1) @ leaves[2]
            O[n, lo:hi, h] = o.detach()
            if train:
                a, b, d = torch.autograd.grad(o, leaves, cut(s["dO"], lo, hi, h))
                dq[n, lo:hi, h] = a
                dk[n, :L, kv] += b
                dv[n, :L, kv] += d
    O = O.flatten(2)
    return dict(O=O, dqkv=torch.cat([x.flatten(2) for x in (dq, dk, dv)], dim=2)) if train else O
