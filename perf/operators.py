"""The operators that stand around the balancing path of an MoE layer, at the
sizes that its workloads meet: the router that draws the routing ids, with its
balance loss and its backward pass, the backward pass of the combine, and the
experts' products in 8-bit integers with the quantisation of their rows.

A case's "kind" says what one pass is:
  route         route: top-k ids, gates and, with "stats", the counts, the sums
                of the scores and the balance loss with its coefficients
  route_grad    route_grad: the logits' gradient from the gates' gradient and
                the balance loss
  combine_grad  combine_grad: the gradients of the experts' output rows and of
                the gates from the gradient of the combined rows
  quant         quant_rows: rows to 8-bit integers with a scale each
  matmul        expert_matmul: each block of rows times its expert's weights

Router: T tokens, E experts, k of them a token, "score" softmax or sigmoid,
"bias" (a selection bias per expert), "groups" / "top_groups" (a token's ids
come from its best groups), "renorm" (a token's gates sum to "scale"), "seq"
(tokens of a sequence, 0: all T are one), "type" of the logits, "pad" (share of
trailing tokens that are padding), "dead" (experts out of service: logit -inf).
Logits are N(0, 1) plus a preference per expert that "layer" fixes.
Products: M rows in "blocks" blocks over "experts" weights of N x K; "act": the
first half of the N channels gates the second (SwiGLU), so a row of y has N / 2
elements; "skew" spreads the blocks' sizes.
"""
import math
import random

import torch

own = False
DEV = "cuda"
ALPHA = 1e-3     # weight of the balance loss
APART = 4e-6     # keys that decide a selection are further apart than this


def _router(name, kind, T, E, k, score, type, bias=False, groups=0, top_groups=0, renorm=True,
            scale=1.0, seq=0, pad=0.0, dead=0, stats=True, spread=0.35, layer=1):
    return dict(name=name, kind=kind, T=T, E=E, k=k, score=score, type=type, bias=bias,
                groups=groups, top_groups=top_groups, renorm=renorm, scale=scale, seq=seq, pad=pad,
                dead=dead, stats=stats, spread=spread, layer=layer)


def _combine(name, T, k, H, pad=0.0):
    return dict(name=name, kind="combine_grad", T=T, k=k, H=H, E=128, pad=pad)


def _quant(name, rows, K, ld, type):
    return dict(name=name, kind="quant", rows=rows, K=K, ld=ld, type=type)


def _matmul(name, M, N, K, blocks, experts, act, type, skew, layer):
    return dict(name=name, kind="matmul", M=M, N=N, K=K, blocks=blocks, experts=experts, act=act,
                type=type, skew=skew, layer=layer)


def listed():
    return [
        # one decoded token through the router, DeepSeek-V3-shaped: latency is everything
        _router("route_token", "route", 1, 256, 8, "sigmoid", "f32", bias=True, groups=8, top_groups=4,
                scale=2.5, stats=False),
        # a training microbatch of four sequences, DeepSeek-V3-shaped, with the balance loss
        _router("route_train", "route", 4096, 256, 8, "sigmoid", "f32", bias=True, groups=8, top_groups=4,
                scale=2.5, seq=1024, layer=9),
        # a softmax router over twice the Qwen3-235B-shaped microbatch, with the balance loss
        _router("route_softmax", "route", 16384, 128, 8, "softmax", "bf16", spread=1.0, layer=8),
        # the training microbatch's backward pass
        _router("route_grad_train", "route_grad", 4096, 256, 8, "sigmoid", "f32", bias=True, groups=8,
                top_groups=4, scale=2.5, seq=1024, layer=9),
        # the backward pass of a ragged batch: padding, top-6 of 72, two experts out of service
        _router("route_grad_ragged", "route_grad", 2999, 72, 6, "softmax", "bf16", renorm=False, seq=700,
                pad=0.11, dead=2, spread=0.5, layer=3),
        # the combine's backward pass, DeepSeek-V3-shaped training layer
        _combine("combine_grad_train", 4096, 8, 7168),
        # the same for a small ragged batch, top-6, rows of 2880
        _combine("combine_grad_ragged", 333, 6, 2880, pad=0.07),
        # the dispatched rows of a prefill layer before the experts' products, DeepSeek-V3-shaped
        _quant("quant_prefill", 131072, 7168, 7168, "bf16"),
        # a ragged batch's rows, whose length is no multiple of 16
        _quant("quant_ragged", 2999, 2888, 2896, "bf16"),
        # decoding: 16 rows over the 10 experts of a rank, gate and up products with SwiGLU
        _matmul("matmul_decode", 16, 4096, 7168, 10, 10, True, "bf16", 0.5, 5),
        # prefill: the rows that a balanced rank of the DeepSeek-V3-shaped layer draws
        _matmul("matmul_prefill", 131072, 4096, 7168, 10, 10, True, "bf16", 0.3, 6),
        # the down product of a GLM-4.5-Air-shaped rank: 6 slots, ragged blocks
        _matmul("matmul_down", 32761, 4096, 1408, 6, 6, False, "bf16", 0.6, 7),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: routers of up to 65536 tokens and 512 experts, combines of
    up to 1 GiB of rows, quantised rows of up to 12288 elements, products of one
    row to 131072 over 1 to 64 blocks."""
    kind = rng.choice(["route", "route", "route_grad", "combine_grad", "quant", "matmul", "matmul", "matmul"])
    layer = rng.randrange(10, 1 << 20)
    if kind in ("route", "route_grad"):
        E = rng.choice([16, 60, 64, 72, 96, 128, 128, 192, 256, 256, 384, 512])
        grouped = E % 8 == 0 and E >= 32 and rng.random() < 0.4
        k = rng.choice([v for v in (1, 2, 4, 6, 8, 8, 10, 12) if v <= E // (2 if grouped else 1)])
        T = _log_int(rng, 1, 65536)
        score = rng.choice(["softmax", "sigmoid"])
        c = _router("", kind, T, E, k, score, rng.choice(["f32", "bf16"]), score == "sigmoid" and rng.random() < 0.7,
                    8 if grouped else 0, 4 if grouped else 0, rng.random() < 0.7, rng.choice([1.0, 2.5, 0.7]),
                    rng.choice([0, 0, max(1, T // rng.randint(1, 9))]), rng.choice([0.0, 0.0, rng.uniform(0.01, 0.3)]),
                    rng.choice([0, 0, 1, 3]), kind == "route_grad" or rng.random() < 0.7, rng.uniform(0.2, 1.2), layer)
    elif kind == "combine_grad":
        k = rng.choice([1, 2, 4, 6, 8, 8, 10, 12])
        T, H = _log_int(rng, 1, 16384), 8 * _log_int(rng, 32, 1536)
        while T * k * H > 1 << 28:
            T //= 2
        c = _combine("", T, k, H if H != 3072 else H + 8, rng.choice([0.0, 0.0, rng.uniform(0.01, 0.3)]))
    elif kind == "quant":
        K = 8 * _log_int(rng, 16, 1536)
        K = K if K != 3072 else K + 8
        rows = _log_int(rng, 1, 131072)
        while rows * K > 1 << 29:
            rows //= 2
        c = _quant("", rows, K, K + 8 * rng.choice([0, 0, 1, 2]), rng.choice(["bf16", "bf16", "f32"]))
    else:
        K, F = 16 * _log_int(rng, 16, 512), 8 * _log_int(rng, 16, 512)
        K, F = (v if v not in (1536, 3072) else v + 32 for v in (K, F))
        act = rng.random() < 0.5
        N = 2 * F if act else F
        blocks = rng.choice([1, 1, 4, 6, 8, 10, 16, 32, 64])
        while blocks * N * K > 1 << 29:
            blocks = (blocks + 1) // 2
        M = _log_int(rng, 1, 131072)
        while M * N * K > 1 << 41 or M * max(N, K) > 1 << 29:
            M //= 2
        c = _matmul("", max(M, 1), N, K, blocks, blocks if rng.random() < 0.7 else max(1, blocks - 1), act,
                    rng.choice(["bf16", "bf16", "f32"]), rng.uniform(0.0, 1.5), layer)
    del c["name"]
    return {n: v + 8 if v == 3072 else v for n, v in c.items()}


def _dtype(c):
    return torch.float32 if c["type"] == "f32" else torch.bfloat16


def _segments(c):
    """Sequences and their tokens."""
    L = c["seq"] or c["T"]
    return -(-c["T"] // L), L


def _block_sizes(c):
    """Rows of each block and its expert, fixed by the case."""
    r = random.Random(c["layer"])
    w = [math.exp(c["skew"] * r.gauss(0, 1)) for _ in range(c["blocks"])]
    cum, at, total = [0], 0.0, sum(w)
    for v in w:
        at += v
        cum.append(min(c["M"], int(round(c["M"] * at / total))))
    cum[-1] = c["M"]
    of = list(range(c["experts"])) + [r.randrange(c["experts"]) for _ in range(c["blocks"] - c["experts"])]
    r.shuffle(of)
    return cum, of


def _int8(gen, rows, n, scale):
    """Rows of normal values as 8-bit integers, and their scales."""
    x = scale * torch.randn(rows, n, device=DEV, generator=gen)
    s = x.abs().amax(1).clamp(min=1e-12) / 127
    return (x / s[:, None]).round_().to(torch.int8), s


def _logits(c, gen):
    lg = torch.Generator(device=DEV).manual_seed(7919 * c["layer"] + 13)
    T, E = c["T"], c["E"]
    prefer = c["spread"] * torch.randn(E, device=DEV, generator=lg)
    bias = None
    if c["bias"]:  # a trained selection bias pulls against the preferences, in steps of 1/1024
        bias = torch.round(-0.1 * prefer * 1024 + 16 * torch.randn(E, device=DEV, generator=lg)) / 1024
    alive = torch.rand(E, device=DEV, generator=lg).argsort() >= c["dead"]

    def some(n):
        z = (torch.randn(n, E, device=DEV, generator=gen) + prefer).to(_dtype(c))
        return z.masked_fill(~alive, float("-inf"))

    z = some(T)
    if c["bias"] or c["groups"]:  # a token whose selection hangs on a rounding is drawn again
        for _ in range(60):
            bad = _close(c, z, bias).nonzero()[:, 0]
            if not bad.numel():
                break
            z[bad] = some(bad.numel())
    return z, bias


def _close(c, z, bias):
    """Tokens that have unequal keys, or sums of a group's two largest, within
    APART of one another where the selection could turn on it (equal keys go to
    the lower id in any precision)."""
    key = z.double()
    if c["score"] == "sigmoid":
        key = torch.sigmoid(key)
    if bias is not None:
        key = key + bias.double()
    key = torch.where(torch.isinf(z), float("-inf"), key)
    bad = torch.zeros(z.shape[0], dtype=torch.bool, device=DEV)

    def near(v, n, least):
        v = v[:, :n].clamp(min=-1e30)
        gap = v[:, :-1] - v[:, 1:]
        return ((gap >= least) & (gap < APART) & (v[:, 1:] > -1e29)).any(1)

    if c["groups"]:
        kg = key.view(-1, c["groups"], c["E"] // c["groups"])
        score, at = kg.topk(2, dim=2).values.sum(2).sort(dim=1, descending=True)
        n = c["top_groups"]
        bad |= near(score[:, n - 1:n + 1], 2, 0.0)
        keep = torch.zeros_like(score, dtype=torch.bool).scatter_(1, at[:, :n], True)
        key = kg.masked_fill(~keep[:, :, None], float("-inf")).reshape(-1, c["E"])
    return bad | near(key.sort(dim=1, descending=True).values, c["k"] + 1, 1e-300)


def _select(c, z, bias, mask):
    """[T, k] ids by falling key, ties to the lower id; -1 where none is left."""
    key = z
    if c["score"] == "sigmoid" and (bias is not None or c["groups"]):
        key = 1.0 / (1.0 + torch.exp(-z))
    if bias is not None:
        key = key + bias
    key = torch.where(torch.isinf(z), float("-inf"), key)
    if c["groups"]:
        kg = key.view(-1, c["groups"], c["E"] // c["groups"])
        score = kg.sort(dim=2, descending=True).values[:, :, :2].sum(2)
        best = score.sort(dim=1, descending=True, stable=True).indices[:, :c["top_groups"]]
        keep = torch.zeros_like(score, dtype=torch.bool).scatter_(1, best, True)
        key = kg.masked_fill(~keep[:, :, None], float("-inf")).reshape(key.shape)
    v, ids = key.sort(dim=1, descending=True, stable=True)
    v, ids = v[:, :c["k"]], ids[:, :c["k"]]
    return torch.where(torch.isinf(v) | (mask[:, None] == 0), -1, ids).to(torch.int32)


def _scores(c, z):
    if c["score"] == "sigmoid":
        s = 1.0 / (1.0 + torch.exp(-z))
        return s, s / s.sum(1, keepdim=True)
    e = torch.exp(z - z.amax(1, keepdim=True))
    p = e / e.sum(1, keepdim=True)
    return p, p


def _gates(c, s, ids):
    g = torch.where(ids < 0, 0.0, s.gather(1, ids.clamp(min=0).long()))
    if c["renorm"]:
        g = torch.where(ids < 0, 0.0, g / g.sum(1, keepdim=True))
    return g * c["scale"]


def _counts(c, ids):
    """Counts of a sequence's ids by expert, and its tokens that have any."""
    n, L = _segments(c)
    seq = (torch.arange(c["T"], device=DEV) // L)[:, None].expand(ids.shape)
    at = torch.where(ids < 0, n * c["E"], seq * c["E"] + ids)
    counts = torch.zeros(n * c["E"] + 1, dtype=torch.int32, device=DEV)
    counts.scatter_add_(0, at.reshape(-1).long(), torch.ones(at.numel(), dtype=torch.int32, device=DEV))
    tokens = torch.zeros(n, dtype=torch.int32, device=DEV)
    tokens.scatter_add_(0, seq[:, 0], (ids[:, 0] >= 0).to(torch.int32))
    return counts[:-1].view(n, c["E"]), tokens


def _coef(c, counts, tokens):
    """The balance loss is the sum of these times the sums of the scores: mean
    over sequences of ALPHA * E * sum_e (share of the ids)_e (mean score)_e."""
    n = tokens.to(torch.float32)[:, None]
    w = ALPHA * c["E"] / (counts.shape[0] * c["k"]) * counts.to(torch.float32) / (n * n)
    return torch.where(n > 0, w, 0.0)


def _by_sequence(c, p):
    """Sums of p over each sequence's tokens."""
    n, L = _segments(c)
    p = torch.nn.functional.pad(p, (0, 0, 0, n * L - c["T"]))
    return p.view(n, L, c["E"]).sum(1)


def _layout(c, gen):
    """row_of_slot of a dispatch (rows by expert, then token) and the routed rows."""
    T, k = c["T"], c["k"]
    ids = (torch.randn(T, c["E"], device=DEV, generator=gen)
           + torch.linspace(0, 2, c["E"], device=DEV)).topk(k, dim=1).indices
    ids[T - int(T * c["pad"]):] = c["E"]
    ids = ids.reshape(-1)
    order = ids.sort(stable=True).indices
    row = torch.empty_like(order)
    row[order] = torch.arange(T * k, device=DEV)
    row = torch.where(ids == c["E"], -1, row).to(torch.int32)
    return row, (row >= 0).sum().view(1)


def prepare(case, seed):
    c, kind = case, case["kind"]
    gen = torch.Generator(device=DEV).manual_seed(seed)
    s = dict(c=c, status=torch.zeros(1, dtype=torch.int32, device=DEV))

    def empty(dtype, *shape):
        return torch.empty(*shape, dtype=dtype, device=DEV)

    def bf16(*shape):
        return empty(torch.bfloat16, *shape).normal_(generator=gen)

    if kind in ("route", "route_grad"):
        T, E, k = c["T"], c["E"], c["k"]
        n, _ = _segments(c)
        s["logits"], s["bias"] = _logits(c, gen)
        s["mask"] = torch.ones(T, dtype=torch.uint8, device=DEV)
        s["mask"][T - int(T * c["pad"]):] = 0
        s["n"] = n
        if own:
            import paper_2606_04101_amd as uep
            s["router"] = uep.Router(E, k, uep.ULTRAEP_SIGMOID if c["score"] == "sigmoid" else uep.ULTRAEP_SOFTMAX,
                                     renorm=c["renorm"], n_group=c["groups"], top_group=c["top_groups"],
                                     scale=c["scale"], seq_len=c["seq"])
        if kind == "route":
            s["topk"], s["gate"] = empty(torch.int32, T, k), empty(torch.float32, T, k)
            s["ws"] = None
            for name, dt, shape in (("counts", torch.int32, (n, E)), ("prob_sum", torch.float32, (n, E)),
                                    ("tokens", torch.int32, (n,)), ("loss", torch.float32, (1,)),
                                    ("coef", torch.float32, (n, E))):
                s[name] = empty(dt, *shape) if c["stats"] else None
            if own and c["stats"]:
                s["ws"] = empty(torch.uint8, uep.ultraep_route_ws_bytes(T, s["router"]))
        else:  # what the forward pass left, and the gates' gradient from the combine
            s["topk"] = _select(c, s["logits"].float(), s["bias"], s["mask"])
            s["coef"] = _coef(c, *_counts(c, s["topk"]))
            s["dgate"] = 1e-3 * torch.randn(T, k, device=DEV, generator=gen)
            s["dloss"] = 1.0 + torch.rand(1, device=DEV, generator=gen)
            s["dlogits"] = torch.zeros_like(s["logits"])
    elif kind == "combine_grad":
        T, k, H = c["T"], c["k"], c["H"]
        s["rows"], s["n_routed"] = _layout(c, gen)
        s["y"], s["dout"] = bf16(T * k, H), bf16(T, H)
        s["gate"] = torch.softmax(torch.randn(T, k, device=DEV, generator=gen), 1).contiguous()
        s["dy"], s["dgate"] = torch.zeros_like(s["y"]), empty(torch.float32, T, k)
    elif kind == "quant":
        x = empty(_dtype(c), c["rows"], c["ld"]).normal_(generator=gen)
        x *= torch.exp(0.5 * torch.randn(c["rows"], 1, device=DEV, generator=gen)).to(x.dtype)
        s["x"] = x
        s["q"] = empty(torch.int8, c["rows"], -(-c["K"] // 16) * 16)
        s["scale"] = empty(torch.float32, c["rows"])
    else:
        M, N, K = c["M"], c["N"], c["K"]
        s["at"], s["of"] = _block_sizes(c)
        s["xq"], s["xs"] = empty(torch.int8, M, K), empty(torch.float32, M)
        for lo in range(0, M, 16384):
            s["xq"][lo:lo + 16384], s["xs"][lo:lo + 16384] = _int8(gen, min(16384, M - lo), K, 1.0)
        s["wq"], s["ws"] = empty(torch.int8, c["experts"], N, K), empty(torch.float32, c["experts"], N)
        for j in range(c["experts"]):
            s["wq"][j], s["ws"][j] = _int8(gen, N, K, K ** -0.5)
        s["block_off"] = torch.tensor(s["at"], dtype=torch.int64, device=DEV)
        s["block_w"] = torch.tensor(s["of"], dtype=torch.int32, device=DEV)
        s["y"] = torch.zeros(M, N // 2 if c["act"] else N, dtype=_dtype(c), device=DEV)
    return s


def _run_own(s):
    import paper_2606_04101_amd as uep
    c, st, kind = s["c"], s["status"], s["c"]["kind"]
    if kind == "route":
        uep.ultraep_route(s["logits"], c["T"], c["E"], s["router"], s["bias"], s["mask"], s["topk"], s["gate"],
                          s["counts"], s["prob_sum"], s["tokens"], s["ws"], st)
        if not c["stats"]:
            return dict(topk=s["topk"], gate=s["gate"])
        uep.ultraep_balance_loss(s["counts"], s["tokens"], s["prob_sum"], s["tokens"], s["n"], s["router"], ALPHA,
                                 s["loss"], s["coef"])
        return {n: s[n] for n in ("topk", "gate", "counts", "prob_sum", "tokens", "loss", "coef")}
    if kind == "route_grad":
        uep.ultraep_route_grad(s["logits"], c["T"], c["E"], s["router"], s["mask"], s["topk"], s["dgate"],
                               s["coef"], s["dloss"], s["dlogits"], st)
        return dict(dlogits=s["dlogits"])
    if kind == "combine_grad":
        uep.ultraep_combine_grad(s["dout"], s["y"], c["T"] * c["k"], s["gate"], s["rows"], c["T"], c["k"], c["H"],
                                 s["n_routed"], s["dy"], s["dgate"], st)
        return dict(dy=s["dy"], dgate=s["dgate"])
    if kind == "quant":
        uep.ultraep_quant_rows(s["x"], c["rows"], c["K"], c["ld"], s["q"], s["q"].shape[1], s["scale"])
        return dict(q=s["q"], scale=s["scale"])
    uep.ultraep_expert_matmul(s["xq"], s["xs"], c["M"], s["wq"], s["ws"], c["experts"], c["N"], c["K"],
                              s["block_off"], s["block_w"], c["blocks"], c["act"], s["y"], st)
    return dict(y=s["y"])


def _plain_route(s):
    c = s["c"]
    z = s["logits"].float()
    ids = _select(c, z, s["bias"], s["mask"])
    score, p = _scores(c, z)
    gate = _gates(c, score, ids)
    if not c["stats"]:
        return dict(topk=ids, gate=gate)
    counts, tokens = _counts(c, ids)
    prob_sum = _by_sequence(c, torch.where(ids[:, :1] < 0, 0.0, p))
    coef = _coef(c, counts, tokens)
    return dict(topk=ids, gate=gate, counts=counts, prob_sum=prob_sum, tokens=tokens,
                loss=(coef * prob_sum).sum().view(1), coef=coef)


def _plain_route_grad(s):
    c, ids = s["c"], s["topk"]
    z = s["logits"].float()
    at = ids.clamp(min=0).long()
    score, p = _scores(c, z)
    seq = torch.arange(c["T"], device=DEV) // _segments(c)[1]
    w = s["dloss"] * s["coef"][seq]                       # of the balance loss with respect to p
    dz = p * (w - (w * p).sum(1, keepdim=True))
    if c["score"] == "sigmoid":
        dz = dz * (1.0 - score)
    dg = torch.where(ids < 0, 0.0, s["dgate"]) * c["scale"]
    sel = torch.where(ids < 0, 0.0, score.gather(1, at))
    if c["renorm"]:
        q = torch.where(ids < 0, 0.0, sel / sel.sum(1, keepdim=True))
        d = q * (dg - (dg * q).sum(1, keepdim=True))
    else:
        d = sel * dg
    if c["score"] == "sigmoid":
        d = d * (1.0 - score.gather(1, at))
    elif not c["renorm"]:
        dz = dz - p * d.sum(1, keepdim=True)
    dz = dz.scatter_add(1, at, torch.where(ids < 0, 0.0, d))
    return dict(dlogits=torch.where(ids[:, :1] < 0, 0.0, dz).to(s["logits"].dtype))


def _plain_combine_grad(s):
    c = s["c"]
    T, k = c["T"], c["k"]
    rows = s["rows"].long()
    dout, y = s["dout"].float(), s["y"][rows.clamp(min=0)].float()
    dgate = torch.where(rows.view(T, k) < 0, 0.0, (y.view(T, k, -1) * dout[:, None, :]).sum(2))
    slot = torch.full((T * k + 1,), -1, dtype=torch.long, device=DEV)  # the last takes the padding
    slot[torch.where(rows < 0, T * k, rows)] = torch.arange(T * k, device=DEV)
    slot = slot[:-1]
    back = slot.clamp(min=0)
    dy = torch.where(slot[:, None] < 0, 0.0, s["gate"].view(-1)[back][:, None] * dout[back // k])
    return dict(dy=dy.to(s["y"].dtype), dgate=dgate)


def _plain_quant(s):
    c = s["c"]
    x = s["x"][:, :c["K"]].float()
    most = x.abs().amax(1)
    top, live = torch.full_like(most, 127.0), most > 2.0 ** -100
    scale, inv = torch.where(live, most / top, 0.0), torch.where(live, top / most, 0.0)
    q = torch.round(x * inv[:, None]).to(torch.int8)
    return dict(q=torch.nn.functional.pad(q, (0, s["q"].shape[1] - c["K"])), scale=scale)


def _plain_matmul(s):
    c, parts = s["c"], []
    for g in range(c["blocks"]):
        lo, hi, j = s["at"][g], s["at"][g + 1], s["of"][g]
        if hi == lo:
            continue
        v = s["xq"][lo:hi].float() @ s["wq"][j].float().t()
        v = v * s["xs"][lo:hi, None] * s["ws"][j]
        if c["act"]:
            a, b = v.chunk(2, 1)
            v = a / (1.0 + torch.exp(-a)) * b
        parts.append(v.to(s["y"].dtype))
    return dict(y=torch.cat(parts))


def run(state):
    if own:
        return _run_own(state)
    return {"route": _plain_route, "route_grad": _plain_route_grad, "combine_grad": _plain_combine_grad,
            "quant": _plain_quant, "matmul": _plain_matmul}[state["c"]["kind"]](state)


def work(case):
    """Bytes read once and written once; the arithmetic of the formulas (an
    exponential counts as one)."""
    c, kind = case, case["kind"]
    if kind in ("route", "route_grad"):
        T, E, k = c["T"], c["E"], c["k"]
        z = T * E * (4 if c["type"] == "f32" else 2)
        stats = 4 * _segments(c)[0] * E
        if kind == "route_grad":
            return {"bytes": 2 * z + T + 8 * T * k + stats, "flops": 8 * T * E}
        return {"bytes": z + T + 8 * T * k + (3 * stats if c["stats"] else 0), "flops": 5 * T * E}
    if kind == "combine_grad":
        T, k, H = c["T"], c["k"], c["H"]
        routed = (T - int(T * c["pad"])) * k
        return {"bytes": 2 * H * (routed + T * k + T) + 12 * T * k, "flops": 3 * routed * H}
    if kind == "quant":
        K = c["K"]
        return {"bytes": c["rows"] * (K * (4 if c["type"] == "f32" else 2) + -(-K // 16) * 16 + 4),
                "flops": 3 * c["rows"] * K}
    M, N, K = c["M"], c["N"], c["K"]
    at, of = _block_sizes(c)
    used = len({e for g, e in enumerate(of) if at[g + 1] > at[g]})
    n_out = N // 2 if c["act"] else N
    return {"bytes": M * (K + 4) + used * N * (K + 4) + M * n_out * (4 if c["type"] == "f32" else 2),
            "flops": 2 * M * N * K}


def exact(case, seed):
    """The floating outputs in 64 bits, from the definitions: the router's
    gradient by differentiating what it is the gradient of."""
    c, kind = case, case["kind"]
    s = prepare(case, seed)
    if kind in ("route", "route_grad"):
        T, E = c["T"], c["E"]
        z = s["logits"].double().requires_grad_(kind == "route_grad")
        s64 = torch.sigmoid(z) if c["score"] == "sigmoid" else torch.softmax(z, 1)
        p = s64 / s64.sum(1, keepdim=True)
        if kind == "route":
            key = s["logits"].double() if c["score"] == "softmax" or not (c["bias"] or c["groups"]) else s64
            key = key + (s["bias"].double() if c["bias"] else 0.0)
            key = key.masked_fill(s["logits"] == float("-inf"), float("-inf"))
            if c["groups"]:
                kg = key.view(T, c["groups"], -1)
                sums = kg.topk(2, dim=2).values.sum(2)
                worst = sums.topk(c["top_groups"], dim=1).values[:, -1:]
                key = kg.masked_fill((sums < worst)[:, :, None], float("-inf")).view(T, E)
            val, ids = torch.sort(key, dim=1, descending=True, stable=True)
            ids = torch.where(torch.isinf(val), -1, ids)[:, :c["k"]]
            ids[s["mask"] == 0] = -1
        else:
            ids = s["topk"].long()
        on = torch.zeros(T, E + 1, dtype=torch.float64, device=DEV)
        on.scatter_(1, torch.where(ids < 0, E, ids), 1.0)
        on = on[:, :E]
        some = (on.sum(1, keepdim=True) > 0).double()
        gate = s64 * on * c["scale"]
        if c["renorm"]:
            gate = gate / (s64 * on).sum(1, keepdim=True).masked_fill(some == 0, 1.0)
        gate = torch.where(ids < 0, 0.0, gate.gather(1, ids.clamp(min=0)))
        if kind == "route_grad":
            seq = torch.arange(T, device=DEV) // _segments(c)[1]
            of = (gate * s["dgate"].double()).sum()
            of = of + s["dloss"].double() * (s["coef"].double()[seq] * p * some).sum()
            (dz,) = torch.autograd.grad(of, z)
            return dict(dlogits=dz)
        if not c["stats"]:
            return dict(topk=None, gate=gate)
        n, L = _segments(c)
        member = torch.nn.functional.one_hot(torch.arange(T, device=DEV) // L, n).double().t()
        total, share = member @ (p * some), member @ on
        tok = member @ some
        coef = torch.where(tok > 0, ALPHA * E * share / (n * c["k"] * tok.clamp(min=1) ** 2), 0.0)
        return dict(topk=None, gate=gate, counts=None, prob_sum=total, tokens=None,
                    loss=(coef * total).sum().view(1), coef=coef)
    if kind == "combine_grad":
        T, k, H = c["T"], c["k"], c["H"]
        dy = torch.zeros(T * k, H, dtype=torch.float64, device=DEV)
        dgate = torch.zeros(T, k, dtype=torch.float64, device=DEV)
        rows, dout = s["rows"].view(T, k).long(), s["dout"].double()
        for j in range(k):
            on = rows[:, j] >= 0
            dgate[on, j] = torch.linalg.vecdot(dout[on], s["y"][rows[on, j]].double())
            dy[rows[on, j]] = s["gate"][on, j, None].double() * dout[on]
        return dict(dy=dy, dgate=dgate)
    if kind == "quant":
        most = s["x"][:, :c["K"]].double().abs().max(1).values
        return dict(q=None, scale=torch.where(most > 2.0 ** -100, most / 127, 0.0))
    y = torch.empty(s["y"].shape, dtype=torch.float64, device=DEV)
    for g in range(c["blocks"]):
        lo, hi, j = s["at"][g], s["at"][g + 1], s["of"][g]
        for a in range(lo, hi, 8192):  # a block's rows in parts: the products in 64 bits are wide
            b = min(hi, a + 8192)
            v = torch.mm(s["xq"][a:b].double(), s["wq"][j].double().t()) * torch.outer(s["xs"][a:b].double(), s["ws"][j].double())
            if c["act"]:
                v = torch.nn.functional.silu(v[:, :c["N"] // 2]) * v[:, c["N"] // 2:]
            y[a:b] = v
    return dict(y=y)
