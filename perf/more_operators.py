"""The experts' products that training needs, in bf16 with their gradients, and
those of serving in 8-bit floating point, at the sizes that MoE layers meet.

A case's "kind" says what one pass is:
  product      expert_matmul_bf16: each block of rows times its expert's weights;
               "trans": the weights' rows are summed over (with them as the forward
               pass keeps them, that is the gradient of the product's input);
               "act" swiglu (the first half of the N channels gates the second;
               with "pre" the channels before it are kept) or swiglu_grad (the
               products are the gradient of a SwiGLU's output, whose kept
               channels are an input, and become the gradient of those)
  weight_grad  expert_weight_grad: the weights' gradients from both sides' rows
  quant        quant_blocks: rows to e4m3 with a power-of-two scale for each 128
               elements
  product8     expert_matmul_fp8: the blocks' products on those

M rows, of which the last "tail" belong to no block, "blocks" blocks over
"experts" weights, N channels, K elements summed over (weight_grad: dw has N x K
elements, the rows are summed over); "skew" spreads the blocks' sizes, "layer"
fixes them; "type" of the result.
"""
import math
import random

import torch

own = False
DEV = "cuda"
BF16, F32, E4M3, E8M0 = torch.bfloat16, torch.float32, torch.float8_e4m3fn, torch.float8_e8m0fnu
BLOCK = 128     # elements that share a scale
PART = 8192     # rows at a time where 64 bits are wide


def _product(name, M, N, K, blocks, experts, trans=False, act="none", pre=False, type="bf16", skew=0.4, layer=1, tail=0,
             kind="product"):
    return dict(name=name, kind=kind, M=M, N=N, K=K, blocks=blocks, experts=experts, trans=trans, act=act, pre=pre,
                type=type, skew=skew, layer=layer, tail=tail)


def _weight_grad(name, M, N, K, blocks, experts, type="f32", skew=0.4, layer=1, tail=0):
    return dict(name=name, kind="weight_grad", M=M, N=N, K=K, blocks=blocks, experts=experts, type=type, skew=skew,
                layer=layer, tail=tail)


def _quant(name, rows, K, ld, type):
    return dict(name=name, kind="quant", rows=rows, K=K, ld=ld, type=type)


def listed():
    return [
        # training layer, DeepSeek-V3-shaped: 4096 tokens, top-8, 4 experts and a replica a rank;
        # gate and up products, their channels kept for the backward pass
        _product("up_train", 32768, 4096, 7168, 5, 5, act="swiglu", pre=True, layer=2),
        # the gradient through the down product and the SwiGLU, the same layer
        _product("down_grad_train", 32768, 2048, 7168, 5, 5, trans=True, act="swiglu_grad", layer=2),
        # the gradient of the gate and up products' input: GLM-4.5-Air-shaped, ragged blocks
        _product("up_grad_ragged", 16381, 4096, 2816, 6, 6, trans=True, skew=0.7, layer=3),
        # both weight gradients of a layer: DeepSeek-V3-shaped gate and up, fp32 main gradients
        _weight_grad("weight_grad_train", 32768, 4096, 7168, 5, 5, layer=2),
        # a small layer's down weights, ragged blocks with masked slots behind them, bf16
        _weight_grad("weight_grad_ragged", 2991, 2880, 1440, 16, 16, type="bf16", skew=0.9, layer=4, tail=37),
        # one row of a decoded token in bf16: the bytes of one expert's weights
        _product("up_token", 1, 4096, 7168, 1, 1, act="swiglu", layer=5),
        # a small ragged batch over many experts, rows of 2880
        _product("down_ragged", 1998, 2880, 1440, 16, 16, skew=0.9, layer=6, tail=14),
        # prefill in 8 bits: the rows that a balanced rank of the DeepSeek-V3-shaped layer draws
        _product("up8_prefill", 131072, 4096, 7168, 10, 10, act="swiglu", layer=7, kind="product8"),
        # decoding: 16 rows over the 10 experts of a rank
        _product("up8_decode", 16, 4096, 7168, 10, 10, act="swiglu", skew=0.5, layer=8, kind="product8"),
        # the down product of a GLM-4.5-Air-shaped rank, ragged blocks
        _product("down8_ragged", 32761, 4096, 1408, 6, 6, skew=0.6, layer=9, kind="product8"),
        # the dispatched rows of a prefill layer before the experts' products
        _quant("quant_prefill", 131072, 7168, 7168, "bf16"),
        # decoded rows, of a length that is no multiple of 128
        _quant("quant_decode", 33, 2880, 2888, "bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: products of one row to 131072 over 1 to 64 blocks, N and K
    from 64 to 8192, weight gradients of the same, quantised rows of up to 12288
    elements."""
    kind = rng.choice(["product", "product", "product", "weight_grad", "weight_grad", "product8", "product8", "quant"])
    layer = rng.randrange(10, 1 << 20)
    if kind == "quant":
        K, rows = 8 * _log_int(rng, 8, 1536), _log_int(rng, 1, 131072)
        while rows * K > 1 << 29:
            rows //= 2
        c = _quant("", rows, K, K + 8 * rng.choice([0, 0, 1, 2]), rng.choice(["bf16", "bf16", "f32"]))
        del c["name"]
        return c
    step = 16 if kind == "product8" else 8
    N, K = 16 * _log_int(rng, 4, 512), step * _log_int(rng, 64 // step, 8192 // step)
    blocks = rng.choice([1, 1, 2, 4, 5, 6, 8, 10, 16, 32, 64])
    while blocks * N * K > 1 << 28:
        blocks = (blocks + 1) // 2
    M = _log_int(rng, 1, 131072)
    while M * N * K > 1 << 40 or M * max(N, K) > 1 << 29:
        M //= 2
    M = max(M, 1)
    common = dict(type=rng.choice(["bf16", "bf16", "f32"]), skew=rng.uniform(0.0, 1.5), layer=layer,
                  tail=rng.choice([0, 0, M // 16]))
    experts = blocks if rng.random() < 0.7 else max(1, blocks - 1)
    if kind == "weight_grad":
        c = _weight_grad("", M, N, K, blocks, experts, **common)
    else:
        act = rng.choice(["none", "swiglu"] if kind == "product8" else ["none", "none", "swiglu", "swiglu_grad"])
        trans = kind == "product" and (act == "swiglu_grad" or rng.random() < 0.4)
        c = _product("", M, N, K, blocks, experts, trans, act, kind == "product" and act == "swiglu" and rng.random() < 0.7,
                     kind=kind, **common)
    del c["name"]
    return c


def _dtype(c):
    return F32 if c["type"] == "f32" else BF16


def _block_sizes(c):
    """Rows of each block and its expert, fixed by the case."""
    r = random.Random(c["layer"])
    w = [math.exp(c["skew"] * r.gauss(0, 1)) for _ in range(c["blocks"])]
    cum, at, total, M = [0], 0.0, sum(w), c["M"] - c["tail"]
    for v in w:
        at += v
        cum.append(min(M, int(round(M * at / total))))
    cum[-1] = M
    of = list(range(c["experts"])) + [r.randrange(c["experts"]) for _ in range(c["blocks"] - c["experts"])]
    r.shuffle(of)
    return cum, of


def _y_width(c):
    """Elements of a row of y."""
    return {"none": c["N"], "swiglu": c["N"] // 2, "swiglu_grad": 2 * c["N"]}[c["act"]]


def _quantise(x):
    """Rows of fp32 values: e4m3 values, and the exponents of their blocks' scales: the
    least e with |x| <= 448 * 2^e in the block, -127 at least."""
    rows, K = x.shape
    n = -(-K // BLOCK)
    b = torch.nn.functional.pad(x, (0, n * BLOCK - K)).view(rows, n, BLOCK)
    m, p = torch.frexp(b.abs().amax(2))
    e = torch.where(m == 0, -127, p - 9 + (m > 0.875).to(p.dtype)).clamp(min=-127)
    q = torch.ldexp(b, -e[:, :, None]).to(E4M3)
    return q.view(rows, n * BLOCK)[:, :K], e


def _scale_bytes(e):
    """Scales as they are held: biased exponents, rows of a multiple of 4 bytes."""
    return torch.nn.functional.pad((e + 127).to(torch.uint8), (0, -e.shape[1] % 4))


def _fp8(gen, rows, K, scale):
    """Rows of normal values, some rows larger, in 8 bits."""
    x = scale * torch.randn(rows, K, device=DEV, generator=gen)
    q, e = _quantise(x * torch.exp(0.3 * torch.randn(rows, 1, device=DEV, generator=gen)))
    return q.contiguous(), _scale_bytes(e)


def prepare(case, seed):
    c, kind = case, case["kind"]
    gen = torch.Generator(device=DEV).manual_seed(seed)
    s = dict(c=c, status=torch.zeros(1, dtype=torch.int32, device=DEV))

    def empty(dtype, *shape):
        return torch.empty(*shape, dtype=dtype, device=DEV)

    def bf16(scale, *shape):
        return empty(BF16, *shape).normal_(std=scale, generator=gen)

    if kind == "quant":
        x = empty(F32 if c["type"] == "f32" else BF16, c["rows"], c["ld"]).normal_(generator=gen)
        x *= torch.exp(0.5 * torch.randn(c["rows"], 1, device=DEV, generator=gen)).to(x.dtype)
        s["x"] = x
        s["q"] = empty(torch.uint8, c["rows"], -(-c["K"] // 16) * 16)
        s["scale"] = empty(torch.uint8, c["rows"], -(-c["K"] // (4 * BLOCK)) * 4)
        return s
    M, N, K, n_w = c["M"], c["N"], c["K"], c["experts"]
    s["at"], s["of"] = _block_sizes(c)
    s["block_off"] = torch.tensor(s["at"], dtype=torch.int64, device=DEV)
    s["block_w"] = torch.tensor(s["of"], dtype=torch.int32, device=DEV)
    if kind == "weight_grad":
        s["dy"], s["x"] = bf16(1e-3, M, N), bf16(1.0, M, K)
        s["dw"] = empty(_dtype(c), n_w, N, K)
        s["ws"] = None
        if own:
            import paper_2606_04101_amd as uep
            s["ws"] = empty(torch.uint8, uep.ultraep_expert_weight_grad_ws_bytes(M, N, K, n_w))
        return s
    s["y"] = torch.zeros(M, _y_width(c), dtype=_dtype(c), device=DEV)
    if kind == "product":
        s["x"] = bf16(1e-3 if c["trans"] else 1.0, M, K)
        s["w"] = bf16(K ** -0.5, n_w, *((K, N) if c["trans"] else (N, K)))
        s["pre"] = None
        if c["act"] == "swiglu_grad":
            s["pre"] = bf16(1.0, M, 2 * N)
        elif c["pre"]:
            s["pre"] = torch.zeros(M, N, dtype=BF16, device=DEV)
        return s
    s["xq"], s["xs"] = empty(E4M3, M, K), empty(torch.uint8, M, -(-K // (4 * BLOCK)) * 4)
    for lo in range(0, M, 16384):
        s["xq"][lo:lo + 16384], s["xs"][lo:lo + 16384] = _fp8(gen, min(16384, M - lo), K, 1.0)
    s["wq"], s["ws"] = empty(E4M3, n_w, N, K), empty(torch.uint8, n_w, N, s["xs"].shape[1])
    for j in range(n_w):
        s["wq"][j], s["ws"][j] = _fp8(gen, N, K, K ** -0.5)
    return s


def _run_own(s):
    import paper_2606_04101_amd as uep
    c, st, kind = s["c"], s["status"], s["c"]["kind"]
    if kind == "quant":
        uep.ultraep_quant_blocks(s["x"], c["rows"], c["K"], c["ld"], s["q"], s["q"].shape[1], s["scale"])
        return dict(q=s["q"].view(E4M3), scale=s["scale"][:, :-(-c["K"] // BLOCK)].view(E8M0))
    M, N, K, n_w = c["M"], c["N"], c["K"], c["experts"]
    if kind == "weight_grad":
        uep.ultraep_expert_weight_grad(s["dy"], s["x"], M, N, K, s["block_off"], s["block_w"], c["blocks"], n_w, N * K,
                                       False, s["dw"], s["ws"], st)
        return dict(dw=s["dw"])
    if kind == "product8":
        uep.ultraep_expert_matmul_fp8(s["xq"], s["xs"], M, s["wq"], s["ws"], n_w, N, K, s["block_off"], s["block_w"],
                                      c["blocks"], c["act"] == "swiglu", s["y"], st)
        return dict(y=s["y"])
    act = {"none": uep.ULTRAEP_NO_ACT, "swiglu": uep.ULTRAEP_SWIGLU, "swiglu_grad": uep.ULTRAEP_SWIGLU_GRAD}[c["act"]]
    uep.ultraep_expert_matmul_bf16(s["x"], M, s["w"], n_w, N * K, N, K, c["trans"], s["block_off"], s["block_w"],
                                   c["blocks"], act, s["pre"], s["y"], st)
    return dict(y=s["y"], pre=s["pre"]) if c["pre"] else dict(y=s["y"])


def _swiglu_grad(v, pre):
    """Gradient of silu(a) * b with respect to a and b, from that of its value."""
    a, b = pre.chunk(2, 1)
    t = 1.0 / (1.0 + torch.exp(-a))
    return torch.cat([v * b * t * (1.0 + a * (1.0 - t)), v * a * t], 1)


def _dequantised(q, scale):
    """fp32 values of e4m3 rows and their scales' bytes."""
    K = q.shape[1]
    f = torch.exp2(scale[:, :-(-K // BLOCK)].float() - 127.0)
    return q.float() * f.repeat_interleave(BLOCK, 1)[:, :K]


def _plain_product(s):
    c = s["c"]
    y, pre = torch.zeros(c["M"], _y_width(c), device=DEV), None
    if c["pre"]:
        pre = torch.zeros(c["M"], c["N"], device=DEV)
    for g in range(c["blocks"]):
        lo, hi, j = s["at"][g], s["at"][g + 1], s["of"][g]
        if hi == lo:
            continue
        if c["kind"] == "product8":
            v = _dequantised(s["xq"][lo:hi], s["xs"][lo:hi]) @ _dequantised(s["wq"][j], s["ws"][j]).t()
        else:
            w = s["w"][j].float()
            v = s["x"][lo:hi].float() @ (w if c["trans"] else w.t())
        if c["pre"]:
            pre[lo:hi] = v
        if c["act"] == "swiglu":
            a, b = v.chunk(2, 1)
            v = a / (1.0 + torch.exp(-a)) * b
        elif c["act"] == "swiglu_grad":
            v = _swiglu_grad(v, s["pre"][lo:hi].float())
        y[lo:hi] = v
    y = y.to(s["y"].dtype)
    return dict(y=y, pre=pre.to(BF16)) if c["pre"] else dict(y=y)


def _plain_weight_grad(s):
    c = s["c"]
    dw = torch.zeros(c["experts"], c["N"], c["K"], device=DEV)
    for g in range(c["blocks"]):
        lo, hi, j = s["at"][g], s["at"][g + 1], s["of"][g]
        if hi > lo:
            dw[j] += s["dy"][lo:hi].float().t() @ s["x"][lo:hi].float()
    return dict(dw=dw.to(s["dw"].dtype))


def _plain_quant(s):
    c = s["c"]
    q, e = _quantise(s["x"][:, :c["K"]].float())
    q = torch.nn.functional.pad(q.view(torch.uint8), (0, s["q"].shape[1] - c["K"]))
    return dict(q=q.view(E4M3), scale=(e + 127).to(torch.uint8).view(E8M0))


def run(state):
    if own:
        return _run_own(state)
    return {"product": _plain_product, "product8": _plain_product, "weight_grad": _plain_weight_grad,
            "quant": _plain_quant}[state["c"]["kind"]](state)


def work(case):
    """Bytes read once and written once, and the arithmetic of the formulas."""
    c, kind = case, case["kind"]
    if kind == "quant":
        K, n = c["K"], -(-c["K"] // BLOCK)
        return {"bytes": c["rows"] * (K * (4 if c["type"] == "f32" else 2) + -(-K // 16) * 16 + n), "flops": 3 * c["rows"] * K}
    M, N, K = c["M"] - c["tail"], c["N"], c["K"]
    at, of = _block_sizes(c)
    used = len({e for g, e in enumerate(of) if at[g + 1] > at[g]})
    size = 4 if c["type"] == "f32" else 2
    if kind == "weight_grad":
        return {"bytes": 2 * M * (N + K) + c["experts"] * N * K * size, "flops": 2 * M * N * K}
    y = M * _y_width(c) * size
    if kind == "product8":
        n = -(-K // BLOCK)
        return {"bytes": M * (K + n) + used * N * (K + n) + y, "flops": 2 * M * N * K}
    kept = 2 * M * (2 * N if c["act"] == "swiglu_grad" else N if c["pre"] else 0)
    return {"bytes": 2 * M * K + 2 * used * N * K + y + kept, "flops": 2 * M * N * K}


def exact(case, seed):
    """The results in 64 bits from the definitions, the SwiGLU's gradient by
    differentiation, e4m3 values by rounding to multiples of their spacing."""
    c, kind = case, case["kind"]
    s = prepare(case, seed)
    if kind == "quant":
        n = -(-c["K"] // BLOCK)
        q = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
        scale = torch.empty(c["rows"], n, dtype=torch.float64, device=DEV)
        for g in range(n):
            lo, hi = g * BLOCK, min(c["K"], (g + 1) * BLOCK)
            x = s["x"][:, lo:hi].double()
            scale[:, g] = torch.exp2(torch.ceil(torch.log2(x.abs().max(1).values / 448)).clamp(min=-127))
            v = x / scale[:, g, None]
            step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3)
            q[:, lo:hi] = torch.round(v / step) * step
        return dict(q=q, scale=scale)
    N, K = c["N"], c["K"]
    if kind == "weight_grad":
        dw = torch.zeros(c["experts"], N, K, dtype=torch.float64, device=DEV)
        for g in range(c["blocks"]):
            for a in range(s["at"][g], s["at"][g + 1], PART):
                b = min(s["at"][g + 1], a + PART)
                dw[s["of"][g]].addmm_(s["dy"][a:b].t().contiguous().double(), s["x"][a:b].double())
        return dict(dw=dw)

    def values(q, scale):
        power = torch.arange(K, device=DEV) // BLOCK
        return torch.ldexp(q.double(), scale[:, power].to(torch.int32) - 127)

    y = torch.zeros(c["M"], _y_width(c), dtype=torch.float64, device=DEV)
    pre = torch.zeros(c["M"], N, dtype=torch.float64, device=DEV) if c["pre"] else None
    for g in range(c["blocks"]):
        j = s["of"][g]
        if s["at"][g + 1] == s["at"][g]:
            continue
        if kind == "product8":
            w = values(s["wq"][j], s["ws"][j])
        else:
            w = s["w"][j].t().contiguous().double() if c["trans"] else s["w"][j].double()
        for a in range(s["at"][g], s["at"][g + 1], PART):
            b = min(s["at"][g + 1], a + PART)
            rows = values(s["xq"][a:b], s["xs"][a:b]) if kind == "product8" else s["x"][a:b].double()
            v = torch.nn.functional.linear(rows, w)
            if c["pre"]:
                pre[a:b] = v
            if c["act"] == "swiglu":
                v = torch.nn.functional.silu(v[:, :N // 2]) * v[:, N // 2:]
            elif c["act"] == "swiglu_grad":
                p = s["pre"][a:b].double().requires_grad_()
                (v,) = torch.autograd.grad(torch.nn.functional.silu(p[:, :N]) * p[:, N:], p, v)
            y[a:b] = v
    return dict(y=y, pre=pre) if c["pre"] else dict(y=y)
