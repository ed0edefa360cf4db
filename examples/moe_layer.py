"""One MoE layer of this rank on one GPU, from the router's logits to the
combined rows and back: what the library's calls look like in a training step
and in serving.

  python examples/moe_layer.py

Training: the router's ids, gates and balance loss, the load count's row taken
from the router's counts, the plan, the dispatch, the experts (bf16, torch), the
combine, and every backward pass; a few steps of SGD bring the balance loss down.
Serving: the same layer with its experts in 8-bit integers.

The other ranks' tokens are random, and all experts' weights are in this process:
the blocks that a real program would send to other ranks are multiplied here.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2606_04101_amd as uep  # noqa: E402

DEV, BF16, F32, I32, I64 = "cuda", torch.bfloat16, torch.float32, torch.int32, torch.int64


class Layer:
    """The plan's buffers and workspaces, made once, and what the latest forward pass
    left: new tensors each time, since earlier ones may still wait for their backward
    pass (whose functions hold on to theirs)."""

    def __init__(self, R, E, n_slot, k, T, H, F, seq_len=0, score=uep.ULTRAEP_SOFTMAX, seed=0):
        self.T, self.k, self.H, self.F, self.E = T, k, H, F, E
        self.g = uep.Group(R, E, n_slot, max(1, T // 16))
        self.plan = uep.Plan(self.g)
        self.r = uep.Router(E, k, score, renorm=True, seq_len=seq_len)
        self.status = torch.zeros(1, dtype=I32, device=DEV)
        gen = torch.Generator(device=DEV).manual_seed(seed)
        other = torch.rand(R, E, device=DEV, generator=gen) + 0.5
        self.load = (other / other.sum(1, keepdim=True) * T * k).to(I32)  # the other ranks' rows
        self.gen = gen
        self.n_seg = self.r.n_seg(T)
        self.route_ws = self.empty(torch.uint8, uep.ultraep_route_ws_bytes(T, self.r))
        self.ws = self.empty(torch.uint8, uep.ultraep_dispatch_ws_bytes(T, k, self.g))

    def empty(self, dtype, *shape):
        return torch.empty(*shape, dtype=dtype, device=DEV)

    def route(self, logits):
        """Ids, gates and statistics of a microbatch."""
        n, E, T, k = self.n_seg, self.E, self.T, self.k
        self.topk, self.gate = self.empty(I32, T, k), self.empty(F32, T, k)
        self.counts, self.prob_sum = self.empty(I32, n, E), self.empty(F32, n, E)
        self.tokens = self.empty(I32, n)
        uep.ultraep_route(logits, T, E, self.r, None, None, self.topk, self.gate, self.counts, self.prob_sum,
                          self.tokens, self.route_ws, self.status)

    def make_plan(self, rank=0):
        """The load matrix's row of this rank is the router's counts (summed over its
        sequences); then the plan and the dispatch's layout."""
        self.rows, self.off = self.empty(I32, self.T * self.k), self.empty(I64, self.g.R * self.g.S + 1)
        torch.sum(self.counts, 0, dtype=I32, out=self.load[rank])
        uep.ultraep_plan(self.load, self.g, self.plan)
        uep.ultraep_dispatch_layout(self.topk, self.T, self.k, rank, self.g, self.plan, self.rows, self.off, self.ws,
                                    self.status)

    def block_experts(self):
        """The expert of each block (destination rank, physical slot), -1 for an empty slot."""
        g = self.g
        main = torch.arange(g.E, dtype=I32, device=DEV).view(g.R, g.n_main)
        return torch.cat([main, self.plan.slot_expert.view(g.R, g.n_slot)], 1).reshape(-1).contiguous()

    def check(self):
        assert int(self.status.item()) == 0, uep.ultraep_strerror(int(self.status.item()))


class Route(torch.autograd.Function):
    """logits [T][E] -> gates [T][k] and the balance loss; the ids stay in the layer."""

    @staticmethod
    def forward(ctx, logits, layer, alpha):
        m, loss = layer, torch.empty(1, device=DEV)
        m.route(logits)
        coef = m.empty(F32, m.n_seg, m.E)
        uep.ultraep_balance_loss(m.counts, m.tokens, m.prob_sum, m.tokens, m.n_seg, m.r, alpha, loss, coef)
        ctx.save_for_backward(logits, m.topk, coef)
        ctx.layer = m
        gate, m.gate = m.gate, m.gate.detach()  # (the layer holds no graph)
        return gate, loss

    @staticmethod
    def backward(ctx, dgate, dloss):
        (logits, topk, coef), m = ctx.saved_tensors, ctx.layer
        dlogits = torch.empty_like(logits)
        uep.ultraep_route_grad(logits, m.T, m.E, m.r, None, topk, dgate.contiguous(), coef, dloss.contiguous(),
                               dlogits, m.status)
        return dlogits, None, None


class Dispatch(torch.autograd.Function):
    """Token rows [T][H] -> rows by expert block [T*k][H]; backward: the combine with gates 1."""

    @staticmethod
    def forward(ctx, x, layer):
        m = ctx.layer = layer
        ctx.save_for_backward(m.rows)
        send = torch.empty(m.T * m.k, m.H, dtype=BF16, device=DEV)
        uep.ultraep_dispatch_scatter(x, m.T, m.k, m.H, m.rows, m.off[-1:], send)
        return send

    @staticmethod
    def backward(ctx, dsend):
        (rows,), m = ctx.saved_tensors, ctx.layer
        dx, one = torch.empty(m.T, m.H, dtype=BF16, device=DEV), torch.ones(m.T, m.k, device=DEV)
        uep.ultraep_combine(dsend.contiguous(), m.T * m.k, one, rows, m.T, m.k, m.H, dx, m.status)
        return dx, None


class Combine(torch.autograd.Function):
    """The experts' output rows and the gates -> token rows."""

    @staticmethod
    def forward(ctx, y, gate, layer):
        m = ctx.layer = layer
        ctx.save_for_backward(y, gate, m.rows, m.off)
        out = torch.empty(m.T, m.H, dtype=BF16, device=DEV)
        uep.ultraep_combine(y, m.T * m.k, gate, m.rows, m.T, m.k, m.H, out, m.status)
        return out

    @staticmethod
    def backward(ctx, dout):
        (y, gate, rows, off), m = ctx.saved_tensors, ctx.layer
        dy, dgate = torch.empty_like(y), torch.empty_like(gate)
        uep.ultraep_combine_grad(dout.contiguous(), y, m.T * m.k, gate, rows, m.T, m.k, m.H, off[-1:], dy, dgate,
                                 m.status)
        return dy, dgate, None


def experts_bf16(send, layer, w1, w2):
    """Each block of rows through its expert: silu(x G) * (x U), then the down product."""
    off, of = layer.off.tolist(), layer.block_experts().tolist()
    parts = []
    for b, e in enumerate(of):
        x = send[off[b]:off[b + 1]]
        if x.shape[0]:
            a, u = (x @ w1[e].t()).float().chunk(2, 1)
            parts.append((torch.nn.functional.silu(a) * u).to(BF16) @ w2[e].t())
    parts.append(send[off[-1]:] * 0)  # the rows of masked slots
    return torch.cat(parts)


def train_step(layer, x, wg, w1, w2, target, alpha):
    """Loss of one step, and its balance part; gradients land in the leaves."""
    logits = x.float() @ wg.t()
    gate, balance = Route.apply(logits, layer, alpha)
    layer.make_plan()
    send = Dispatch.apply(x, layer)
    out = Combine.apply(experts_bf16(send, layer, w1, w2), gate, layer)
    loss = ((out.float() - target) ** 2).mean() + balance.sum()
    loss.backward()
    return float(loss.detach()), float(balance.detach())


class Int8Experts:
    """The experts' weights as 8-bit integers with a scale a channel."""

    def __init__(self, w1, w2):
        self.w = []
        for w in (w1, w2):
            n, N, K = w.shape
            q, s = torch.empty(n, N, K, dtype=torch.int8, device=DEV), torch.empty(n, N, device=DEV)
            uep.ultraep_quant_rows(w.detach().contiguous(), n * N, K, K, q, K, s)
            self.w.append((q, s, n, N, K))

    def product(self, i, x, layer, of, act):
        q, s, n, N, K = self.w[i]
        M = x.shape[0]
        xq, xs = torch.empty(M, K, dtype=torch.int8, device=DEV), torch.empty(M, device=DEV)
        y = torch.zeros(M, N // 2 if act else N, dtype=BF16, device=DEV)
        uep.ultraep_quant_rows(x, M, K, K, xq, K, xs)
        uep.ultraep_expert_matmul(xq, xs, M, q, s, n, N, K, layer.off, of, of.numel(), act, y, layer.status)
        return y


def serve(layer, x, wg, experts):
    m = layer
    m.route((x.float() @ wg.t()).contiguous())
    m.make_plan()
    send = torch.empty(m.T * m.k, m.H, dtype=BF16, device=DEV)
    uep.ultraep_dispatch_scatter(x, m.T, m.k, m.H, m.rows, m.off[-1:], send)
    of = m.block_experts()
    y = experts.product(1, experts.product(0, send, m, of, True), m, of, False)
    out = torch.empty(m.T, m.H, dtype=BF16, device=DEV)
    uep.ultraep_combine(y, m.T * m.k, m.gate, m.rows, m.T, m.k, m.H, out, m.status)
    return out


def plain_layer(x, wg, w1, w2, k, ids):
    """The layer's output by torch alone, for given ids, in fp32."""
    s = torch.softmax(x.float() @ wg.t(), 1)
    g = s.gather(1, ids)
    g = g / g.sum(1, keepdim=True)
    out = torch.zeros(x.shape, device=DEV)
    for j in range(k):
        for e in ids[:, j].unique().tolist():
            t = (ids[:, j] == e).nonzero()[:, 0]
            a, u = (x[t].float() @ w1[e].float().t()).chunk(2, 1)
            out = out.index_add(0, t, g[t, j, None] * ((torch.nn.functional.silu(a) * u) @ w2[e].float().t()))
    return out


def main(T=512, H=256, F=512, steps=30, verbose=True):
    """Returns (relative error of the training output, of the 8-bit output, balance
    losses, relative errors of the gradients by name)."""
    R, E, n_slot, k = 4, 16, 2, 2
    layer = Layer(R, E, n_slot, k, T, H, F)
    gen = layer.gen
    x = torch.randn(T, H, device=DEV, generator=gen).to(BF16)
    lead = torch.randn(1, H, device=DEV, generator=gen)
    x = (x.float() + 0.5 * lead).to(BF16)  # a common direction: the router begins unbalanced
    wg = (H ** -0.5 * torch.randn(E, H, device=DEV, generator=gen)).requires_grad_()
    w1 = (H ** -0.5 * torch.randn(E, 2 * F, H, device=DEV, generator=gen)).to(BF16).requires_grad_()
    w2 = (F ** -0.5 * torch.randn(E, H, F, device=DEV, generator=gen)).to(BF16).requires_grad_()
    target = torch.randn(T, H, device=DEV, generator=gen)

    def rel(a, b):
        return float((a.double() - b.double()).norm() / b.double().norm())

    # one step against torch's own gradients of the same function
    x.requires_grad_()
    alpha = 0.05
    train_step(layer, x, wg, w1, w2, target, alpha)
    layer.check()
    ids = layer.topk.long()
    leaves = dict(x=x, wg=wg, w1=w1, w2=w2)
    ours = {n: t.grad.clone() for n, t in leaves.items()}
    for t in leaves.values():
        t.grad = None
    out = plain_layer(x, wg, w1, w2, k, ids)
    p = torch.softmax(x.float() @ wg.t(), 1)
    share = torch.bincount(ids.reshape(-1), minlength=E).float() / (T * k)
    (((out - target) ** 2).mean() + alpha * E * (share * p.mean(0)).sum()).backward()
    grads = {n: rel(ours[n], t.grad) for n, t in leaves.items()}
    with torch.no_grad():
        out = plain_layer(x, wg, w1, w2, k, ids)
        send = Dispatch.apply(x.detach(), layer)
        bf16 = torch.empty(T, H, dtype=BF16, device=DEV)
        uep.ultraep_combine(experts_bf16(send, layer, w1, w2), T * k, layer.gate, layer.rows, T, k, H, bf16, layer.status)
        int8 = serve(layer, x.detach(), wg.detach(), Int8Experts(w1, w2))
    layer.check()
    x.requires_grad_(False)

    losses = []
    for _ in range(steps):  # the router's weights alone, with a heavy balance loss
        wg.grad = None
        losses.append(train_step(layer, x, wg, w1, w2, target, 1.0)[1])
        with torch.no_grad():
            wg -= 0.02 * wg.grad
    layer.check()
    errors = rel(bf16, out), rel(int8, out)
    if verbose:
        print(f"output against torch in fp32: bf16 experts {errors[0]:.2e}, 8-bit experts {errors[1]:.2e}")
        print("gradients against torch: " + ", ".join(f"{n} {v:.2e}" for n, v in grads.items()))
        print(f"balance loss over {steps} steps: {losses[0]:.3f} -> {losses[-1]:.3f} (1 is even)")
    return errors[0], errors[1], losses, grads


if __name__ == "__main__":
    main()
