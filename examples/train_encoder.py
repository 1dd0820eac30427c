"""A small encoder trained by two simulated workers that exchange sparsified gradients.

    python examples/train_encoder.py [--steps 200]

Everything between the matrix products of a layer is one of this library's operators:
attention over a padded batch with dropout (okt_attention_forward / _backward), and
dropout, the sum with the residual stream and the norm after it in one call
(okt_residual_norm_forward / _backward), and the dropout of the embeddings (okt_dropout).
The gradients of all parameters land in one flat fp32 vector: the norms' are written there by
the operator, the products' are added there by autograd.  Each worker accumulates the vector into
its residual and selects its top-k entries (okt_accumulate_topk_select), and the reduced entries
(okt_sparse_reduce) update the weights.

The task is synthetic: a third of a sequence's tokens are one and the same, and every position has
to name it, which takes attention.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2201_07598_amd as okt  # noqa: E402

DEV = "cuda:0"
WORKERS, BATCH, LENGTH, VOCAB = 2, 16, 96, 32
LAYERS, WIDTH, HEADS, INNER, DROP = 2, 128, 2, 256, 0.05
DENSITY, RATE = 0.05, 0.3


class Dropout(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, seed, site, p):
        ctx.rest = (seed, site, p)
        y = torch.empty_like(x)
        okt.okt_dropout(x, y, p, seed, site)
        return y

    @staticmethod
    def backward(ctx, dy):
        seed, site, p = ctx.rest
        dy = dy.contiguous()
        dx = torch.empty_like(dy)
        okt.okt_dropout(dy, dx, p, seed, site)           # the same mask, drawn again
        return dx, None, None, None


class Attention(torch.autograd.Function):
    """[batch, length, 3 heads, dim] of queries, keys and values to [batch, length, heads, dim]."""

    @staticmethod
    def forward(ctx, qkv, lens, seed, site, p):
        heads = qkv.shape[2] // 3
        q, k, v = qkv.split(heads, 2)
        o = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        lse = torch.empty(q.shape[0], heads, q.shape[1], device=q.device)
        ws = torch.empty(okt.okt_attention_workspace_bytes(q.shape[0], heads, heads, q.shape[1], q.shape[1], q.shape[3]),
                         dtype=torch.uint8, device=q.device)
        okt.okt_attention_forward(q, k, v, o, lse, ws, q_lens=lens, k_lens=lens, dropout_p=p, seed=seed, site=site)
        ctx.save_for_backward(qkv, o, lse)
        ctx.rest = (lens, seed, site, p, ws)
        return o

    @staticmethod
    def backward(ctx, do):
        qkv, o, lse = ctx.saved_tensors
        lens, seed, site, p, ws = ctx.rest
        heads = o.shape[2]
        dqkv = torch.empty_like(qkv)                     # the three gradients, as the projection wants them
        okt.okt_attention_backward(*qkv.split(heads, 2), o, lse, do.contiguous(), *dqkv.split(heads, 2), ws,
                                   q_lens=lens, k_lens=lens, dropout_p=p, seed=seed, site=site)
        return dqkv, None, None, None, None


class SumNorm(torch.autograd.Function):
    """norm(x + dropout(u)) on [rows, width].  The gradients of weight and bias are written where `weight.grad` and
    `bias.grad` lie, in the flat vector, by the call itself; the graph hands on nothing for them."""

    @staticmethod
    def forward(ctx, u, x, weight, bias, seed, site, p):
        h, y = torch.empty_like(x), torch.empty_like(x)
        stats = torch.empty(x.shape[0], 4, device=x.device)
        okt.okt_residual_norm_forward(u, x, h, y, stats, pre_weight=weight, pre_bias=bias, dropout_p=p, seed=seed, site=site)
        ctx.save_for_backward(u, h, stats, weight, bias)
        ctx.rest = (weight.grad, bias.grad, seed, site, p)
        return y

    @staticmethod
    def backward(ctx, dy):
        u, h, stats, weight, bias = ctx.saved_tensors
        dw, db, seed, site, p = ctx.rest
        dx, du = torch.empty_like(h), torch.empty_like(h)
        ws = torch.empty(okt.okt_residual_norm_workspace_bytes(*h.shape), dtype=torch.uint8, device=h.device)
        okt.okt_residual_norm_backward(u, h, stats, None, dy.contiguous(), dx, du, ws, dpre_weight=dw, dpre_bias=db,
                                       pre_weight=weight, pre_bias=bias, dropout_p=p, seed=seed, site=site)
        return du, dx, None, None, None, None, None


class Encoder:
    """Parameters are views of one flat fp32 vector, their gradients of another."""

    def __init__(self):
        shapes = {"embed": (VOCAB, WIDTH), "place": (LENGTH, WIDTH), "out": (VOCAB, WIDTH)}
        for n in range(LAYERS):
            shapes |= {f"{n}.qkv": (3 * WIDTH, WIDTH), f"{n}.proj": (WIDTH, WIDTH), f"{n}.up": (INNER, WIDTH),
                       f"{n}.down": (WIDTH, INNER)}
            shapes |= {f"{n}.{norm}_{part}": (WIDTH,) for norm in ("mid", "end") for part in ("weight", "bias")}
        sizes = {k: -(-torch.Size(s).numel() // 4) * 4 for k, s in shapes.items()}       # 16-byte steps
        self.flat = torch.zeros(sum(sizes.values()), device=DEV)
        self.grad = torch.zeros_like(self.flat)
        self.par, at = {}, 0
        gen = torch.Generator().manual_seed(1)
        for name, shape in shapes.items():
            n = torch.Size(shape).numel()
            view = self.flat[at:at + n].view(shape)
            if name.endswith("weight"):
                view.fill_(1.0)
            elif not name.endswith("bias"):
                view.copy_(torch.randn(shape, generator=gen) * (0.5 if name in ("embed", "place") else WIDTH ** -0.5))
            self.par[name] = view.requires_grad_()
            self.par[name].grad = self.grad[at:at + n].view(shape)
            at += sizes[name]

    def loss(self, tokens, names, lens, seed):
        par = self.par
        rows = tokens.numel()

        def linear(x, name):
            return x @ par[name].to(torch.bfloat16).t()

        x = (par["embed"][tokens] + par["place"]).to(torch.bfloat16).view(rows, WIDTH)
        x = Dropout.apply(x, seed, 100, DROP)
        for n in range(LAYERS):
            qkv = linear(x, f"{n}.qkv").view(*tokens.shape, 3 * HEADS, WIDTH // HEADS)
            o = Attention.apply(qkv, lens, seed, 4 * n, DROP).reshape(rows, WIDTH)
            x = SumNorm.apply(linear(o, f"{n}.proj"), x, par[f"{n}.mid_weight"], par[f"{n}.mid_bias"], seed, 4 * n + 1, DROP)
            inner = torch.relu(linear(x, f"{n}.up"))
            x = SumNorm.apply(linear(inner, f"{n}.down"), x, par[f"{n}.end_weight"], par[f"{n}.end_bias"], seed, 4 * n + 2, DROP)
        scores = linear(x, "out").float().view(*tokens.shape, VOCAB)
        counts = torch.arange(tokens.shape[1], device=DEV)[None] < lens[:, None]
        each = torch.nn.functional.cross_entropy(scores.transpose(1, 2), names[:, None].expand_as(tokens), reduction="none")
        return (each * counts).sum() / counts.sum()


class Worker:
    """One data-parallel worker's residual and selection."""

    def __init__(self, number, n):
        self.gen = torch.Generator(device=DEV).manual_seed(100 + number)
        self.seed = torch.tensor([1 << 40 | number], dtype=torch.int64, device=DEV)
        self.k = int(n * DENSITY)
        self.residual = torch.zeros(n, device=DEV)
        self.threshold, self.count = torch.zeros(1, device=DEV), torch.zeros(1, dtype=torch.int64, device=DEV)
        self.idx = torch.zeros(2 * self.k, dtype=torch.int32, device=DEV)
        self.val = torch.zeros(2 * self.k, device=DEV)
        self.nnz = torch.zeros(2, dtype=torch.int64, device=DEV)
        self.ws = torch.empty(okt.okt_workspace_bytes(n, WORKERS), dtype=torch.uint8, device=DEV)

    def step(self, model):
        """Loss of this worker's batch; its top-k entries are left in idx and val."""
        names = torch.randint(VOCAB, (BATCH,), generator=self.gen, device=DEV)
        tokens = torch.randint(VOCAB, (BATCH, LENGTH), generator=self.gen, device=DEV)
        said = torch.rand(BATCH, LENGTH, generator=self.gen, device=DEV) < 1 / 3
        tokens = torch.where(said, names[:, None], tokens)
        lens = torch.randint(LENGTH // 3, LENGTH + 1, (BATCH,), generator=self.gen, device=DEV).to(torch.int32)
        model.grad.zero_()
        loss = model.loss(tokens, names, lens, self.seed)
        loss.backward()
        okt.okt_accumulate_topk_select(model.grad, self.residual, RATE / WORKERS, self.k, self.threshold, self.count,
                                       self.idx, self.val, self.nnz, self.ws)
        self.seed += 1 << 20                              # another mask for the next step
        return loss.detach()


def train(steps, report=None):
    """Losses of every step, averaged over the workers."""
    model = Encoder()
    n = model.flat.numel()
    workers = [Worker(i, n) for i in range(WORKERS)]
    capacity = sum(2 * w.k for w in workers)
    red_idx, red_val = torch.zeros(capacity, dtype=torch.int32, device=DEV), torch.zeros(capacity, device=DEV)
    red_nnz = torch.zeros(2, dtype=torch.int64, device=DEV)
    update = torch.zeros(n, device=DEV)
    losses = []
    for step in range(steps):
        losses.append(torch.stack([w.step(model) for w in workers]).mean())
        kept = [int(w.nnz[0]) for w in workers]           # what an exchange would learn from its peers
        idx = torch.cat([w.idx[:c] for w, c in zip(workers, kept)])
        val = torch.cat([w.val[:c] for w, c in zip(workers, kept)])
        off = torch.tensor([0, *torch.tensor(kept).cumsum(0).tolist()], dtype=torch.int64).to(DEV)
        okt.okt_sparse_reduce(idx, val, off, 0, n, red_idx, red_val, red_nnz, workers[0].ws, dense_out=update)
        model.flat.detach().sub_(update)
        if report and (step % report == 0 or step == steps - 1):
            print(f"step {step:4d}  loss {float(losses[-1]):.4f}  entries {sum(kept)} of {n}", flush=True)
    return [float(x) for x in losses]


if __name__ == "__main__":
    args = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    args.add_argument("--steps", type=int, default=200)
    train(args.parse_args().steps, report=20)
