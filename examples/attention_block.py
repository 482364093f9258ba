#!/usr/bin/env python3
"""A small attention block trained by several simulated learners on one GPU, with every gradient packed by AdaComp.

The block is y = norm(x + dropout(attention(norm(x)))), its attention biased by learned buckets of relative position.  The weights
are one flat float32 buffer and the gradient of each learner another one, laid out by one layer table.  What stands between the
matrix products (dropout, both norms, the biased softmax) are the library's calls, and they write the gradients of gamma, beta and
the bias table straight into the learner's flat gradient; the products' gradients are written there by torch.  Then the learner's
gradient is packed (adacomp_compress_batch), and the packets of all learners are summed and applied with Adam
(adacomp_unpack_update).

The task: say what the token before said.  Only the bias can tell a head which one that is.

    python examples/attention_block.py [steps]
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1712_02679_amd as A  # noqa: E402

DEV = "cuda:0"
BUCKETS, DISTANCE = 16, 32


class Layout:
    """Where each parameter lies in the flat buffers, and the layer table that says so."""

    def __init__(self, dim, heads):
        self.parts, self.table, at = {}, [], 0
        for name, shape, lt in (("qkv", (dim, 3 * dim), 500), ("out", (dim, dim), 500), ("gamma1", (dim,), 50), ("beta1", (dim,), 50), ("gamma2", (dim,), 50),
                                ("beta2", (dim,), 50), ("bias", (BUCKETS, heads), 50)):
            n = 1
            for s in shape:
                n *= s
            self.parts[name] = (at, n, shape)
            self.table.append((at, n, lt))
            at += (n + 3) // 4 * 4
        self.total = at

    def view(self, flat, name):
        at, n, shape = self.parts[name]
        return flat[at:at + n].view(shape)


class Block:
    """The block's forward and backward pass over [batch, length, dim], with the buffers that a training loop keeps."""

    def __init__(self, layout, batch, length, dim, heads, rate, seed):
        self.layout, self.b, self.n, self.dim, self.heads, self.rate, self.seed = layout, batch, length, dim, heads, rate, seed
        self.scale = (dim // heads) ** -0.5
        self.map = torch.from_numpy(A.adacomp_relative_buckets(BUCKETS, DISTANCE, False)).to(DEV)
        rows = batch * length
        new = lambda *s: torch.empty(*s, device=DEV)
        self.y1, self.z, self.y, self.dz, self.dx, self.dy1, self.dx0 = (new(rows, dim) for _ in range(7))
        self.mean1, self.rstd1, self.mean2, self.rstd2 = (new(rows) for _ in range(4))
        self.probs, self.dscores = new(batch, heads, length, length), new(batch, heads, length, length)
        self.lse = new(batch, heads, length)
        self.norm_ws = torch.empty(A.adacomp_norm_workspace_bytes(rows, dim), dtype=torch.uint8, device=DEV)
        self.soft_ws = torch.empty(A.adacomp_bias_softmax_workspace_bytes(batch, heads, length, length, DISTANCE), dtype=torch.uint8, device=DEV)

    def drop(self, which, step):
        """The mask of a place and step: the same in the forward and the backward pass, another one everywhere else."""
        return A.Dropout(self.rate, self.seed, 4 * step + which) if self.rate > 0 else None

    def split(self, t):
        return t.view(self.b, self.n, self.heads, -1).transpose(1, 2).reshape(self.b * self.heads, self.n, -1)

    def join(self, t):
        return t.view(self.b, self.heads, self.n, -1).transpose(1, 2).reshape(self.b * self.n, -1)

    def forward(self, x, weights, step):
        w = lambda name: self.layout.view(weights, name)
        self.x = x
        A.adacomp_norm_forward(x, w("gamma1"), w("beta1"), self.y1, mean=self.mean1, rstd=self.rstd1)
        self.q, self.k, self.v = (self.split(t.contiguous()) for t in torch.mm(self.y1, w("qkv")).chunk(3, dim=1))
        self.scores = torch.bmm(self.q, self.k.transpose(1, 2).contiguous()).view(self.b, self.heads, self.n, self.n)
        self.bias = A.RelativeBias(w("bias"), self.map)
        A.adacomp_bias_softmax_forward(self.scores, self.bias, self.probs, self.soft_ws, lse=self.lse, scale=self.scale, causal=True, dropout=self.drop(0, step))
        self.mixed = self.join(torch.bmm(self.probs.view(-1, self.n, self.n), self.v))
        A.adacomp_norm_forward(torch.mm(self.mixed, w("out")), w("gamma2"), w("beta2"), self.y, residual=x, dropout=self.drop(1, step), z=self.z,
                               mean=self.mean2, rstd=self.rstd2)
        return self.y

    def backward(self, dy, weights, grad, step):
        """Every parameter's gradient, into the flat gradient; the gradient of x is returned."""
        w = lambda name: self.layout.view(weights, name)
        g = lambda name: self.layout.view(grad, name)
        # without dropout the gradient of what it would have dropped is dz itself
        drop = self.drop(1, step)
        A.adacomp_norm_backward(dy, self.z, self.mean2, self.rstd2, w("gamma2"), self.dz, g("gamma2"), g("beta2"), self.norm_ws, dropout=drop,
                                dx=self.dx if drop else None)
        dx = self.dx if drop else self.dz
        torch.mm(self.mixed.t(), dx, out=g("out"))
        dmixed = self.split(torch.mm(dx, w("out").t()))
        dprobs = torch.bmm(dmixed, self.v.transpose(1, 2).contiguous()).view_as(self.scores)
        dv = torch.bmm(self.probs.view(-1, self.n, self.n).transpose(1, 2).contiguous(), dmixed)
        A.adacomp_bias_softmax_backward(self.scores, self.bias, self.lse, dprobs, self.dscores, g("bias"), self.soft_ws, scale=self.scale, causal=True,
                                        dropout=self.drop(0, step))
        ds = self.dscores.view(-1, self.n, self.n)
        dqkv = torch.cat([self.join(t) for t in (torch.bmm(ds, self.k), torch.bmm(ds.transpose(1, 2).contiguous(), self.q), dv)], dim=1)
        torch.mm(self.y1.t(), dqkv, out=g("qkv"))
        torch.mm(dqkv, w("qkv").t(), out=self.dy1)
        A.adacomp_norm_backward(self.dy1, self.x, self.mean1, self.rstd1, w("gamma1"), self.dx0, g("gamma1"), g("beta1"), self.norm_ws, dz_add=self.dz)
        return self.dx0


def initial_weights(layout, dim, seed):
    g = torch.Generator().manual_seed(seed)
    weights = torch.zeros(layout.total)
    layout.view(weights, "qkv").normal_(generator=g).mul_(dim ** -0.5)
    layout.view(weights, "out").normal_(generator=g).mul_(dim ** -0.5)
    layout.view(weights, "gamma1").fill_(1.0)
    layout.view(weights, "gamma2").fill_(1.0)
    return weights.to(DEV)


def batch_of(batch, length, dim, seed):
    """(x, target): tokens, and for each the one before it (the first one says itself)."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.randn(batch, length, dim, generator=g, device=DEV)
    return x.reshape(-1, dim), torch.cat([x[:, :1], x[:, :-1]], dim=1).reshape(-1, dim)


def train(steps, learners=2, batch=8, length=48, dim=64, heads=4, rate=0.1, lr=3e-3, seed=1):
    """The learners' mean losses, step by step."""
    layout = Layout(dim, heads)
    weights = initial_weights(layout, dim, seed)
    m, v = torch.zeros_like(weights), torch.zeros_like(weights)
    blocks = [Block(layout, batch, length, dim, heads, rate, seed * 1000 + k) for k in range(learners)]
    grads = [torch.zeros_like(weights) for _ in range(learners)]
    residues = [torch.zeros_like(weights) for _ in range(learners)]
    packets = [torch.zeros(A.adacomp_packet_bound(layout.table), dtype=torch.uint8, device=DEV) for _ in range(learners)]
    ws = torch.zeros(A.adacomp_workspace_bytes_batch(layout.table, learners), dtype=torch.uint8, device=DEV)
    A.adacomp_workspace_init(layout.table, ws)
    losses = []
    for step in range(1, steps + 1):
        total = 0.0
        for k, block in enumerate(blocks):
            x, target = batch_of(batch, length, dim, (seed * 100003 + step) * 64 + k)
            off = block.forward(x, weights, step) - target
            total = total + off.square().mean()
            block.backward(off * (2.0 / off.numel()), weights, grads[k], step)
        A.adacomp_compress_batch(layout.table, grads, residues, packets, ws)
        A.adacomp_unpack_update(layout.table, packets, None, weights, m, v, ws, A.OPT_ADAM, lr, bias1=1.0 - 0.9 ** step, bias2=1.0 - 0.999 ** step)
        losses.append(total / learners)
    A.adacomp_workspace_release(ws)
    return torch.stack(losses).tolist()


if __name__ == "__main__":
    n = int(sys.argv[1]) if len(sys.argv) > 1 else 600
    for i, loss in enumerate(train(n)):
        if i % max(1, n // 12) == 0 or i == n - 1:
            print(f"step {i + 1:5d}  loss {loss:.4f}")
