#!/usr/bin/env python3
"""A small recurrent student of characters trained by several simulated learners on one GPU, with every gradient packed by AdaComp.

The student is logits = norm(e + recurrence(norm(e) W)) V with e = dropout(scale * embedding of the characters); the product with W leaves the
recurrence's input, its forget gate and its output gate side by side.  A teacher says the logits of its top characters, and the text what came
next: the loss is a mixture of distillation and cross entropy.  The weights are one flat float32 buffer and the gradient of each learner another
one, laid out by one layer table.  Everything between the matrix products (embedding, norms, recurrence, loss) are the library's calls, and they write
the gradients of the embedding table, of gamma, beta and the forget gate's bias straight into the learner's flat gradient; the products' gradients
are written there by torch.  Then the learner's gradient is packed (adacomp_compress_batch), and the packets of all learners are summed and
applied with Adam (adacomp_unpack_update).  write() lets the student go on with a text, a character at a time.

The text: a random chain in which two characters decide the next one; the teacher knows its probabilities.

    python examples/recurrent_student.py [steps]
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1712_02679_amd as A  # noqa: E402

DEV = "cuda:0"
TEMPERATURE, SOFT, HARD = 2.0, 0.5, 0.5


class Layout:
    """Where each parameter lies in the flat buffers, and the layer table that says so."""

    def __init__(self, vocab, dim):
        self.vocab, self.dim = vocab, dim
        self.parts, self.table, at = {}, [], 0
        for name, shape, lt in (("embedding", (vocab, dim), 50), ("gates", (dim, 3 * dim), 500), ("out", (dim, vocab), 500), ("gamma1", (dim,), 50), ("beta1", (dim,), 50),
                                ("gamma2", (dim,), 50), ("beta2", (dim,), 50), ("forget", (dim,), 50)):
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


class Student:
    """Forward and backward pass over tokens [batch, length], with the buffers that a training loop keeps."""

    def __init__(self, layout, batch, length, rate, seed):
        self.layout, self.b, self.n, self.rate, self.seed = layout, batch, length, rate, seed
        dim, vocab, rows = layout.dim, layout.vocab, batch * length
        self.scale = dim ** 0.5
        new = lambda *s: torch.empty(*s, device=DEV)
        self.e, self.y1, self.r, self.z, self.y2, self.dy2, self.dz, self.dy1, self.de = (new(batch, length, dim) for _ in range(9))
        self.mean1, self.rstd1, self.mean2, self.rstd2, self.loss = (new(batch, length) for _ in range(5))
        self.dgates = new(batch, length, 3 * dim)
        self.states = new(batch, A.adacomp_recurrence_kept(length), dim)
        self.dlogits = new(batch, length, vocab)
        bytes_ = max(A.adacomp_norm_workspace_bytes(rows, dim), A.adacomp_embed_workspace_bytes(rows, vocab, dim), A.adacomp_recurrence_workspace_bytes(batch, length, dim))
        self.ws = torch.empty(bytes_, dtype=torch.uint8, device=DEV)   # one call after the other uses it

    def drop(self, step):
        return A.Dropout(self.rate, self.seed, step) if self.rate > 0 else None

    def forward(self, tokens, weights, step, teacher_tokens, teacher_logits, targets, dloss, lengths=None, resets=None):
        """The loss of every place; the gradient of the logits is made at the same time.  A target that is no character and top tokens that are none
        are places that count for nothing."""
        w = lambda name: self.layout.view(weights, name)
        dim = self.layout.dim
        self.tokens, self.lengths, self.resets = tokens, lengths, resets
        A.adacomp_embed_forward(tokens, w("embedding"), self.e, scale=self.scale, dropout=self.drop(step))
        A.adacomp_norm_forward(self.e, w("gamma1"), w("beta1"), self.y1, mean=self.mean1, rstd=self.rstd1)
        self.gates = torch.mm(self.y1.view(-1, dim), w("gates")).view(self.b, self.n, 3 * dim)
        x, forget, out = self.gates.chunk(3, dim=2)
        A.adacomp_recurrence_forward(x, forget, self.r, self.ws, out=out, bias=w("forget"), states=self.states, lengths=lengths, resets=resets)
        A.adacomp_norm_forward(self.r, w("gamma2"), w("beta2"), self.y2, residual=self.e, z=self.z, mean=self.mean2, rstd=self.rstd2)
        logits = torch.mm(self.y2.view(-1, dim), w("out"))
        A.adacomp_distill_forward(logits, self.loss, teacher_tokens=teacher_tokens, teacher_logits=teacher_logits, targets=targets, temperature=TEMPERATURE, soft=SOFT,
                                  hard=HARD, dlogits=self.dlogits.view_as(logits), dloss=dloss)
        return self.loss

    def backward(self, weights, grad, step):
        """Every parameter's gradient, into the flat gradient."""
        w = lambda name: self.layout.view(weights, name)
        g = lambda name: self.layout.view(grad, name)
        dim = self.layout.dim
        flat = lambda t: t.view(-1, t.shape[-1])
        torch.mm(flat(self.y2).t(), flat(self.dlogits), out=g("out"))
        torch.mm(flat(self.dlogits), w("out").t(), out=flat(self.dy2))
        A.adacomp_norm_backward(self.dy2, self.z, self.mean2, self.rstd2, w("gamma2"), self.dz, g("gamma2"), g("beta2"), self.ws)
        x, forget, out = self.gates.chunk(3, dim=2)
        dx, dforget, dout = self.dgates.chunk(3, dim=2)
        A.adacomp_recurrence_backward(self.dz, x, forget, self.states, dx, dforget, self.ws, out=out, dout=dout, bias=w("forget"), dbias=g("forget"), lengths=self.lengths,
                                      resets=self.resets)
        torch.mm(flat(self.y1).t(), flat(self.dgates), out=g("gates"))
        torch.mm(flat(self.dgates), w("gates").t(), out=flat(self.dy1))
        A.adacomp_norm_backward(self.dy1, self.e, self.mean1, self.rstd1, w("gamma1"), self.de, g("gamma1"), g("beta1"), self.ws, dz_add=self.dz)
        A.adacomp_embed_backward(self.tokens, self.de, g("embedding"), self.ws, scale=self.scale, dropout=self.drop(step))


def write(layout, weights, tokens, count):
    """The student's most likely way to go on with each of some texts, tokens [batch, length]: what is written, [batch, count]."""
    w = lambda name: layout.view(weights, name)
    b, dim = tokens.shape[0], layout.dim
    state = torch.zeros(b, dim, device=DEV)
    new = lambda: torch.empty(b, 1, dim, device=DEV)
    e, y1, r, y2 = new(), new(), new(), new()
    ws = torch.empty(A.adacomp_recurrence_workspace_bytes(b, 1, dim), dtype=torch.uint8, device=DEV)
    out, token = [], tokens[:, :1].contiguous()
    for i in range(tokens.shape[1] + count - 1):
        A.adacomp_embed_forward(token, w("embedding"), e, scale=dim ** 0.5)
        A.adacomp_norm_forward(e, w("gamma1"), w("beta1"), y1)
        x, forget, gate = torch.mm(y1.view(b, dim), w("gates")).view(b, 1, 3 * dim).chunk(3, dim=2)
        A.adacomp_recurrence_forward(x, forget, r, ws, out=gate, bias=w("forget"), first=state, last=state)
        A.adacomp_norm_forward(r, w("gamma2"), w("beta2"), y2, residual=e)
        token = torch.mm(y2.view(b, dim), w("out")).argmax(dim=1, keepdim=True)
        if i + 1 < tokens.shape[1]:
            token = tokens[:, i + 1:i + 2].contiguous()
        else:
            out.append(token)
    return torch.cat(out, dim=1)


def initial_weights(layout, seed):
    g = torch.Generator().manual_seed(seed)
    weights = torch.zeros(layout.total)
    layout.view(weights, "embedding").normal_(generator=g).mul_(layout.dim ** -0.5)
    layout.view(weights, "gates").normal_(generator=g).mul_(layout.dim ** -0.5)
    layout.view(weights, "out").normal_(generator=g).mul_(layout.dim ** -0.5)
    layout.view(weights, "gamma1").fill_(1.0)
    layout.view(weights, "gamma2").fill_(1.0)
    layout.view(weights, "forget").uniform_(-1.0, 3.0, generator=g)
    return weights.to(DEV)


class Text:
    """A chain in which two characters decide the probabilities of the next one."""

    def __init__(self, vocab, seed):
        g = torch.Generator(device=DEV).manual_seed(seed)
        self.vocab, self.logits = vocab, torch.randn(vocab, vocab, vocab, generator=g, device=DEV) * 3.0

    def batch(self, batch, length, top, seed):
        """(tokens, targets, the teacher's top tokens and their logits)"""
        g = torch.Generator(device=DEV).manual_seed(seed)
        text = torch.randint(0, self.vocab, (batch, length + 1), generator=g, device=DEV)
        for i in range(2, length + 1):
            text[:, i] = torch.multinomial(torch.softmax(self.logits[text[:, i - 2], text[:, i - 1]], dim=1), 1, generator=g)[:, 0]
        best = torch.topk(self.logits[text[:, :-2], text[:, 1:-1]], top, dim=2)
        tokens, targets = text[:, :-1].contiguous(), text[:, 1:].clone()
        teacher_tokens, teacher_logits = torch.full((batch, length, top), -1, device=DEV), torch.zeros(batch, length, top, device=DEV)
        teacher_tokens[:, 1:], teacher_logits[:, 1:] = best.indices, best.values   # nobody can know what follows the first one
        targets[:, 0] = -1
        return tokens, targets, teacher_tokens, teacher_logits


def train(steps, learners=2, batch=8, length=48, vocab=20, dim=64, top=5, rate=0.05, lr=3e-3, seed=1):
    """(the learners' mean losses, step by step; weights; layout)"""
    layout, text = Layout(vocab, dim), Text(vocab, seed)
    weights = initial_weights(layout, seed)
    m, v = torch.zeros_like(weights), torch.zeros_like(weights)
    students = [Student(layout, batch, length, rate, seed * 1000 + k) for k in range(learners)]
    grads = [torch.zeros_like(weights) for _ in range(learners)]
    residues = [torch.zeros_like(weights) for _ in range(learners)]
    packets = [torch.zeros(A.adacomp_packet_bound(layout.table), dtype=torch.uint8, device=DEV) for _ in range(learners)]
    ws = torch.zeros(A.adacomp_workspace_bytes_batch(layout.table, learners), dtype=torch.uint8, device=DEV)
    A.adacomp_workspace_init(layout.table, ws)
    dloss = torch.full((batch, length), 1.0 / (batch * (length - 1)), device=DEV)
    losses = []
    for step in range(1, steps + 1):
        total = 0.0
        for k, student in enumerate(students):
            tokens, targets, teacher_tokens, teacher_logits = text.batch(batch, length, top, (seed * 100003 + step) * 64 + k)
            total = total + (student.forward(tokens, weights, step, teacher_tokens, teacher_logits, targets, dloss) * dloss).sum()
            student.backward(weights, grads[k], step)
        A.adacomp_compress_batch(layout.table, grads, residues, packets, ws)
        A.adacomp_unpack_update(layout.table, packets, None, weights, m, v, ws, A.OPT_ADAM, lr, bias1=1.0 - 0.9 ** step, bias2=1.0 - 0.999 ** step)
        losses.append(total / learners)
    A.adacomp_workspace_release(ws)
    return torch.stack(losses).tolist(), weights, layout


if __name__ == "__main__":
    n = int(sys.argv[1]) if len(sys.argv) > 1 else 300
    losses, weights, layout = train(n)
    for i, loss in enumerate(losses):
        if i % max(1, n // 12) == 0 or i == n - 1:
            print(f"step {i + 1:5d}  loss {loss:.4f}")
    start = torch.tensor([[1, 2, 3]], device=DEV)
    print("after 1 2 3:", *write(layout, weights, start, 12)[0].tolist())
