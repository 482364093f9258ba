"""The example's recurrent student: its flat gradient against automatic differentiation in 64 bits, its steps with packed gradients, and
that it writes a character at a time what the whole text at once says."""
import math
import os
import sys

import pytest
import torch

import layers_reference as R

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def E():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import recurrent_student
    return recurrent_student


def norm(t, gamma, beta):
    return R.norm_forward(t, gamma, beta, float(torch.tensor(1e-5)))[0]


def reference(layout, weights, tokens, factors, lengths, resets):
    """The student's logits from formulas, in 64 bits on the CPU."""
    w = lambda name: layout.view(weights, name)
    dim = layout.dim
    b, n = tokens.shape
    there = (tokens >= 0) & (tokens < layout.vocab)
    e = torch.where(there[..., None], w("embedding")[torch.where(there, tokens, 0)], 0.0) * float(torch.tensor(dim ** 0.5)) * factors.view(b, n, dim)
    x, forget, out = (norm(e, w("gamma1"), w("beta1")) @ w("gates")).chunk(3, dim=2)
    a = torch.sigmoid(forget + w("forget"))
    h, rows = torch.zeros(b, dim, dtype=torch.float64), []
    for t in range(n):
        new = torch.where((resets[:, t] != 0)[:, None], 0.0, a[:, t] * h) + (1.0 - a[:, t]) * x[:, t]
        inside = (t < lengths)[:, None]
        h = torch.where(inside, new, h)
        rows.append(torch.where(inside, torch.sigmoid(out[:, t]) * new, 0.0))
    return norm(e + torch.stack(rows, dim=1), w("gamma2"), w("beta2")) @ w("out")


def loss_of(logits, teacher_tokens, teacher_logits, targets, tau, soft, hard):
    good = (teacher_tokens >= 0) & (teacher_tokens < logits.shape[-1])
    taught = good.any(dim=-1)
    t = torch.where(good, teacher_logits / tau, -1e300)
    p = torch.where(good, torch.softmax(t, dim=-1), 0.0)
    logq = torch.log_softmax(logits / tau, dim=-1).gather(-1, teacher_tokens.clamp(0, logits.shape[-1] - 1))
    kl = (p * (torch.log(torch.where(p > 0, p, 1.0)) - logq)).sum(dim=-1)
    told = targets >= 0
    ce = -torch.log_softmax(logits, dim=-1).gather(-1, targets.clamp(min=0)[..., None])[..., 0]
    return torch.where(taught, soft * tau ** 2 * kl, 0.0) + torch.where(told, hard * ce, 0.0)


@pytest.mark.parametrize("rate", [0.0, 0.2])
def test_flat_gradient_against_automatic_differentiation(E, rate):
    b, n, vocab, dim, top, step, seed = 3, 41, 19, 36, 4, 6, 78
    layout = E.Layout(vocab, dim)
    weights = E.initial_weights(layout, 3)
    g = torch.Generator().manual_seed(9)
    weights += torch.randn(layout.total, generator=g).mul_(0.1).to(E.DEV)   # betas that are not zeros
    tokens = torch.randint(0, vocab, (b, n), generator=g)
    tokens[0, 5] = -1
    targets = torch.randint(0, vocab, (b, n), generator=g)
    teacher_tokens, teacher_logits = torch.randint(0, vocab, (b, n, top), generator=g), torch.randn(b, n, top, generator=g) * 2
    teacher_tokens[1, 3] = torch.tensor([2, 2, 7, -1])
    lengths, resets = torch.tensor([41, 30, 17], dtype=torch.int32), torch.zeros(b, n, dtype=torch.uint8)
    resets[0, 20], resets[1, 0], resets[2, 16] = 1, 1, 1
    for i, end in enumerate(lengths.tolist()):   # padding counts for nothing
        targets[i, end:], teacher_tokens[i, end:] = -1, -1
    dloss = torch.rand(b, n, generator=g) / 50
    student = E.Student(layout, b, n, rate, seed)
    dev = lambda t: t.to(E.DEV)
    loss = student.forward(dev(tokens), weights, step, dev(teacher_tokens), dev(teacher_logits), dev(targets), dev(dloss), lengths=dev(lengths), resets=dev(resets))
    grad = torch.full_like(weights, float("nan"))
    student.backward(weights, grad, step)
    w64 = weights.cpu().double().requires_grad_()
    factors = R.factors(b * n, dim, rate, seed, step) if rate else torch.ones(b * n, dim, dtype=torch.float64)
    want = loss_of(reference(layout, w64, tokens, factors, lengths, resets), teacher_tokens, teacher_logits.double(), targets, E.TEMPERATURE, E.SOFT, E.HARD)
    (want * dloss.double()).sum().backward()
    # products of 36 to 108 terms, sums over 123 rows and a recurrence in 32 bits, one after another: some 1e-6 of each result's size
    close = lambda got, ref, what: (got.cpu().double() - ref).norm() <= 2e-5 * ref.norm() or pytest.fail(what)
    close(loss, want.detach(), "loss")
    for name in layout.parts:
        close(layout.view(grad, name), layout.view(w64.grad, name), name)


def test_steps_with_packed_gradients(E):
    losses, weights, layout = E.train(12)
    assert len(losses) == 12 and all(math.isfinite(v) for v in losses) and torch.isfinite(weights).all()
    assert not torch.equal(weights, E.initial_weights(layout, 1))


def test_writing_follows_the_whole_text(E):
    """Character by character with a state carried along, each character is the most likely one by the formula over all that came before (where the formula's two
    best are apart by more than float32 leaves uncertain)."""
    layout = E.Layout(23, 40)
    weights = E.initial_weights(layout, 4)
    start = torch.randint(0, 23, (4, 5), generator=torch.Generator().manual_seed(5))
    written = E.write(layout, weights, start.to(E.DEV), 30).cpu()
    text = torch.cat([start, written], dim=1)
    n = text.shape[1] - 1
    logits = reference(layout, weights.cpu().double(), text[:, :-1], torch.ones(4 * n, 40, dtype=torch.float64), torch.full((4,), n), torch.zeros(4, n))
    best = torch.topk(logits[:, start.shape[1] - 1:], 2, dim=2)
    clear = best.values[..., 0] - best.values[..., 1] > 1e-3
    assert clear.float().mean() > 0.9 and torch.equal(best.indices[..., 0][clear], written[clear])
