"""The example's attention block: its flat gradient against automatic differentiation in 64 bits, and that its learners learn
through packed gradients."""
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
    import attention_block
    return attention_block


def reference(E, layout, weights, x, dims, rate, seed, step):
    """The block's output from formulas, in 64 bits on the CPU, with the generator's masks."""
    b, n, dim, heads = dims
    w = lambda name: layout.view(weights, name)

    def norm(t, gamma, beta):
        return R.norm_forward(t, gamma, beta, float(torch.tensor(1e-5)))[0]

    q, k, v = (t.reshape(b, n, heads, -1).transpose(1, 2) for t in (norm(x, w("gamma1"), w("beta1")) @ w("qkv")).chunk(3, dim=1))
    far = E.DISTANCE
    import paper_1712_02679_amd as A
    bucket = torch.from_numpy(A.adacomp_relative_buckets(E.BUCKETS, far, False)).long()[R.places(1, n, n, 0).clamp(-far, far) + far]
    t = q @ k.transpose(2, 3) * (dim // heads) ** -0.5 + w("bias")[bucket].permute(0, 3, 1, 2)
    t = t.masked_fill(R.places(1, n, n, 0)[:, None] > 0, -math.inf)
    f0 = R.factors(b * heads * n, n, rate, seed, 4 * step).view(b, heads, n, n) if rate else 1.0
    f1 = R.factors(b * n, dim, rate, seed, 4 * step + 1) if rate else 1.0
    mixed = ((torch.softmax(t, -1) * f0) @ v).transpose(1, 2).reshape(b * n, dim)
    return norm(x + f1 * (mixed @ w("out")), w("gamma2"), w("beta2"))


@pytest.mark.parametrize("rate", [0.0, 0.2])
def test_flat_gradient_against_automatic_differentiation(E, rate):
    b, n, dim, heads, step, seed = 3, 37, 48, 3, 5, 77
    layout = E.Layout(dim, heads)
    weights = E.initial_weights(layout, dim, 3)
    g = torch.Generator().manual_seed(9)
    weights += torch.randn(layout.total, generator=g).mul_(0.1).to(E.DEV)   # a bias and betas that are not zeros
    x, C = torch.randn(b * n, dim, generator=g), torch.randn(b * n, dim, generator=g)
    block = E.Block(layout, b, n, dim, heads, rate, seed)
    y = block.forward(x.to(E.DEV), weights, step)
    grad = torch.full_like(weights, float("nan"))
    dx = block.backward(C.to(E.DEV), weights, grad, step)
    w64, x64 = weights.cpu().double().requires_grad_(), x.double().requires_grad_()
    want = reference(E, layout, w64, x64, (b, n, dim, heads), rate, seed, step)
    (want * C.double()).sum().backward()
    # products of 48 to 144 terms and sums over 111 rows in 32 bits, one after another: some 1e-6 of each result's size
    close = lambda got, ref, what: (got.cpu().double() - ref).norm() <= 2e-5 * ref.norm() or pytest.fail(what)
    close(y, want.detach(), "y")
    close(dx, x64.grad, "dx")
    for name in layout.parts:
        close(layout.view(grad, name), layout.view(w64.grad, name), name)


def test_learners_learn_through_packed_gradients(E):
    losses = E.train(150)
    assert all(math.isfinite(v) for v in losses)
    first, last = sum(losses[:5]) / 5, sum(losses[-5:]) / 5
    assert last < 0.8 * first, (first, last)
