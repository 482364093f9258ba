"""The biased softmax where scores are infinities or the ends of their type: rows whose waves or parts have nothing but -infinity beside
others far below zero."""
import pytest
import torch

import layers_reference as R
from layers_reference import DEEP, HALF_STEP, TINY, U, within

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16, torch.float16]
KEYS = [40, 700, 2048, 3000, 5000, 9000, 20000, 40000]   # one wave to a row, several, cut rows


@pytest.fixture(scope="module")
def A():
    import paper_1712_02679_amd as A
    return A


def call(A, rows, dtype, scale, seed=1):
    """Scores [1, 1, rows, keys] with their gradients of the probabilities, and the forward and backward call on them, without bias."""
    keys = rows.shape[-1]
    scores = rows.to(dtype).view(1, 1, -1, keys).to(DEV)
    g = torch.Generator().manual_seed(seed)
    up = torch.randn(scores.shape, generator=g).to(dtype).to(DEV)
    bias = A.RelativeBias(torch.zeros(32, 1, device=DEV), torch.from_numpy(A.adacomp_relative_buckets(32, 128, True)).to(DEV))
    ws = torch.empty(A.adacomp_bias_softmax_workspace_bytes(1, 1, rows.shape[0], keys, 128), dtype=torch.uint8, device=DEV)
    probs, ds, lse = torch.empty_like(scores), torch.empty_like(scores), torch.empty(scores.shape[:3], device=DEV)
    A.adacomp_bias_softmax_forward(scores, bias, probs, ws, lse=lse, scale=scale)
    A.adacomp_bias_softmax_backward(scores, bias, lse, up, ds, None, ws, scale=scale)
    return scores.cpu().double()[0, 0], up.cpu().double()[0, 0], probs.cpu()[0, 0], lse.cpu()[0, 0], ds.cpu()[0, 0]


def check_gradient(got, s, up, lse, scale, dtype, rows, exact):
    """dscores of some rows from the lse that the call was given; exact: the rows' exponents have no rounding."""
    p = torch.exp(s[rows] * scale - lse.double()[rows][:, None])
    e = p * (up[rows] - (p * up[rows]).sum(-1, keepdim=True))
    size = 0.0 if exact else (torch.where(torch.isinf(s[rows]), 0.0, s[rows].abs() * scale).amax(-1, keepdim=True) + lse.double()[rows].abs()[:, None])
    bound = p * (2 * U * (8 * size + DEEP) + DEEP * U) * (up[rows].abs() + (p * up[rows].abs()).sum(-1, keepdim=True))
    want = scale * e
    within(got[rows], want, HALF_STEP[dtype] * 1.01 * want.abs() + 2 * scale * bound + TINY[dtype], ("dscores", rows))


@pytest.mark.parametrize("keys", KEYS)
@pytest.mark.parametrize("dtype", TYPES)
def test_stretches_of_minus_infinity_beside_low_scores(A, keys, dtype):
    """Scores of -infinity have a probability of zero, however low the others of the row are, and a row's NaN reaches all of it."""
    scale, low, inf = float(torch.tensor(0.3)), -400.0, float("inf")   # exp(120) is beyond float32
    rows = torch.full((7, keys), -inf)
    g = torch.Generator().manual_seed(keys)
    rows[0, -1] = low
    rows[1, -8:] = torch.finfo(dtype).min
    rows[2, keys // 2:] = low + torch.randn(keys - keys // 2, generator=g)
    rows[4] = torch.randn(keys, generator=g)
    rows[5, -1], rows[5, 1] = low, float("nan")
    rows[6, :9] = low
    s, up, probs, lse, ds = call(A, rows, dtype, scale)
    want = torch.zeros(keys, dtype=dtype)
    want[-1] = 1.0
    assert torch.equal(probs[0], want)
    want[-8:] = 0.125                       # differences of equal numbers are zeros, and the sum is exact
    assert torch.equal(probs[1], want)
    assert torch.all(probs[3] == 0) and lse[3] == -inf
    assert torch.isnan(probs[5]).all() and torch.isnan(lse[5])
    for i in (2, 4, 6):
        p, exact_lse = R.softmax_forward(s[i] * scale)
        size = torch.where(torch.isinf(s[i]), 0.0, s[i].abs() * scale).max() + exact_lse.abs()
        rho = U * (8 * size + DEEP)
        within(probs[i], p, p * (HALF_STEP[dtype] * 1.01 + 2 * rho) + TINY[dtype], ("probs", i))
        within(lse[i], exact_lse, rho, ("lse", i))
        assert torch.all(probs[i][torch.isinf(s[i])] == 0)
    check_gradient(ds, s, up, lse, scale, dtype, [0, 2, 4, 6], False)
    assert torch.all(ds[3] == 0) and torch.all(ds[1, :-8] == 0)


@pytest.mark.parametrize("keys", KEYS)
@pytest.mark.parametrize("dtype", TYPES)
def test_finite_scores_at_the_ends_of_their_type_count(A, keys, dtype):
    """At scale 1 every finite score is a finite exponent: a row of the type's lowest value is even, not empty, its largest value takes all."""
    inf, low, high = float("inf"), torch.finfo(dtype).min, torch.finfo(dtype).max
    g = torch.Generator().manual_seed(keys)
    rows = torch.randn(6, keys, generator=g)
    rows[0] = low
    rows[1, keys // 2] = high
    rows[2] = high
    rows[3], rows[3, :keys // 2] = -inf, low
    rows[5, ::2] = low
    s, up, probs, lse, ds = call(A, rows, dtype, 1.0)
    for i, n in ((0, keys), (2, keys), (3, keys // 2)):   # differences of equal numbers are zeros, a sum of ones is exact
        want = torch.where(torch.isinf(s[i]), 0.0, 1.0 / n)
        within(probs[i], want, want * (HALF_STEP[dtype] * 1.01 + 2 * U) + TINY[dtype], ("probs", i))
        within(lse[i], s[i, 0] + torch.tensor(float(n)).double().log(), 4 * U * (abs(s[i, 0]) + 20), ("lse", i))
    only = torch.zeros(keys, dtype=dtype)
    only[keys // 2] = 1.0
    assert torch.equal(probs[1], only) and abs(lse[1].double() - s[1, keys // 2]) <= 4 * U * high
    for i in (4, 5):
        p, exact_lse = R.softmax_forward(s[i])
        rho = U * (8 * (s[4].abs().max() + exact_lse.abs()) + DEEP)
        within(probs[i], p, p * (HALF_STEP[dtype] * 1.01 + 2 * rho) + TINY[dtype], ("probs", i))
        within(lse[i], exact_lse, rho, ("lse", i))
    check_gradient(ds, s, up, lse, 1.0, dtype, [4], False)
    check_gradient(ds, s, up, lse, 1.0, dtype, [0, 1, 2, 3], dtype is not torch.float16)   # float16's ends have fractions of an exponent left
    assert torch.isfinite(ds[5].double()).all()
