"""Dropout, layer norm and the biased softmax on the GPU against their formulas in 64 bits (layers_reference.py), at the sizes,
types, strides and masks where a kernel can go wrong.  Every bound follows from the arithmetic."""
import ctypes
import math

import pytest
import torch

import layers_reference as R
from layers_reference import DEEP, HALF_STEP, TINY, U, within

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16, torch.float16]
WIDTHS = [1, 7, 8, 9, 63, 64, 65, 127, 129, 256, 257, 500, 512, 513, 577, 1024, 1025, 2047, 2048, 2056, 4096, 4099, 8192, 8200, 16384, 16391, 32768]


@pytest.fixture(scope="module")
def A():
    import paper_1712_02679_amd as A
    return A


def rand(shape, dtype, seed, scale=1.0, shift=0.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale + shift).to(dtype)


def on_gpu(t, pad=0, lead=0):
    """A copy on the GPU; with pad or lead its rows lie in wider ones, from odd addresses on."""
    if t is None or not (pad or lead):
        return None if t is None else t.to(DEV)
    wide = torch.full((*t.shape[:-1], t.shape[-1] + pad + lead), 3.0, dtype=t.dtype, device=DEV)
    part = wide[..., lead:lead + t.shape[-1]]
    part.copy_(t)
    return part


def untouched(part, pad, lead):
    """What lies between the rows of on_gpu's tensors is as it was."""
    wide = part._base
    assert torch.all(wide[..., :lead] == 3.0) and torch.all(wide[..., wide.shape[-1] - pad:] == 3.0)


# ---- dropout --------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,pad,lead", [(1, 1, 0, 0), (1, 7, 0, 0), (3, 8, 0, 0), (100, 500, 0, 0), (17, 577, 3, 1), (5, 4096, 0, 0),
                                                (2, 70001, 0, 0), (9000, 3, 0, 0), (1, 300000, 5, 3)])
def test_dropout(A, rows, cols, pad, lead, dtype):
    x, res = rand((rows, cols), dtype, 1), rand((rows, cols), dtype, 2)
    for p, seed, stream in ((0.1, 2 ** 63 + 12345, 7), (0.5, 1, 2 ** 40 + 3)):
        f = R.factors(rows, cols, p, seed, stream)
        for r in (None, res):
            gx, gr, gy = on_gpu(x, pad, lead), on_gpu(r, pad, lead), on_gpu(torch.zeros_like(x), pad, lead)
            A.adacomp_dropout(gx, gy, A.Dropout(p, seed, stream), residual=gr)
            parts = x.double() * f, (r.double() if r is not None else torch.zeros(rows, cols, dtype=torch.float64))
            want = parts[0] + parts[1]
            within(gy, want, HALF_STEP[dtype] * want.abs() * 1.01 + 4 * U * (parts[0].abs() + parts[1].abs()) + TINY[dtype], (p, r is None))
            if r is None:
                assert torch.equal(gy.cpu() == 0, (f == 0) | (x == 0) | (gy.cpu() == 0) & (want.abs() < TINY[dtype]))
            if pad or lead:
                untouched(gy, pad, lead)


def test_dropout_keeps_the_stated_share_and_calls_differ(A):
    n = 1 << 22
    x, y, z = torch.ones(n, device=DEV), torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    for p in (0.05, 0.3, 0.9):
        A.adacomp_dropout(x, y, A.Dropout(p, 11, 1))
        A.adacomp_dropout(x, z, A.Dropout(p, 11, 2))
        q = math.floor(p * 65536 + 0.5) / 65536
        six = 6 * math.sqrt(q * (1 - q) / n)   # six deviations of the share, and of what two independent masks drop together
        assert abs((y == 0).double().mean().item() - q) < six
        assert abs(((y == 0) & (z == 0)).double().mean().item() - q * q) < 6 * math.sqrt(q * q * (1 - q * q) / n)


def test_dropout_of_masked_values_and_of_rate_zero(A):
    x = torch.full((4, 64), float("nan"), device=DEV)
    y = torch.empty_like(x)
    A.adacomp_dropout(x, y, A.Dropout(0.4, 5, 6))
    f = R.factors(4, 64, 0.4, 5, 6)
    assert torch.equal(y.cpu() == 0, f == 0) and torch.equal(torch.isnan(y.cpu()), f != 0)
    x = rand((33, 77), torch.bfloat16, 3).to(DEV)
    y = torch.empty_like(x)
    A.adacomp_dropout(x, y, A.Dropout(0.0, 5, 6))
    assert torch.equal(x, y)


def test_dropout_in_place_strided_batches_and_none(A):
    x = rand((4, 6, 40), torch.float32, 4).to(DEV)
    want = torch.empty_like(x)
    A.adacomp_dropout(x, want, A.Dropout(0.3, 8, 9))
    A.adacomp_dropout(x, x, A.Dropout(0.3, 8, 9))
    assert torch.equal(x, want)
    every_other = rand((4, 12, 40), torch.float32, 4).to(DEV)[:, ::2]
    y = torch.empty(4, 6, 40, device=DEV)
    A.adacomp_dropout(every_other, y, A.Dropout(0.3, 8, 9))
    within(y, every_other.cpu().double() * R.factors(24, 40, 0.3, 8, 9).view(4, 6, 40), 4 * U * every_other.cpu().abs().double() * 2, "strided")
    for shape in ((0, 5), (5, 0)):
        A.adacomp_dropout(torch.empty(shape, device=DEV), torch.empty(shape, device=DEV), A.Dropout(0.3, 8, 9))


def test_dropout_step_in_memory_and_replayed_graph(A):
    """A captured call draws another mask when the number in memory has changed, and the same one when it has not."""
    x, y = rand((64, 500), torch.float32, 5).to(DEV), torch.empty(64, 500, device=DEV)
    step = torch.zeros(1, dtype=torch.int64, device=DEV)
    drop = A.Dropout(0.25, 77, 1000, step)
    A.adacomp_dropout(x, y, drop)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            A.adacomp_dropout(x, y, drop)
    for number in (0, 1, 5, 5):
        step.fill_(number)
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        eager = torch.empty_like(y)
        A.adacomp_dropout(x, eager, A.Dropout(0.25, 77, 1000 + number))
        assert torch.equal(y, eager)


# ---- layer norm -----------------------------------------------------------------------------------------------------

def norm_bound(dtype, z, want, mean, rstd, gamma, beta, cols):
    """Mean off by DEEP U average|z| at most, rstd by DEEP U (and what the mean's error does, which is of second order), and the
    rounding of z itself where it was a sum."""
    h = ((z - mean[:, None]) * rstd[:, None]).abs()
    size = z.abs().mean(-1, keepdim=True) * rstd[:, None]
    return HALF_STEP[dtype] * 1.01 * want.abs() + U * (gamma.abs() * (h * (DEEP + 8) + DEEP * size * (1 + h * size * DEEP * U) + 4 * z.abs() * rstd[:, None]) + 4 * beta.abs()) + TINY[dtype]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", WIDTHS)
def test_norm_forward(A, cols, dtype):
    rows, eps = (37 if cols < 5000 else 5), 1e-5
    gamma, beta = rand(cols, torch.float32, 1, 0.2, 1.0), rand(cols, torch.float32, 2, 0.5)
    x, res = rand((rows, cols), dtype, 3), rand((rows, cols), dtype, 4, 2.0, 0.5)
    for pad, lead, residual, p in ((0, 0, False, 0.0), (3, 1, True, 0.2), (0, 0, True, 0.0), (8, 0, False, 0.1)):
        gx, gr = on_gpu(x, pad, lead), on_gpu(res if residual else None, pad, lead)
        y, z = on_gpu(torch.zeros_like(x), pad, lead), on_gpu(torch.zeros_like(x), pad, lead)
        mean, rstd = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
        drop = A.Dropout(p, 99, 5) if p else None
        A.adacomp_norm_forward(gx, gamma.to(DEV), beta.to(DEV), y, residual=gr, dropout=drop, z=z, mean=mean, rstd=rstd, eps=eps)
        kept = x.double() * (R.factors(rows, cols, p, 99, 5) if p else 1.0)
        full = kept + (res.double() if residual else 0.0)
        want, m, r = R.norm_forward(full, gamma.double(), beta.double(), float(torch.tensor(eps)))
        bound_z = 4 * U * (kept.abs() + (res.double().abs() if residual else 0.0))
        within(z, full, HALF_STEP[dtype] * 1.01 * full.abs() + bound_z + TINY[dtype], "z")
        within(mean, m, U * DEEP * full.abs().mean(-1) + bound_z.mean(-1) + 2 ** -126, "mean")
        size = (1 + (full.abs().mean(-1) * r) ** 2)   # what z's and the mean's errors do to a variance that is small beside them
        within(rstd, r, U * DEEP * r * size + 2 ** -126, "rstd")
        size = size[:, None] * U * DEEP
        bound = norm_bound(dtype, full, want, m, r, gamma.double(), beta.double(), cols) + size * ((full - m[:, None]) * r[:, None] * gamma).abs()
        within(y, want, bound + bound_z * r[:, None] * gamma.abs() * 4, "y")
        if pad or lead:
            untouched(y, pad, lead)
            untouched(z, pad, lead)


def test_norm_forward_without_parameters_in_place_and_far_from_zero(A):
    x = rand((300, 96), torch.float32, 6, 1e-3, 10.0)   # the mean is 10^4 deviations away
    y = x.to(DEV)
    A.adacomp_norm_forward(y, None, None, y, eps=0.0)
    want, m, r = R.norm_forward(x.double(), 1.0, 0.0, 0.0)
    # the sum's error moves all of a row's values alike: DEEP U |mean| rstd is 0.1 of a deviation; its square enters the variance
    off = DEEP * U * m.abs() * r
    within(y, want, (off + off ** 2)[:, None] * (1 + want.abs()), "far")
    one = torch.full((3, 50), 2.5, device=DEV)
    A.adacomp_norm_forward(one, None, None, one, eps=1e-5)
    assert torch.equal(one, torch.zeros_like(one))
    A.adacomp_norm_forward(torch.empty(0, 50, device=DEV), None, None, torch.empty(0, 50, device=DEV))


def test_norm_forward_rows_stand_alone(A):
    """A NaN or an infinity stays in its row."""
    x = rand((9, 700), torch.bfloat16, 7).to(DEV)
    clean, dirty = torch.empty_like(x), torch.empty_like(x)
    A.adacomp_norm_forward(x, None, None, clean)
    x[3, 11], x[6, 699] = float("nan"), float("inf")
    A.adacomp_norm_forward(x, None, None, dirty)
    keep = [0, 1, 2, 4, 5, 7, 8]
    assert torch.equal(clean[keep], dirty[keep]) and torch.isnan(dirty[3]).all() and torch.isnan(dirty[6]).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", WIDTHS)
def test_norm_backward(A, cols, dtype):
    rows = 43 if cols < 5000 else 6
    gamma = rand(cols, torch.float32, 1, 0.2, 1.0)
    dy, add, z = rand((rows, cols), dtype, 2), rand((rows, cols), dtype, 3), rand((rows, cols), dtype, 4, 2.0, 0.5)
    _, mean, rstd = R.norm_forward(z.double(), 1.0, 0.0, 1e-5)
    mean, rstd = mean.float(), rstd.float()
    ws = torch.empty(A.adacomp_norm_workspace_bytes(rows, cols), dtype=torch.uint8, device=DEV)
    for pad, lead, with_add, p, with_gamma in ((0, 0, False, 0.0, True), (3, 1, True, 0.2, True), (8, 0, True, 0.0, False)):
        gd, ga, gz = on_gpu(dy, pad, lead), on_gpu(add if with_add else None, pad, lead), on_gpu(z, pad, lead)
        dz, dx = on_gpu(torch.zeros_like(dy), pad, lead), on_gpu(torch.zeros_like(dy), pad, lead) if p else None
        flat = torch.full((3 + 2 * cols + 5,), 0.25, device=DEV)   # gradients at odd places of a flat buffer
        dgamma, dbeta = flat[3:3 + cols], flat[4 + cols:4 + 2 * cols]
        kind = A.Dropout(p, 99, 5) if p else None
        ws.fill_(0xFF)
        A.adacomp_norm_backward(gd, gz, mean.to(DEV), rstd.to(DEV), gamma.to(DEV) if with_gamma else None, dz, dgamma, dbeta, ws, dz_add=ga, dropout=kind, dx=dx)
        w = gamma.double() if with_gamma else torch.ones(cols, dtype=torch.float64)
        want, wg, wb = R.norm_backward(dy.double(), z.double(), mean.double(), rstd.double(), w)
        more = add.double() if with_add else torch.zeros_like(want)
        h, g = ((z.double() - mean.double()[:, None]) * rstd.double()[:, None]).abs(), (dy.double() * w).abs()
        off = U * rstd.double()[:, None] * (8 * g + (DEEP + 8) * g.mean(-1, keepdim=True) + (DEEP + 16) * h * (g * h).mean(-1, keepdim=True)) + 4 * U * more.abs()
        total = want + more
        within(dz, total, HALF_STEP[dtype] * 1.01 * total.abs() + off + TINY[dtype], "dz")
        if p:
            f = R.factors(rows, cols, p, 99, 5)
            within(dx, total * f, HALF_STEP[dtype] * 1.01 * (total * f).abs() + 4 * f * (off + U * total.abs()) + TINY[dtype], "dx")
        within(dgamma, wg, U * DEEP * (dy.double() * h).abs().sum(0) + 2 ** -126, "dgamma")
        within(dbeta, wb, U * DEEP * dy.double().abs().sum(0) + 2 ** -126, "dbeta")
        assert torch.all(flat[:3] == 0.25) and flat[3 + cols] == 0.25 and torch.all(flat[4 + 2 * cols:] == 0.25)
        first = flat.clone()
        A.adacomp_norm_backward(gd, gz, mean.to(DEV), rstd.to(DEV), gamma.to(DEV) if with_gamma else None, dz, dgamma, dbeta, ws, dz_add=ga, dropout=kind, dx=dx, accumulate=True)
        assert torch.equal(flat[3:3 + cols], 2 * first[3:3 + cols]) and torch.equal(dbeta, 2 * first[4 + cols:4 + 2 * cols])   # the same sum once more, bit for bit
        if pad or lead:
            untouched(dz, pad, lead)


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 4096), (2, 64), (31, 40), (33, 40), (5000, 64), (5000, 500), (4097, 1030), (3000, 2304), (1500, 4096), (700, 9000)])
def test_norm_backward_sums_over_many_rows(A, rows, cols):
    dy, z = rand((rows, cols), torch.bfloat16, 2), rand((rows, cols), torch.bfloat16, 4, 2.0, 0.5)
    _, mean, rstd = R.norm_forward(z.double(), 1.0, 0.0, 1e-5)
    mean, rstd = mean.float(), rstd.float()
    ws = torch.empty(A.adacomp_norm_workspace_bytes(rows, cols), dtype=torch.uint8, device=DEV)
    dz, dgamma, dbeta = torch.empty(rows, cols, dtype=torch.bfloat16, device=DEV), torch.empty(cols, device=DEV), torch.empty(cols, device=DEV)
    args = (dy.to(DEV), z.to(DEV), mean.to(DEV), rstd.to(DEV), None, dz)
    A.adacomp_norm_backward(*args, dgamma, dbeta, ws)
    _, wg, wb = R.norm_backward(dy.double(), z.double(), mean.double(), rstd.double(), 1.0)
    h = (z.double() - mean.double()[:, None]) * rstd.double()[:, None]
    within(dgamma, wg, U * DEEP * (dy.double() * h).abs().sum(0) + 2 ** -126, "dgamma")
    within(dbeta, wb, U * DEEP * dy.double().abs().sum(0) + 2 ** -126, "dbeta")
    one = torch.empty_like(dgamma)
    A.adacomp_norm_backward(*args, one, None, ws)
    assert torch.equal(one, dgamma)
    A.adacomp_norm_backward(*args, None, one, ws)
    assert torch.equal(one, dbeta)
    before = dz.clone()
    A.adacomp_norm_backward(*args, None, None, ws)
    assert torch.equal(before, dz)
    inplace = dy.to(DEV)
    A.adacomp_norm_backward(inplace, *args[1:5], inplace, None, None, ws)
    assert torch.equal(before, inplace)


def test_norm_backward_without_rows(A):
    ws = torch.empty(A.adacomp_norm_workspace_bytes(0, 50), dtype=torch.uint8, device=DEV)
    none, stat = torch.empty(0, 50, device=DEV), torch.empty(0, device=DEV)
    dgamma, dbeta = torch.ones(50, device=DEV), torch.ones(50, device=DEV)
    A.adacomp_norm_backward(none, none, stat, stat, None, none, dgamma, dbeta, ws, accumulate=True)
    assert torch.all(dgamma == 1) and torch.all(dbeta == 1)
    A.adacomp_norm_backward(none, none, stat, stat, None, none, dgamma, dbeta, ws)
    assert torch.all(dgamma == 0) and torch.all(dbeta == 0)


# ---- softmax --------------------------------------------------------------------------------------------------------

# batch, heads, queries, keys, causal, starts, lengths, mask: "single" places, "row" one mask row for all, buckets, distance
SHAPES = [
    (1, 1, 1, 1, False, 0, None, None, 4, 3),
    (2, 3, 1, 64, True, [63, 10], None, None, 32, 128),
    (2, 3, 5, 63, True, [58, 3], [63, 8], None, 32, 128),
    (3, 2, 33, 65, False, 0, [65, 1, 0], None, 32, 128),
    (2, 5, 37, 128, False, 0, None, "single", 64, 250),
    (1, 4, 130, 130, True, 0, None, None, 32, 128),
    (2, 2, 40, 257, True, [217, -20], [257, 20], "single", 16, 40),
    (1, 3, 70, 500, False, 0, None, "row", 320, 800),
    (2, 2, 9, 777, False, 100, [777, 300], "single", 64, 250),
    (1, 2, 21, 1031, True, [1010], None, None, 33, 2048),
    (1, 2, 300, 300, True, 0, None, None, 32, 2048),
    (4, 2, 50, 33, False, 0, None, None, 32, 2048),
    (1, 2, 19, 2048, False, 1000, None, None, 32, 128),
    (1, 2, 11, 2051, True, [2040], None, "single", 32, 128),
    (2, 1, 3, 4096, True, [4093, 5], [4096, 8], None, 32, 128),
    (1, 1, 3, 5000, False, 2500, [4999], "single", 320, 800),
    (1, 2, 2, 8200, True, [8198], None, None, 32, 128),
    (1, 1, 3, 16384, False, 16000, None, None, 32, 128),
    (2, 1, 2, 16400, True, [16398, 8000], None, "single", 32, 128),
    (1, 2, 1, 70001, True, [70000], None, None, 32, 2048),
    (1, 3, 4, 100, False, -2 ** 31, None, None, 32, 128),
    (1, 3, 4, 100, False, 2 ** 31 - 4, None, None, 32, 128),
]


class Case:
    """Inputs of a shape and type, on the CPU and on the GPU, and the reference's results."""

    def __init__(self, A, shape, dtype, p, order="bhqk", wild=True):
        b, h, q, k, self.causal, starts, lengths, mask, buckets, far = shape
        self.A, self.dtype, self.p, self.scale = A, dtype, p, 0.3
        self.scores, self.dprobs = rand((b, h, q, k), dtype, 1, 4.0), rand((b, h, q, k), dtype, 2)
        self.table = rand((buckets, h), torch.float32, 3)
        self.map = torch.from_numpy(A.adacomp_relative_buckets(buckets // 2 * 2, far, not self.causal)) if buckets > 4 else torch.arange(2 * far + 1, dtype=torch.int32) - 1
        self.start, self.starts = (0, torch.tensor(starts, dtype=torch.int32)) if isinstance(starts, list) else (starts, None)
        self.lengths = None if lengths is None else torch.tensor(lengths, dtype=torch.int32)
        g = torch.Generator().manual_seed(5)
        self.mask = None
        if mask == "row":
            self.mask = torch.rand(1, 1, 1, k, generator=g) < 0.7
        if mask == "single":
            self.mask = (torch.rand(b, 1, q, k, generator=g) < 0.7) & (torch.rand(b, 1, q, 1, generator=g) < 0.8)
            self.mask[:, :, -1] = False
        self.ok = R.admitted(b, h, q, k, starts, self.causal, self.lengths, self.mask)
        clean = torch.where(self.ok, self.scores.double(), 0.0)
        t, self.bucket = R.biased(clean, self.table.double(), self.map.numpy(), float(torch.tensor(self.scale)), starts, self.ok)
        self.P, self.lse = R.softmax_forward(t)
        self.f = R.factors(b * h * q, k, p, 3, 4).view(b, h, q, k) if p else torch.ones(())
        up = torch.where(self.ok, self.dprobs.double(), 0.0) * self.f
        self.e, self.dtable = R.softmax_backward(self.P, up, self.bucket, buckets)
        # exponents are off by a few roundings of what they are made of; a sum of exponentials by that and its additions
        size = torch.where(self.ok, clean.abs() * self.scale + self.table.abs().max().double(), 0.0)
        size = (size.amax(-1, keepdim=True) if k else torch.zeros(b, h, q, 1, dtype=torch.float64)) + torch.where(torch.isfinite(self.lse), self.lse.abs(), 0.0)[..., None]
        self.rho = U * (8 * size + DEEP)
        self.lse_bound = U * (8 * size + DEEP)[..., 0]
        inner = (self.P * up.abs()).sum(-1, keepdim=True)
        self.e_bound = self.P * (2 * self.rho + DEEP * U) * (up.abs() + inner) + 2 ** -120
        if wild:   # places that are not admitted hold anything
            gw = torch.rand(b, h, q, k, generator=g)
            for low, value in ((0.0, float("nan")), (0.4, float("inf")), (0.7, -float("inf")), (0.8, torch.finfo(dtype).min)):
                hit = ~self.ok & (gw >= low)
                self.scores[hit], self.dprobs[hit] = value, float("nan")
        to = lambda t: None if t is None else t.to(DEV)
        place = {"bhqk": lambda t: t, "bqhk": lambda t: t.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3), "odd": lambda t: on_gpu(t, 3, 1)}[order]
        self.g_scores, self.g_dprobs = place(to(self.scores)), place(to(self.dprobs))
        self.out = place(torch.zeros(b, h, q, k, dtype=dtype, device=DEV))
        self.bias = A.RelativeBias(to(self.table), to(self.map))
        self.ws = torch.empty(A.adacomp_bias_softmax_workspace_bytes(b, h, q, k, far), dtype=torch.uint8, device=DEV).fill_(0xFF)
        self.options = dict(scale=self.scale, causal=self.causal, query_start=self.start, query_starts=to(self.starts), key_lengths=to(self.lengths),
                            mask=to(self.mask), dropout=A.Dropout(p, 3, 4) if p else None)

    def forward(self):
        lse = torch.full(self.lse.shape, 7.0, device=DEV)
        self.A.adacomp_bias_softmax_forward(self.g_scores, self.bias, self.out, self.ws, lse=lse, **self.options)
        want = self.P * self.f
        within(self.out, want, want * (HALF_STEP[self.dtype] * 1.01 + 2 * self.rho) + TINY[self.dtype], "probs")
        within(lse, self.lse, self.lse_bound, "lse")
        return lse

    def backward(self, accumulate=False):
        lse = self.lse.float().to(DEV)
        dtable = torch.ones(self.table.shape, device=DEV)
        self.A.adacomp_bias_softmax_backward(self.g_scores, self.bias, lse, self.g_dprobs, self.out, dtable, self.ws, accumulate=accumulate, **self.options)
        want = self.e * self.scale
        within(self.out, want, HALF_STEP[self.dtype] * 1.01 * want.abs() + 2 * self.scale * self.e_bound + TINY[self.dtype], "dscores")
        bound = torch.zeros_like(self.dtable)
        each = self.e_bound + DEEP * U * self.e.abs()
        bound.index_add_(0, self.bucket.reshape(-1), each.permute(0, 2, 3, 1).reshape(-1, self.table.shape[1]))
        within(dtable, self.dtable + (1.0 if accumulate else 0.0), bound + U * (1 + self.dtable.abs()) + 2 ** -126, "dtable")
        return dtable


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s[:4])))
def test_softmax(A, shape, dtype):
    for p, order in ((0.0, "bhqk"), (0.2, "odd"), (0.1, "bqhk")):
        c = Case(A, shape, dtype, p, order)
        c.forward()
        first = c.backward()
        assert torch.equal(first, c.backward())   # sums in a fixed order
        c.backward(accumulate=True)
        if order == "odd":
            untouched(c.out, 3, 1)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("far,buckets", [(3, 4), (128, 32), (250, 64), (800, 320), (2048, 32)])
def test_softmax_of_few_keys(A, far, buckets, dtype):
    """Rows shorter than a group of 8, and just longer ones, whatever form the distances make them take."""
    for keys in (1, 2, 5, 7, 8, 9, 15, 16, 17):
        for mask in (None, "single"):
            c = Case(A, (2, 3, 21, keys, mask is None, 0 if mask else [keys - 21, 4], None if mask else [keys, (keys + 1) // 2], mask, buckets, far), dtype, 0.1, "odd")
            c.forward()
            c.backward()
            untouched(c.out, 3, 1)


@pytest.mark.parametrize("keys", [65, 129, 200, 257, 511, 513, 900, 1025, 1500, 2049, 3500, 4097, 8193, 12001, 16385, 30001, 32769])
def test_softmax_at_the_bounds_of_its_forms(A, keys):
    for far, buckets, dtype, mask in ((128, 32, torch.bfloat16, None), (800, 320, torch.float32, "single"), (2048, 33, torch.float16, "row")):
        queries = 40 if keys < 1000 else 7
        c = Case(A, (2, 2, queries, keys, True, [keys - queries, keys // 2], [keys, keys // 2 + 1], mask, buckets, far), dtype, 0.1)
        c.forward()
        c.backward()


def test_softmax_of_many_short_sequences(A):
    """More (batch, head) pairs than workgroups fit the GPU, and heads without rows for every workgroup."""
    for shape in ((300, 7, 3, 20, True, 17, None, None, 32, 128), (1, 600, 2, 40, False, 0, None, None, 32, 128), (50, 1, 90, 33, False, 0, None, None, 32, 128)):
        c = Case(A, shape, torch.bfloat16, 0.1)
        c.forward()
        c.backward()


@pytest.mark.parametrize("batch,heads,queries,keys", [(70, 3, 1, 17), (70, 3, 5, 60), (45, 5, 7, 100), (37, 2, 1, 300), (21, 3, 1, 1000), (4099, 1, 1, 700), (700, 6, 1, 2100),
                                                      (9000, 4, 3, 9)])
def test_softmax_of_sequences_that_share_workgroups(A, batch, heads, queries, keys):
    """Sequences of so few rows that a workgroup takes rows of several, each with its own start, length and mask."""
    starts, lengths = [(7 * b) % (keys + 3) - 1 for b in range(batch)], [(5 * b) % (keys + 1) for b in range(batch)]
    for mask, dtype, order in ((None, torch.bfloat16, "bqhk"), ("single", torch.float32, "odd")):
        c = Case(A, (batch, heads, queries, keys, True, starts, lengths, mask, 32, 128), dtype, 0.1, order)
        c.forward()
        if order == "odd":
            untouched(c.out, 3, 1)


def test_softmax_in_place_and_without_the_table_gradient(A):
    for shape in (SHAPES[4], SHAPES[12], SHAPES[18]):
        c = Case(A, shape, torch.bfloat16, 0.1)
        c.forward()
        probs = c.out.clone()
        c.backward()
        dscores = c.out.clone()
        lse = c.lse.float().to(DEV)
        A.adacomp_bias_softmax_backward(c.g_scores, c.bias, lse, c.g_dprobs, c.g_dprobs, None, c.ws, **c.options)
        assert torch.equal(c.g_dprobs, dscores)
        A.adacomp_bias_softmax_forward(c.g_scores, c.bias, c.g_scores, c.ws, **c.options)
        assert torch.equal(c.g_scores, probs)


@pytest.mark.parametrize("keys", [40, 300, 1500, 3000, 20000])
def test_softmax_of_infinities_and_lowest_values(A, keys):
    """Admitted scores of -infinity count nothing, a row of them is empty, rows of the type's lowest value are even, and a NaN stays in
    its row."""
    for dtype in TYPES:
        c = Case(A, (1, 1, 6, keys, False, 0, None, None, 32, 128), dtype, 0.0)
        s = c.g_scores
        s[0, 0, 1] = -float("inf")
        s[0, 0, 2, keys // 2:] = -float("inf")
        s[0, 0, 3] = torch.finfo(dtype).min
        s[0, 0, 4, 3] = float("nan")
        c.bias.table.zero_()
        lse = torch.empty(1, 1, 6, device=DEV)
        A.adacomp_bias_softmax_forward(s, c.bias, c.out, c.ws, lse=lse, **c.options)
        out = c.out[0, 0].cpu()
        assert torch.all(out[1] == 0) and lse[0, 0, 1] == -float("inf")
        assert torch.all(out[2, keys // 2:] == 0) and abs(out[2].double().sum() - 1) < keys * HALF_STEP[dtype] / keys * 2 + DEEP * U
        even = torch.full((keys,), 1.0 / keys).to(dtype)
        assert (out[3].double() - 1.0 / keys).abs().max() <= abs(even[0].double() - 1.0 / keys) + HALF_STEP[dtype] * 2 / keys + TINY[dtype]
        assert torch.isnan(out[4]).all()
        for i in (0, 5):
            assert torch.isfinite(out[i].double()).all()
        A.adacomp_bias_softmax_backward(s, c.bias, lse, c.g_dprobs, c.out, None, c.ws, **c.options)
        out = c.out[0, 0].cpu()
        assert torch.all(out[1] == 0) and torch.all(out[2, keys // 2:] == 0) and torch.isfinite(out[[0, 1, 2, 3, 5]].double()).all()


@pytest.mark.parametrize("keys", [30, 100, 700, 2000, 5000, 20000, 40000])
def test_softmax_of_rows_with_nan_is_zero_where_it_does_not_look(A, keys):
    """A NaN among the admitted scores or gradients of a row reaches the row's admitted places, no other place and no other row."""
    for dtype in (torch.float32, torch.bfloat16):
        c = Case(A, (1, 2, 5, keys, False, keys // 2, [keys - 3], "row", 32, 128), dtype, 0.1, wild=False)
        first = int(c.ok[0, 0, 1].nonzero()[0])
        c.g_scores[0, 0, 1, first] = float("nan")
        c.g_dprobs[0, 1, 2, int(c.ok[0, 1, 2].nonzero()[0])] = float("nan") if not c.f.dim() or c.f[0, 1, 2, int(c.ok[0, 1, 2].nonzero()[0])] else 0.0
        lse = torch.empty(1, 2, 5, device=DEV)
        A.adacomp_bias_softmax_forward(c.g_scores, c.bias, c.out, c.ws, lse=lse, **c.options)
        out, ok = c.out.cpu().double(), c.ok
        assert torch.all(out[~ok] == 0) and torch.isnan(lse.cpu()).sum() == 1 and torch.isnan(out).any(-1).sum() == 1
        A.adacomp_bias_softmax_backward(c.g_scores, c.bias, lse, c.g_dprobs, c.out, None, c.ws, **c.options)
        out = c.out.cpu().double()
        assert torch.all(out[~ok] == 0) and torch.isnan(out).any(-1).sum() <= 2 and torch.isnan(out[0, 0, 1][ok[0, 0, 1]]).all()


def test_softmax_of_nothing(A):
    bias = A.RelativeBias(torch.zeros(8, 3, device=DEV), torch.zeros(9, dtype=torch.int32, device=DEV))
    ws = torch.empty(1024, dtype=torch.uint8, device=DEV)
    for shape in ((0, 3, 4, 5), (2, 3, 0, 5), (2, 3, 4, 0)):
        s, lse = torch.empty(shape, device=DEV), torch.ones(shape[:3], device=DEV)
        A.adacomp_bias_softmax_forward(s, bias, s, ws, lse=lse)
        assert torch.all(torch.isneginf(lse))
        for accumulate in (True, False):
            dtable = torch.ones(8, 3, device=DEV)
            A.adacomp_bias_softmax_backward(s, bias, lse, s, s, dtable, ws, accumulate=accumulate)
            assert torch.all(dtable == (1.0 if accumulate else 0.0))


def test_softmax_of_buckets_outside_the_table(A):
    """Numbers of a map beyond the table count as the nearest bucket: nothing outside is read or written."""
    flat = torch.full((4 + 8 * 2 + 4,), 9.0, device=DEV)
    bias = A.RelativeBias(torch.zeros(8, 2, device=DEV), torch.tensor([-5, 0, 3, 8, 10 ** 9], dtype=torch.int32, device=DEV))
    s, up = rand((1, 2, 6, 6), torch.float32, 1).to(DEV), rand((1, 2, 6, 6), torch.float32, 2).to(DEV)
    out, lse, ws = torch.empty_like(s), torch.empty(1, 2, 6, device=DEV), torch.empty(A.adacomp_bias_softmax_workspace_bytes(1, 2, 6, 6, 2), dtype=torch.uint8, device=DEV)
    A.adacomp_bias_softmax_forward(s, bias, out, ws, lse=lse)
    dtable = flat[4:20].view(8, 2)
    A.adacomp_bias_softmax_backward(s, bias, lse, up, out, dtable, ws)
    assert torch.all(flat[:4] == 9) and torch.all(flat[20:] == 9)
    assert torch.all(dtable[[1, 2, 4, 5, 6]] == 0) and torch.all(dtable[[0, 3, 7]] != 0)


def test_softmax_offsets_beyond_32_bits(A):
    """Two sequences whose scores lie more than 2^32 elements apart."""
    q, k = 3, 200
    far = 2 ** 32 + 4096
    wide = torch.zeros(far + 2 * q * k, dtype=torch.bfloat16, device=DEV)
    s = wide.as_strided((2, 2, q, k), (far, q * k, k, 1))
    near = rand((2, 2, q, k), torch.bfloat16, 8).to(DEV)
    s.copy_(near)
    bias = A.RelativeBias(rand((32, 2), torch.float32, 9).to(DEV), torch.from_numpy(A.adacomp_relative_buckets(32, 128, True)).to(DEV))
    ws = torch.empty(A.adacomp_bias_softmax_workspace_bytes(2, 2, q, k, 128), dtype=torch.uint8, device=DEV)
    want, lse = torch.empty_like(near), torch.empty(2, 2, q, device=DEV)
    A.adacomp_bias_softmax_forward(near, bias, want, ws, lse=lse)
    A.adacomp_bias_softmax_forward(s, bias, s, ws)
    assert torch.equal(s, want)


# ---- large calls ----------------------------------------------------------------------------------------------------

def test_large_calls_agree_with_small_ones(A):
    """Calls beyond the caches, whose inputs and results go past them, give their first rows what a call of those rows alone gives."""
    few = 700
    for rows, cols in ((26000, 4096), (110000, 1024), (13000, 8192)):
        g = torch.Generator(device=DEV).manual_seed(cols)
        new = lambda: torch.randn(rows, cols, generator=g, device=DEV).to(torch.bfloat16)
        x, res, drop = new(), new(), A.Dropout(0.1, 4, 5)
        y, part = torch.empty_like(x), torch.empty(few, cols, dtype=torch.bfloat16, device=DEV)
        A.adacomp_dropout(x, y, drop, residual=res)
        A.adacomp_dropout(x[:few], part, drop, residual=res[:few])
        assert torch.equal(y[:few], part)
        gamma, beta = torch.randn(cols, generator=g, device=DEV), torch.randn(cols, generator=g, device=DEV)
        z, mean, rstd = torch.empty_like(x), torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
        A.adacomp_norm_forward(x, gamma, beta, y, residual=res, dropout=drop, z=z, mean=mean, rstd=rstd)
        A.adacomp_norm_forward(x[:few], gamma, beta, part, residual=res[:few], dropout=drop)
        assert torch.equal(y[:few], part)
        dz, dx, dgamma, dbeta = torch.empty_like(x), torch.empty_like(x), torch.empty_like(gamma), torch.empty_like(beta)
        ws = torch.empty(A.adacomp_norm_workspace_bytes(rows, cols), dtype=torch.uint8, device=DEV)
        A.adacomp_norm_backward(x, z, mean, rstd, gamma, dz, dgamma, dbeta, ws, dz_add=res, dropout=drop, dx=dx)
        part_x = torch.empty_like(part)
        A.adacomp_norm_backward(x[:few], z[:few], mean[:few], rstd[:few], gamma, part, None, None, ws, dz_add=res[:few], dropout=drop, dx=part_x)
        assert torch.equal(dz[:few], part) and torch.equal(dx[:few], part_x)
        h = (z.double() - mean.double()[:, None]) * rstd.double()[:, None]
        within(dgamma, (x.double() * h).sum(0).cpu(), U * 400 * (x.double() * h).abs().sum(0).cpu(), "dgamma")   # up to 110000 / 2048 rows a thread
        within(dbeta, x.double().sum(0).cpu(), U * 400 * x.double().abs().sum(0).cpu(), "dbeta")
        del h
    for keys in (1024, 2048, 4096, 8192, 16384, 32768):
        batch, heads, queries = 4, 4, (1 << 22) // keys
        g = torch.Generator(device=DEV).manual_seed(keys)
        s, up = (torch.randn(batch, heads, queries, keys, generator=g, device=DEV).to(torch.float16) for _ in range(2))
        bias = A.RelativeBias(torch.randn(32, heads, generator=g, device=DEV), torch.from_numpy(A.adacomp_relative_buckets(32, 128, True)).to(DEV))
        ws = torch.empty(A.adacomp_bias_softmax_workspace_bytes(batch, heads, queries, keys, 128), dtype=torch.uint8, device=DEV)
        lengths = torch.tensor([keys - 5, keys, keys // 2, 1], dtype=torch.int32, device=DEV)
        out, part, lse = torch.empty_like(s), torch.empty_like(s[:1]), torch.empty(batch, heads, queries, device=DEV)
        options = dict(scale=0.5, query_start=keys // 2, dropout=A.Dropout(0.2, 7, 8))
        A.adacomp_bias_softmax_forward(s, bias, out, ws, lse=lse, key_lengths=lengths, **options)
        A.adacomp_bias_softmax_forward(s[:1], bias, part, ws, key_lengths=lengths[:1], **options)
        assert torch.equal(out[:1], part)
        dtable, small = torch.empty(32, heads, device=DEV), torch.zeros(32, heads, device=DEV)
        A.adacomp_bias_softmax_backward(s, bias, lse, up, out, dtable, ws, key_lengths=lengths, **options)
        for b in range(batch):
            drop = dict(options, dropout=None)
            if b == 0:
                A.adacomp_bias_softmax_backward(s[:1], bias, lse[:1], up[:1], part, None, ws, key_lengths=lengths[:1], **options)
                assert torch.equal(out[:1], part)
            A.adacomp_bias_softmax_backward(s[b:b + 1], bias, lse[b:b + 1], up[b:b + 1], part, small, ws, key_lengths=lengths[b:b + 1], accumulate=True, **drop)
        whole = torch.empty_like(dtable)
        A.adacomp_bias_softmax_backward(s, bias, lse, up, out, whole, ws, key_lengths=lengths, **drop)
        # the same terms in another order: |e| is below 5 P, and a row's P add up to 1
        assert (whole.double() - small.double()).abs().max() <= U * 400 * batch * queries * 10


def test_more_rows_than_one_launch_takes(A):
    """Dropout beyond 2^30 groups and norm beyond 2^22 rows, which go in several launches, and more (batch, head) pairs than a launch of the
    forward softmax has workgroups: what lies behind the seams is what calls of those rows give."""
    rows = (1 << 30) + 700
    x = torch.ones(rows, 1, dtype=torch.bfloat16, device=DEV)
    A.adacomp_dropout(x, x, A.Dropout(0.5, 12, 13))
    for first in (0, (1 << 30) - 300, rows - 500):
        assert torch.equal(x[first:first + 500, 0].cpu().double(), R.factors(500, 1, 0.5, 12, 13, first)[:, 0])
    del x
    rows, cols = (1 << 22) + 700, 9
    g = torch.Generator(device=DEV).manual_seed(3)
    x = torch.randn(rows, cols, generator=g, device=DEV)
    y, mean, rstd = torch.empty_like(x), torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
    A.adacomp_norm_forward(x, None, None, y, mean=mean, rstd=rstd)
    part, part_mean, part_rstd = torch.empty(900, cols, device=DEV), torch.empty(900, device=DEV), torch.empty(900, device=DEV)
    for first in (0, (1 << 22) - 300, rows - 900):
        A.adacomp_norm_forward(x[first:first + 900], None, None, part, mean=part_mean, rstd=part_rstd)
        assert torch.equal(y[first:first + 900], part) and torch.equal(mean[first:first + 900], part_mean) and torch.equal(rstd[first:first + 900], part_rstd)
    A.adacomp_norm_forward(x, None, None, y, dropout=A.Dropout(0.5, 1, 2), z=y.new_empty(y.shape), mean=mean)
    first = (1 << 22) - 300
    kept = x[first:first + 900].cpu().double() * R.factors(900, cols, 0.5, 1, 2, first)
    within(mean[first:first + 900], kept.mean(-1), U * DEEP * kept.abs().mean(-1), "mean of what dropout leaves")
    batch, keys = (1 << 20) + 500, 11
    s = torch.randn(batch, 1, 1, keys, generator=g, device=DEV)
    bias = A.RelativeBias(torch.randn(8, 1, generator=g, device=DEV), torch.from_numpy(A.adacomp_relative_buckets(8, 6, True)).to(DEV))
    ws = torch.empty(A.adacomp_bias_softmax_workspace_bytes(batch, 1, 1, keys, 6), dtype=torch.uint8, device=DEV)
    probs, part = torch.empty_like(s), torch.empty_like(s[:900])
    A.adacomp_bias_softmax_forward(s, bias, probs, ws, query_start=5)
    for first in (0, batch - 900):
        A.adacomp_bias_softmax_forward(s[first:first + 900], bias, part, ws, query_start=5)
        assert torch.equal(probs[first:first + 900], part)
    lse, ds, dtable = torch.empty(batch, 1, 1, device=DEV), torch.empty_like(s), torch.empty(8, 1, device=DEV)
    A.adacomp_bias_softmax_forward(s, bias, probs, ws, query_start=5, lse=lse)
    A.adacomp_bias_softmax_backward(s, bias, lse, s, ds, dtable, ws, query_start=5)
    p = probs.double()
    e = p * (s.double() - (p * s.double()).sum(-1, keepdim=True))
    bucket = bias.map.long()[(torch.arange(keys, device=DEV) - 5).clamp(-6, 6) + 6]
    want = torch.zeros(8, dtype=torch.float64, device=DEV).index_add_(0, bucket, e.sum((0, 1, 2)))
    size = torch.zeros(8, dtype=torch.float64, device=DEV).index_add_(0, bucket, (p * (s.double().abs() + 5)).sum((0, 1, 2)))
    assert torch.all((dtable[:, 0].double() - want).abs() <= U * 400 * size)   # a thread adds up to 25 of the rows


def test_more_sequences_than_a_launch_of_the_softmax_has_workgroups(A):
    """Sequences that have workgroups of their own, since they have too many rows to share them."""
    g = torch.Generator(device=DEV).manual_seed(3)
    batch, queries, keys = (1 << 20) + 500, 130, 2
    s = torch.randn(batch, 1, queries, keys, generator=g, dtype=torch.bfloat16, device=DEV)
    bias = A.RelativeBias(torch.randn(8, 1, generator=g, device=DEV), torch.from_numpy(A.adacomp_relative_buckets(8, 6, True)).to(DEV))
    ws = torch.empty(A.adacomp_bias_softmax_workspace_bytes(batch, 1, queries, keys, 6), dtype=torch.uint8, device=DEV)
    probs, part = torch.empty_like(s), torch.empty_like(s[:900])
    A.adacomp_bias_softmax_forward(s, bias, probs, ws)
    for first in (0, (1 << 20) - 450, batch - 900):
        A.adacomp_bias_softmax_forward(s[first:first + 900], bias, part, ws)
        assert torch.equal(probs[first:first + 900], part)


# ---- gradients against differences of the kernels' own results -----------------------------------------------------

def test_norm_gradients_against_differences(A):
    """Along random directions in float32: sums of C y over the batch change by the gradients' products, up to the step's square
    and the rounding of the sums."""
    rows, cols, eps, step = 24, 130, 1e-5, 1e-2
    x, gamma, beta, C = (rand(s, torch.float32, i).to(DEV) for i, s in enumerate([(rows, cols), (cols,), (cols,), (rows, cols)]))
    drop = A.Dropout(0.2, 4, 4)
    y, z, mean, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)

    def value(x, gamma, beta):
        A.adacomp_norm_forward(x, gamma, beta, y, dropout=drop, z=z, mean=mean, rstd=rstd, eps=eps)
        return (y.double() * C.double()).sum().item()

    value(x, gamma, beta)
    dz, dx, dgamma, dbeta = torch.empty_like(x), torch.empty_like(x), torch.empty_like(gamma), torch.empty_like(beta)
    ws = torch.empty(A.adacomp_norm_workspace_bytes(rows, cols), dtype=torch.uint8, device=DEV)
    A.adacomp_norm_backward(C, z.clone(), mean.clone(), rstd.clone(), gamma, dz, dgamma, dbeta, ws, dropout=drop, dx=dx)
    for which, grad in enumerate((dx, dgamma, dbeta)):
        at = [x, gamma, beta]
        u = rand(grad.shape, torch.float32, 20 + which).to(DEV)
        up, down = list(at), list(at)
        up[which], down[which] = at[which] + step * u, at[which] - step * u
        got = (value(*up) - value(*down)) / (2 * step)
        want = (grad.double() * u.double()).sum().item()
        scale = (C.abs().double().sum().item())
        # third derivatives of y are of the order of 1; y's own float32 errors, divided by the step
        assert abs(got - want) < scale * (step ** 2 * 4 + 8 * U / step), (which, got, want)


def test_softmax_gradients_against_differences(A):
    b, h, q, k, step = 2, 2, 9, 60, 1e-2
    s, C, table = rand((b, h, q, k), torch.float32, 1).to(DEV), rand((b, h, q, k), torch.float32, 2).to(DEV), rand((32, h), torch.float32, 3).to(DEV)
    buckets = torch.from_numpy(A.adacomp_relative_buckets(32, 40, False)).to(DEV)
    ws = torch.empty(A.adacomp_bias_softmax_workspace_bytes(b, h, q, k, 40), dtype=torch.uint8, device=DEV)
    probs, lse = torch.empty_like(s), torch.empty(b, h, q, device=DEV)
    options = dict(scale=0.7, causal=True, query_start=k - q, dropout=A.Dropout(0.1, 6, 6))

    def value(s, table):
        A.adacomp_bias_softmax_forward(s, A.RelativeBias(table, buckets), probs, ws, lse=lse, **options)
        return (probs.double() * C.double()).sum().item()

    value(s, table)
    ds, dtable = torch.empty_like(s), torch.empty_like(table)
    A.adacomp_bias_softmax_backward(s, A.RelativeBias(table, buckets), lse.clone(), C, ds, dtable, ws, **options)
    for which, grad in enumerate((ds, dtable)):
        at = [s, table]
        u = rand(grad.shape, torch.float32, 30 + which).to(DEV)
        up, down = list(at), list(at)
        up[which], down[which] = at[which] + step * u, at[which] - step * u
        got = (value(*up) - value(*down)) / (2 * step)
        want = (grad.double() * u.double()).sum().item()
        # a row's probabilities add up to 1, and |C| is below 5
        assert abs(got - want) < b * h * q * 5 * (step ** 2 * 8 + 64 * U / step), (which, got, want)


# ---- streams, graphs, refusals --------------------------------------------------------------------------------------

def test_calls_run_on_the_current_stream_and_can_be_captured(A):
    c = Case(A, SHAPES[8], torch.bfloat16, 0.1)
    rows, cols = 50, 577
    dy, z = rand((rows, cols), torch.float32, 2).to(DEV), rand((rows, cols), torch.float32, 4).to(DEV)
    y, dz, mean, rstd = torch.empty_like(z), torch.empty_like(z), torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
    dgamma, dbeta, dtable = torch.empty(cols, device=DEV), torch.empty(cols, device=DEV), torch.empty_like(c.bias.table)
    ws = torch.empty(A.adacomp_norm_workspace_bytes(rows, cols), dtype=torch.uint8, device=DEV)
    lse = torch.empty(c.lse.shape, device=DEV)
    ds = torch.empty_like(c.g_scores)

    def calls():
        A.adacomp_norm_forward(z, None, None, y, mean=mean, rstd=rstd)
        A.adacomp_norm_backward(dy, z, mean, rstd, None, dz, dgamma, dbeta, ws)
        A.adacomp_bias_softmax_forward(c.g_scores, c.bias, c.out, c.ws, lse=lse, **c.options)
        A.adacomp_bias_softmax_backward(c.g_scores, c.bias, lse, c.g_dprobs, ds, dtable, c.ws, **c.options)

    results = [y, mean, rstd, dz, dgamma, dbeta, c.out, lse, ds, dtable]
    calls()
    torch.cuda.synchronize()
    eager = [t.clone() for t in results]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        calls()
        with torch.cuda.graph(graph, stream=side):
            calls()
    torch.cuda.synchronize()
    for _ in range(3):
        for t in results:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for want, got in zip(eager, results):
            assert torch.equal(want, got)


def test_refusals(A):
    x = torch.zeros(4, 16, device=DEV)
    drop = A.Dropout(0.1, 1)
    E = A.AdacompError
    with pytest.raises(E):
        A.adacomp_dropout(x, x, None)
    with pytest.raises(E):
        A.adacomp_dropout(x, torch.zeros(4, 17, device=DEV), drop)
    with pytest.raises(E):
        A.adacomp_dropout(x, x.bfloat16(), drop)
    with pytest.raises(E):
        A.adacomp_dropout(x.double(), x.double(), drop)
    with pytest.raises(E):
        A.adacomp_dropout(x.cpu(), x.cpu(), drop)
    with pytest.raises(E):
        A.adacomp_dropout(x.t(), x.t(), drop)
    with pytest.raises(E):
        A.adacomp_dropout(x, x[:1].expand(4, 16), drop)              # an output whose rows are one
    for p in (-0.1, 1.0, 1.5, float("nan"), 0.9999999):
        with pytest.raises(E):
            A.adacomp_dropout(x, x, A.Dropout(p, 1))
    y, w = torch.zeros_like(x), torch.zeros(16, device=DEV)
    with pytest.raises(E):
        A.adacomp_norm_forward(x, w[:8], w, y)
    with pytest.raises(E):
        A.adacomp_norm_forward(x, w.bfloat16(), w, y)
    with pytest.raises(E):
        A.adacomp_norm_forward(x, w, w, y, eps=-1.0)
    with pytest.raises(E):
        A.adacomp_norm_forward(x, w, w, y, z=y)
    with pytest.raises(E):
        A.adacomp_norm_forward(torch.zeros(1, 32769, device=DEV), None, None, torch.zeros(1, 32769, device=DEV))
    stat = torch.zeros(4, device=DEV)
    small = torch.zeros(16, dtype=torch.uint8, device=DEV)
    with pytest.raises(E) as error:
        A.adacomp_norm_backward(x, x, stat, stat, w, y, w, w.clone(), small)
    assert error.value.code == -6
    ws = torch.zeros(A.adacomp_norm_workspace_bytes(4, 16), dtype=torch.uint8, device=DEV)
    with pytest.raises(E):
        A.adacomp_norm_backward(x, x, stat, stat, w, y, w, w.clone(), ws, dx=torch.zeros_like(x))   # dx is dz without dropout
    with pytest.raises(E):
        A.adacomp_norm_backward(x, x, stat[:3], stat, w, y, w, w.clone(), ws)
    s = torch.zeros(2, 3, 4, 5, device=DEV)
    table, buckets = torch.zeros(8, 3, device=DEV), torch.zeros(9, dtype=torch.int32, device=DEV)
    bias = A.RelativeBias(table, buckets)
    room = torch.zeros(1 << 16, dtype=torch.uint8, device=DEV)
    lse = torch.zeros(2, 3, 4, device=DEV)
    for bad in (lambda: A.RelativeBias(table, buckets[:8]), lambda: A.RelativeBias(table.t(), buckets), lambda: A.RelativeBias(table, buckets.long()),
                lambda: A.adacomp_bias_softmax_forward(s[0], bias, s[0], room),
                lambda: A.adacomp_bias_softmax_forward(s, A.RelativeBias(torch.zeros(8, 2, device=DEV), buckets), s, room),
                lambda: A.adacomp_bias_softmax_forward(s, bias, s.transpose(2, 3), room),
                lambda: A.adacomp_bias_softmax_forward(s, bias, s, room, mask=torch.zeros(2, 3, 4, 5, device=DEV)),
                lambda: A.adacomp_bias_softmax_forward(s, bias, s, room, key_lengths=torch.zeros(3, dtype=torch.int32, device=DEV)),
                lambda: A.adacomp_bias_softmax_forward(s, bias, s, room, key_lengths=torch.zeros(2, dtype=torch.int64, device=DEV)),
                lambda: A.adacomp_bias_softmax_forward(s, bias, s[:1].expand(2, 3, 4, 5), room),
                lambda: A.adacomp_bias_softmax_forward(s, A.RelativeBias(table, torch.zeros(4099, dtype=torch.int32, device=DEV)), s, room),
                lambda: A.adacomp_bias_softmax_backward(s, bias, lse, s, s.clone(), torch.zeros(7, 3, device=DEV), room),
                lambda: A.adacomp_bias_softmax_backward(s, bias, lse[:1], s, s.clone(), table.clone(), room),
                lambda: A.adacomp_bias_softmax_backward(s, bias, None, s, s.clone(), table.clone(), room)):
        with pytest.raises(E):
            bad()
    with pytest.raises(E) as error:
        A.adacomp_bias_softmax_backward(s, bias, lse, s, s.clone(), table.clone(), small)
    assert error.value.code == -6
    torch.cuda.synchronize()
