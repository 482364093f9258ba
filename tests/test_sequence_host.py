"""What needs no GPU of adacomp_sequence.h: exports, structures, sizes, refusals by their codes and in Python, and the reference's gradients
against differences in 64 bits."""
import ctypes
import os
import re

import numpy as np
import pytest
import torch

import sequence_reference as S
from paper_1712_02679_amd import binding, layers, sequence
from test_layers_host import differences

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(binding.LIB_PATH):
        from paper_1712_02679_amd import build
        build.build()
    return sequence._lib()


def test_exports_every_declared_symbol(L):
    text = open(os.path.join(ROOT, "include", "adacomp_sequence.h")).read()
    declared = set(re.findall(r"\b(adacomp_[a-z0-9_]+)\s*\(", re.sub(r"/\*.*?\*/", "", text, flags=re.S)))
    assert declared == set(sequence.SEQUENCE_EXPORTS)
    for name in declared:
        assert hasattr(L, name), name
    assert f"ADACOMP_RECURRENCE_KEEP {sequence.RECURRENCE_KEEP}u" in text and f"ADACOMP_TEACHER_TOP_MAX {sequence.TEACHER_TOP_MAX}u" in text
    assert S.KEEP == sequence.RECURRENCE_KEEP


def test_struct_sizes():
    assert ctypes.sizeof(sequence._Embed) == 48 and ctypes.sizeof(sequence._Steps) == 24
    assert ctypes.sizeof(sequence._Recurrence) == 48 and ctypes.sizeof(sequence._Distill) == 104


def test_sizes(L):
    beyond = 2 ** 32
    assert sequence.adacomp_embed_workspace_bytes(1000, 50, 8) > 0
    for bad in ((2 ** 31, 50, 8), (1000, 0, 8), (1000, 2 ** 30 + 1, 8), (1000, 50, 2 ** 20 + 1), (2 ** 30, 50, 2 ** 9), (beyond + 5, 50, 8), (1000, beyond + 5, 8), (1000, 50, beyond + 8), (-1, 50, 8)):
        assert sequence.adacomp_embed_workspace_bytes(*bad) == 0, bad
    assert 0 < sequence.adacomp_embed_workspace_bytes(0, 1, 0) <= 1024
    assert sequence.adacomp_recurrence_workspace_bytes(8, 100, 64) > 0
    for bad in ((2 ** 31, 1, 8), (1, 2 ** 31, 8), (1, 1, 2 ** 20 + 1), (2 ** 16, 2 ** 15, 8), (beyond + 1, 5, 8), (1, beyond + 5, 8), (1, 5, beyond + 8), (1, -1, 8)):
        assert sequence.adacomp_recurrence_workspace_bytes(*bad) == 0, bad
    assert 0 < sequence.adacomp_recurrence_workspace_bytes(0, 0, 0) <= 1024
    assert [sequence.adacomp_recurrence_kept(n) for n in (0, 1, 64, 65, 128, 129)] == [0, 1, 1, 2, 2, 3]


def test_refusals_by_code(L):
    buf = np.zeros(1 << 16, np.uint8)
    base = (buf.ctypes.data + 255) // 256 * 256
    out, ws = base + 8192, base + 16384
    drop = lambda p=0.1: ctypes.byref(layers._Dropout(p, 0, 1, 2, None))

    def embed(rows=4, stride=8, vocab=5, cols=8, dtype=0, index=8, tokens=base, reserved=0):
        return ctypes.byref(sequence._Embed(rows, stride, vocab, cols, dtype, index, tokens, 1.0, reserved))
    forward = lambda op=None, table=base, y=out, d=None: L.adacomp_embed_forward(op or embed(), table, y, d, None)
    backward = lambda op=None, dy=base, dtable=out, d=None, w=ws, n=1 << 14: L.adacomp_embed_backward(op or embed(), dy, dtable, d, 0, w, n, None)
    for call in (forward, backward):
        for op in (embed(rows=2 ** 31), embed(vocab=0), embed(vocab=2 ** 30 + 1), embed(cols=2 ** 20 + 1), embed(rows=2 ** 30, cols=2 ** 9), embed(dtype=3), embed(index=2), embed(tokens=None), embed(reserved=1)):
            assert call(op) == binding.EINVAL
        assert call(embed(tokens=base + 4)) == binding.EALIGN and call(embed(index=4, tokens=base + 2)) == binding.EALIGN
        assert call(d=drop(1.0)) == binding.EINVAL
        assert call(embed(cols=0, tokens=None)) == binding.OK
    assert forward(embed(stride=7)) == binding.EINVAL and forward(table=None) == binding.EINVAL and forward(y=None) == binding.EINVAL
    assert forward(table=base + 2) == binding.EALIGN and forward(y=out + 2) == binding.EALIGN and forward(embed(rows=0, tokens=None), y=None) == binding.OK
    assert backward(dy=None) == binding.EINVAL and backward(dtable=None) == binding.EINVAL and backward(w=None) == binding.EINVAL
    assert backward(dy=base + 2) == binding.EALIGN and backward(dtable=out + 2) == binding.EALIGN and backward(w=ws + 8) == binding.EALIGN
    assert backward(n=sequence.adacomp_embed_workspace_bytes(4, 5, 8) - 1) == binding.EWORKSPACE

    def recurrence(b=2, n=3, c=8, dtype=0, bias=None, lengths=None):
        return ctypes.byref(sequence._Recurrence(b, n, c, dtype, bias, lengths, None, 0))
    steps = lambda data=base, b=24, n=8: ctypes.byref(sequence._Steps(data, b, n))

    def rec(op=None, x=None, forget=None, o=None, first=None, y=None, last=None, states=None, w=ws, n=1 << 14):
        return L.adacomp_recurrence_forward(op or recurrence(), x or steps(), forget or steps(), o, first, y or steps(out), last, states, w, n, None)

    def back(op=None, dy=None, x=None, o=None, states=base, dlast=None, dx=None, df=None, do=None, dbias=None, dfirst=None, w=ws, n=1 << 14):
        return L.adacomp_recurrence_backward(op or recurrence(), dy or steps(), x or steps(), steps(), o, states, dlast, dx or steps(out), df or steps(out + 1024), do,
                                             dbias, dfirst, 0, w, n, None)
    for call in (rec, back):
        for op in (recurrence(b=2 ** 31), recurrence(n=2 ** 31), recurrence(c=2 ** 20 + 1), recurrence(b=2 ** 16, n=2 ** 15), recurrence(dtype=3)):
            assert call(op) == binding.EINVAL
        assert call(recurrence(bias=base + 2)) == binding.EALIGN and call(recurrence(lengths=base + 2)) == binding.EALIGN
        assert call(x=steps(None)) == binding.EINVAL and call(x=steps(base + 2)) == binding.EALIGN and call(o=steps(None)) == binding.EINVAL
        assert call(w=None) == binding.EINVAL and call(w=ws + 8) == binding.EALIGN and call(n=255) == binding.EWORKSPACE
        assert call(recurrence(c=0), x=steps(None)) == binding.OK
    assert rec(y=steps(out, b=7)) == binding.EINVAL and rec(y=steps(out, n=7)) == binding.EINVAL and rec(y=steps(out, n=0)) == binding.EINVAL
    assert rec(first=base + 2) == binding.EALIGN and rec(last=base + 2) == binding.EALIGN and rec(states=base + 2) == binding.EALIGN
    assert back(states=None) == binding.EINVAL and back(o=steps()) == binding.EINVAL and back(do=steps(out + 2048)) == binding.EINVAL
    assert back(dx=steps(out, n=7)) == binding.EINVAL and back(df=steps(out, b=0)) == binding.EINVAL
    for name in ("states", "dlast", "dbias", "dfirst"):
        assert back(**{name: base + 2}) == binding.EALIGN

    def distill(rows=4, vocab=9, dtype=0, sz=9, sd=9, tokens=base, t=base, targets=base, top=3, tdtype=0, tb=8, gb=8, temperature=1.0, soft=1.0, hard=1.0, scale=1.0):
        return ctypes.byref(sequence._Distill(rows, vocab, dtype, sz, sd, tokens, t, targets, top, top, top, tdtype, tb, gb, temperature, soft, hard, scale))
    loss = lambda op=None, z=base, loss=out, lse=None, dloss=None, dz=None: L.adacomp_distill_forward(op or distill(), z, loss, lse, dloss, dz, None)
    grad = lambda op=None, z=base, lse=base, dloss=None, dz=out: L.adacomp_distill_backward(op or distill(), z, lse, dloss, dz, None)
    inf, nan = float("inf"), float("nan")
    for call in (loss, grad):
        for op in (distill(rows=2 ** 31), distill(vocab=0), distill(vocab=2 ** 30 + 1), distill(dtype=3), distill(top=257), distill(tdtype=3), distill(tb=2), distill(gb=1),
                   distill(tokens=None), distill(t=None), *(distill(temperature=v) for v in (0.0, -1.0, nan, inf, 1e-45, 1e39)), *(distill(soft=v) for v in (-0.1, nan, inf)),
                   *(distill(hard=v) for v in (-0.1, nan, inf)), distill(scale=nan), distill(scale=inf), distill(temperature=1e30, soft=1.0)):
            assert call(op) == binding.EINVAL
        assert call(z=None) == binding.EINVAL and call(z=base + 2) == binding.EALIGN and call(dloss=base + 2) == binding.EALIGN
        assert call(distill(tokens=base + 4)) == binding.EALIGN and call(distill(t=base + 2)) == binding.EALIGN and call(distill(targets=base + 4)) == binding.EALIGN
        assert call(dz=out + 2) == binding.EALIGN and call(distill(sd=8), dz=out) == binding.EINVAL
        assert call(distill(rows=0), z=None) == binding.OK and call(lse=base + 2) == binding.EALIGN
    assert loss(loss=None) == binding.EINVAL and loss(loss=out + 2) == binding.EALIGN
    assert grad(lse=None) == binding.EINVAL and grad(dz=None) == binding.EINVAL


def test_no_cpu_fallback(L):
    if torch.cuda.is_available():
        pytest.skip("GPU present")
    buf = np.zeros(1 << 14, np.uint8)
    base = (buf.ctypes.data + 255) // 256 * 256
    op = ctypes.byref(sequence._Embed(4, 8, 5, 8, 0, 8, base, 1.0, 0))
    assert L.adacomp_embed_forward(op, base, base + 4096, None, None) == binding.EHIP
    z = torch.zeros(4, 8)
    for call in (lambda: sequence.adacomp_embed_forward(torch.zeros(4, dtype=torch.int64), torch.zeros(5, 8), z),
                 lambda: sequence.adacomp_recurrence_forward(z[None], z[None], z[None], z),
                 lambda: sequence.adacomp_distill_forward(z, torch.zeros(4), targets=torch.zeros(4, dtype=torch.int64))):
        with pytest.raises(binding.AdacompError):
            call()


def test_reference_embedding_gradient_against_differences():
    g = torch.Generator().manual_seed(1)
    tokens = torch.tensor([[3, 0, 3, -1], [5, 3, 9, 0]])
    table, C = torch.randn(7, 11, generator=g, dtype=torch.float64), torch.randn(2, 4, 11, generator=g, dtype=torch.float64)
    drop = (0.3, 5, 6)
    dtable, _, count = S.embed_backward(tokens, C, 7, 1.7, drop)
    assert count.tolist() == [2, 0, 0, 3, 0, 1, 0]
    differences(lambda t: (S.embed_forward(tokens, t, 1.7, drop) * C).sum(), table, dtable, places=40)


@pytest.mark.parametrize("gate", [False, True])
def test_reference_recurrence_gradients_against_differences(gate):
    g = torch.Generator().manual_seed(2)
    b, n, c = 3, 9, 4
    x, forget, out, C = (torch.randn(b, n, c, generator=g, dtype=torch.float64) for _ in range(4))
    bias, first, D = (torch.randn(s, generator=g, dtype=torch.float64) for s in ((c,), (b, c), (b, c)))
    lengths = torch.tensor([9, 5, 0])
    resets = torch.zeros(b, n, dtype=torch.uint8)
    resets[0, 0], resets[0, 4], resets[1, 3], resets[1, 7] = 1, 1, 1, 1

    def of(x, forget, out, bias, first):
        return S.Recurrence(x, forget, out if gate else None, bias, first, lengths, resets)

    def value(*args):
        r = of(*args)
        return (r.y * C).sum() + (r.last * D).sum()
    args = [x, forget, out, bias, first]
    got = of(*args).backward(C, D)
    for i, name in enumerate(("dx", "dforget", "dout", "dbias", "dfirst")):
        if name in got:
            differences(lambda v: value(*[v if j == i else args[j] for j in range(5)]), args[i], got[name][0], places=30)
    assert torch.equal(of(*args).last[2], first[2]) and torch.all(of(*args).y[1, 5:] == 0)


@pytest.mark.parametrize("temperature,soft,hard", [(1.0, 1.0, 0.0), (2.5, 0.6, 0.4), (0.7, 0.0, 1.0)])
def test_reference_distillation_gradients_against_differences(temperature, soft, hard):
    g = torch.Generator().manual_seed(3)
    rows, vocab, top = 5, 13, 4
    z, t, w = torch.randn(rows, vocab, generator=g, dtype=torch.float64), torch.randn(rows, top, generator=g, dtype=torch.float64), torch.rand(rows, generator=g, dtype=torch.float64)
    tokens = torch.randint(0, vocab, (rows, top), generator=g)
    tokens[0] = torch.tensor([2, 2, 7, -1])
    tokens[1] = -1
    targets = torch.tensor([2, 5, -100, 12, 13])
    of = lambda z: S.Distill(z, tokens, t, targets, temperature, soft, hard)
    d = of(z)
    assert torch.all(d.loss >= -1e-12) and d.taught.tolist() == [soft > 0, False] + [soft > 0] * 3 and d.told.tolist() == ([True, True, False, True, False] if hard > 0 else [False] * 5)
    differences(lambda v: (of(v).loss * w).sum(), z, d.gradient(w)[0], places=60)
