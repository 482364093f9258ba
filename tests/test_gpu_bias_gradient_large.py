"""The backward biased softmax of large line-aligned 16-bit inputs, which go past the caches: dscores and the table's gradient against 64 bits, with
and without dropout.

dprobs and the table favour near keys, so that without dropout every bucket's gradient is a sum of terms of one sign, far above its bound."""
import pytest
import torch

import layers_reference as R
from layers_reference import DEEP, HALF_STEP, TINY, U

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BUCKETS, FAR, SCALE = 32, 128, 0.5


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("keys", [1056, 2048, 4096, 8192, 16384, 32768])
def test_against_64_bits(keys, dtype):
    import paper_1712_02679_amd as A
    batch, heads, queries = 4, 4, (1 << 22) // keys
    assert batch * heads * queries * keys * 4 >= 192 << 20 and keys % 32 == 0   # the inputs' bytes and lines from which they go past the caches
    g = torch.Generator(device=DEV).manual_seed(keys)
    start = keys // 2
    lengths = [keys - 5, keys, keys // 2, 1]
    away = torch.arange(keys, device=DEV)[None, :] - start - torch.arange(queries, device=DEV)[:, None]
    where = torch.from_numpy(A.adacomp_relative_buckets(BUCKETS, FAR, True)).to(DEV)
    bucket = where.long()[away.clamp(-FAR, FAR) + FAR]
    table = torch.randn(BUCKETS, heads, generator=g, device=DEV) + 4.0
    table[[BUCKETS // 2 - 1, BUCKETS - 1]] -= 4.0
    s = torch.randn(batch, heads, queries, keys, generator=g, device=DEV).to(dtype)
    up = (torch.randn(batch, heads, queries, keys, generator=g, device=DEV) * 0.1 + 3.0 * (bucket % (BUCKETS // 2) < BUCKETS // 2 - 1)).to(dtype)
    rows = batch * heads * queries
    ws = torch.empty(A.adacomp_bias_softmax_workspace_bytes(batch, heads, queries, keys, FAR), dtype=torch.uint8, device=DEV)
    options = dict(scale=SCALE, query_start=start, key_lengths=torch.tensor(lengths, dtype=torch.int32, device=DEV))
    bias, lse, ds = A.RelativeBias(table, where), torch.empty(batch, heads, queries, device=DEV), torch.empty_like(s)
    A.adacomp_bias_softmax_forward(s, bias, torch.empty_like(s), ws, lse=lse, **options)
    for p in (0.0, 0.2):
        drop = A.Dropout(p, 7, 8) if p else None
        factor = None
        if p:   # dropout of ones: the factors, which its own tests hold against the generator
            factor = torch.ones(rows, keys, dtype=torch.float32, device=DEV)
            A.adacomp_dropout(factor, factor, drop)
            assert torch.equal(factor[:2].cpu().double(), R.factors(2, keys, p, 7, 8).float().double())
            factor = factor.view(s.shape)
        dtable = torch.empty_like(table)
        A.adacomp_bias_softmax_backward(s, bias, lse, up, ds, dtable, ws, dropout=drop, **options)
        want, bound = (torch.zeros(BUCKETS, heads, dtype=torch.float64, device=DEV) for _ in range(2))
        for b in range(batch):
            ok = torch.arange(keys, device=DEV) < lengths[b]
            for h in range(heads):
                t = s[b, h].double() * SCALE + table[:, h].double()[bucket]
                prob = torch.where(ok, torch.exp(t - lse[b, h].double()[:, None]), 0.0)
                dp = up[b, h].double() * (factor[b, h].double() if p else 1.0)
                e = prob * (dp - (prob * dp).sum(-1, keepdim=True))
                size = torch.where(ok, t.abs(), 0.0).amax(-1, keepdim=True) + lse[b, h].double().abs()[:, None]
                off = prob * (2 * U * (8 * size + DEEP) + DEEP * U) * (dp.abs() + (prob * dp.abs()).sum(-1, keepdim=True))
                far = (ds[b, h].double() - SCALE * e).abs() - (HALF_STEP[dtype] * 1.01 * SCALE * e.abs() + 2 * SCALE * off + TINY[dtype])
                assert far.max() <= 0, (p, b, h, "dscores over their bound by", far.max().item())
                off += DEEP * U * e.abs()
                for n in range(BUCKETS):   # scattered additions of so many numbers to so few places take seconds
                    here = bucket == n
                    want[n, h] += (e * here).sum()
                    bound[n, h] += (off * here).sum()
        used = want != 0
        assert used.sum() == (BUCKETS - 1) * heads and not used[BUCKETS // 2].any()   # no distance has this bucket
        assert p or torch.all((bound <= 0.05 * want.abs())[used])
        far = (dtable.double() - want).abs() - bound - U * want.abs()
        assert far.max() <= 0, (p, "dtable over its bound by", far.max().item())
