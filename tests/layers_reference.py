"""The calls of adacomp_layers.h in 64 bits on the CPU, from their formulas, and how far a kernel may be from them.

Bounds come from the arithmetic, before any run: U is the rounding of one float32 operation, DEEP the longest chain of
float32 additions behind a sum over a row or over rows (32 values of a thread, 6 steps in a wave, 16 waves, or for sums over rows the
rows of one thread, the rows side by side in a workgroup, 32 slices of workgroups), with room for the few operations around it.
"""
import math

import numpy as np
import torch

U = 2.0 ** -24
DEEP = 160
HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}   # of a result's own rounding
TINY = {torch.float32: 2.0 ** -126, torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -25}      # where the type has no more digits


def philox(counter, key, rounds):
    """Philox-4x32 of uint64 arrays that hold 32-bit words."""
    low = np.uint64(0xFFFFFFFF)
    c = [np.asarray(x, np.uint64) for x in counter]
    k = [int(x) for x in key]
    for _ in range(rounds):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), b & low, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), a & low]
        k = [(k[0] + 0x9E3779B9) % 2 ** 32, (k[1] + 0xBB67AE85) % 2 ** 32]
    return c


def factors(rows, cols, p, seed, stream, first_row=0):
    """[rows, cols] of 0 and the factor of what is kept."""
    groups = np.arange((cols + 7) // 8, dtype=np.uint64)[None, :]
    row = np.arange(first_row, first_row + rows, dtype=np.uint64)[:, None]
    words = philox((groups + 0 * row, row + 0 * groups, stream % 2 ** 32, stream // 2 ** 32), (seed % 2 ** 32, seed // 2 ** 32), 7)
    halves = np.stack([h for w in np.broadcast_arrays(*words) for h in (w & np.uint64(0xFFFF), w >> np.uint64(16))], axis=-1)
    t = math.floor(float(np.float32(p)) * 65536 + 0.5)
    kept = halves.reshape(rows, -1)[:, :cols] >= t
    return torch.from_numpy(np.where(kept, 65536.0 / (65536 - t), 0.0))


def norm_forward(z, gamma, beta, eps):
    """(y, mean, rstd) of rows."""
    mean = z.mean(-1, keepdim=True)
    rstd = 1.0 / torch.sqrt(((z - mean) ** 2).mean(-1, keepdim=True) + eps)
    return (z - mean) * rstd * gamma + beta, mean[..., 0], rstd[..., 0]


def norm_backward(dy, z, mean, rstd, gamma):
    """(dz, dgamma, dbeta)."""
    h = (z - mean[..., None]) * rstd[..., None]
    g = dy * gamma
    dz = rstd[..., None] * (g - g.mean(-1, keepdim=True) - h * (g * h).mean(-1, keepdim=True))
    over = tuple(range(dy.dim() - 1))
    return dz, (dy * h).sum(over), dy.sum(over)


def places(batch, queries, keys, starts):
    """key - query, [batch, queries, keys]."""
    at = torch.as_tensor(starts, dtype=torch.int64).expand(batch)[:, None, None] + torch.arange(queries)[None, :, None]
    return torch.arange(keys)[None, None, :] - at


def admitted(batch, heads, queries, keys, starts, causal, lengths, mask):
    ok = torch.ones(batch, heads, queries, keys, dtype=torch.bool)
    if causal:
        ok &= (places(batch, queries, keys, starts) <= 0)[:, None]
    if lengths is not None:
        ok &= (torch.arange(keys)[None, :] < lengths[:, None])[:, None, None, :]
    if mask is not None:
        ok &= mask.expand(batch, heads, queries, keys) != 0
    return ok


def biased(scores, table, bucket_map, scale, starts, ok):
    """t, -infinity where not admitted; and every place's bucket."""
    b, h, q, k = scores.shape
    far = len(bucket_map) // 2
    bucket = torch.as_tensor(bucket_map).long().clamp(0, table.shape[0] - 1)[places(b, q, k, starts).clamp(-far, far) + far]
    t = scale * scores + table[bucket].permute(0, 3, 1, 2)
    return torch.where(ok, t, -math.inf), bucket


def softmax_forward(t):
    """(P, lse); zeros and -infinity for rows without anything."""
    lse = torch.logsumexp(t, -1) if t.shape[-1] else torch.full(t.shape[:-1], -math.inf, dtype=t.dtype)
    return torch.where(torch.isneginf(t), 0.0, torch.exp(t - torch.where(torch.isneginf(lse), 0.0, lse)[..., None])), lse


def softmax_backward(p, dp, bucket, n_buckets):
    """(e, dtable [n_buckets, heads]) of e = P (dP - sum P dP)."""
    e = p * (dp - (p * dp).sum(-1, keepdim=True))
    dtable = torch.zeros(n_buckets, p.shape[1], dtype=p.dtype)
    dtable.index_add_(0, bucket.reshape(-1), e.permute(0, 2, 3, 1).reshape(-1, p.shape[1]))
    return e, dtable


def within(got, want, bound, what):
    """|got - want| <= bound everywhere, and the same infinities and NaN."""
    got, want = got.detach().cpu().double(), want.double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what
    assert torch.equal(got[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)]), what
    off = (got - want).abs()[fine] - torch.as_tensor(bound, dtype=torch.float64).expand(want.shape)[fine]
    assert off.numel() == 0 or off.max() <= 0, (what, "over its bound by", off.max().item(), "at", int(off.argmax()), "of", off.numel())
