"""The calls of adacomp_sequence.h in 64 bits on the CPU, from their formulas, and how far a kernel may be from them.

Bounds come from the arithmetic, before any run.  U is the rounding of one float32 operation.  An exponential's argument is rounded in a
product or sum or two (its size times U each), the hardware's exponential and reciprocal are off by one unit in the last place (2 U) each.
"""
import math

import torch

import layers_reference as R
from layers_reference import HALF_STEP, TINY, U

KEEP = 64


# ---- embedding ------------------------------------------------------------------------------------------------------

def drop_factors(rows, cols, drop):
    """[rows, cols] of 0 and the factor of what is kept; drop = (p, seed, stream) or None."""
    return R.factors(rows, cols, *drop) if drop else torch.ones(rows, cols, dtype=torch.float64)


def embed_forward(tokens, table, scale, drop=None):
    t = tokens.reshape(-1).long()
    there = (t >= 0) & (t < table.shape[0])
    y = torch.where(there[:, None], table[torch.where(there, t, 0)], torch.zeros((), dtype=table.dtype)) * scale * drop_factors(t.numel(), table.shape[1], drop)
    return y.reshape(*tokens.shape, table.shape[1])


def embed_backward(tokens, dy, vocab, scale, drop=None):
    """(dtable, the sum of its terms' magnitudes, how many terms each token has)"""
    t, up = tokens.reshape(-1).long(), dy.reshape(-1, dy.shape[-1])
    f = drop_factors(*up.shape, drop)
    up = torch.where(f == 0, torch.zeros((), dtype=up.dtype), up * scale * f)
    there = (t >= 0) & (t < vocab)
    out, size = torch.zeros(vocab, up.shape[1], dtype=up.dtype), torch.zeros(vocab, up.shape[1], dtype=up.dtype)
    out.index_add_(0, t[there], up[there])
    size.index_add_(0, t[there], up[there].abs())
    return out, size, torch.bincount(t[there], minlength=vocab)


# ---- gated linear recurrence ----------------------------------------------------------------------------------------

def scan(m, v, first, back=False):
    """h[t] = m[t] h[t -+ 1] + v[t] of [batch, length, channels], from the state `first` on; a place with m = 0 takes nothing over, whatever it is."""
    out, h = torch.empty_like(v), first
    for t in range(v.shape[1] - 1, -1, -1) if back else range(v.shape[1]):
        h = torch.where(m[:, t] == 0, torch.zeros((), dtype=v.dtype), m[:, t] * h) + v[:, t]
        out[:, t] = h
    return out


def shifted(h, first, back=False):
    """The state that each place begins with."""
    return torch.cat([h[:, 1:], first[:, None]], 1) if back else torch.cat([first[:, None], h[:, :-1]], 1)


class Recurrence:
    """Values of both passes, and bounds for a kernel's.  All arguments in 64 bits, gradients of none."""

    def __init__(self, x, forget, out=None, bias=None, first=None, lengths=None, resets=None):
        b, n, c = x.shape
        zero = torch.zeros((), dtype=x.dtype)
        inside = torch.ones(b, n, 1, dtype=torch.bool) if lengths is None else torch.arange(n)[None, :, None] < lengths.clamp(0, n)[:, None, None]
        f = forget if bias is None else forget + bias
        f = torch.where(inside, f, zero)
        self.inside, self.n = inside, n
        self.x = torch.where(inside, x, zero)
        self.first = torch.zeros(b, c, dtype=x.dtype) if first is None else first
        self.on, self.off = torch.sigmoid(f), torch.sigmoid(-f)
        self.rest = torch.where(inside, self.off, zero)
        self.m = torch.where(inside, self.on, zero + 1)
        if resets is not None:
            self.m = torch.where(inside & (resets != 0)[..., None], zero, self.m)
        self.h = scan(self.m, self.rest * self.x, self.first)
        self.last = self.h[:, -1] if n else self.first
        self.before = torch.where(self.m == 0, zero, shifted(self.h, self.first)) if n else self.h
        self.o = None if out is None else torch.where(inside, out, zero)
        self.o_on = torch.ones_like(x) if out is None else torch.sigmoid(self.o)
        self.o_off = None if out is None else torch.sigmoid(-self.o)
        self.y = torch.where(inside, self.o_on * self.h, zero)
        # every place: a relative error of the gates (their argument is a sum and twice part of a product; exponential, sum, reciprocal, product) and a dozen
        # roundings of the scan, of the sum of magnitudes that the state is made of
        self.gate_off = U * (3 * f.abs() + 16)
        self.o_off_by = U * (3 * self.o.abs() + 16) if out is not None else torch.zeros_like(x)
        self.size = scan(self.m, self.rest * self.x.abs(), self.first.abs())
        self.h_off = scan(self.m, self.size * (2 * self.gate_off + 24 * U), torch.zeros_like(self.first))

    def y_bound(self, dtype):
        return torch.where(self.inside, self.o_on * self.h_off + self.o_on * self.size * (self.o_off_by + 4 * U), 0.0) + HALF_STEP[dtype] * 1.01 * self.y.abs() + TINY[dtype]

    def last_bound(self):
        return (self.h_off[:, -1] if self.n else torch.zeros_like(self.first)) + 4 * U * self.last.abs() + TINY[torch.float32]

    def states(self):
        return shifted(self.h, self.first)[:, ::KEEP], shifted(self.h_off, torch.zeros_like(self.first))[:, ::KEEP] + TINY[torch.float32]

    def backward(self, dy, dlast=None):
        """{name: (value, how far float32 arithmetic may be off)}, before a result's own rounding."""
        zero = torch.zeros((), dtype=dy.dtype)
        dy = torch.where(self.inside, dy, zero)
        dlast = torch.zeros_like(self.first) if dlast is None else dlast
        d = dy * self.o_on
        next_m = torch.cat([self.m[:, 1:], torch.ones_like(self.m[:, :1])], 1)
        g, size = scan(next_m, d, dlast, back=True), scan(next_m, d.abs(), dlast.abs(), back=True)
        each = size * (2 * self.gate_off + self.o_off_by + 24 * U)
        g_off = scan(next_m, each, torch.zeros_like(dlast), back=True)
        p_size = torch.where(self.m == 0, zero, shifted(self.size, self.first.abs()))
        p_off = torch.where(self.m == 0, zero, shifted(self.h_off, torch.zeros_like(self.first)))
        both = self.on * self.rest
        spread = p_size + self.x.abs()
        out = {"dx": (self.rest * g, self.rest * (g_off + size * (self.gate_off + 4 * U))),
               "dforget": (both * g * (self.before - self.x), both * (g_off * spread + size * (p_off + spread * (2 * self.gate_off + 8 * U))))}
        if self.o is not None:
            slope = self.o_on * self.o_off
            out["dout"] = (dy * self.h * slope, dy.abs() * slope * (self.h_off + self.size * (2 * self.o_off_by + self.gate_off + 8 * U)))
        df, off = out["dforget"]
        out["dbias"] = (df.sum((0, 1)), off.sum((0, 1)) + U * (self.n + df.shape[0] + 64) * df.abs().sum((0, 1)))
        if self.n:
            out["dfirst"] = (torch.where(self.m[:, 0] == 0, zero, self.m[:, 0] * g[:, 0]), self.m[:, 0] * (g_off[:, 0] + size[:, 0] * (self.gate_off[:, 0] + 4 * U)))
        else:
            out["dfirst"] = (dlast, torch.zeros_like(dlast))
        return {k: (v, b + TINY[torch.float32]) for k, (v, b) in out.items()}


# ---- distillation ---------------------------------------------------------------------------------------------------

class Distill:
    """Loss and gradient of every row, and bounds for a kernel's.  z [rows, vocab], tokens and t [rows, top], targets [rows]."""

    def __init__(self, z, tokens=None, t=None, targets=None, temperature=1.0, soft=1.0, hard=1.0):
        rows, vocab = z.shape
        self.tau, self.soft, self.hard, self.vocab = temperature, soft, hard, vocab
        nothing = torch.zeros(rows, dtype=torch.bool)
        self.taught, self.told = nothing, nothing.clone()
        self.p = torch.zeros_like(z)
        self.one = torch.zeros_like(z)
        self.loss, self.loss_off = torch.zeros(rows, dtype=z.dtype), torch.zeros(rows, dtype=z.dtype)
        self.lse, self.lse_off = torch.zeros(rows, 2, dtype=z.dtype), torch.zeros(rows, 2, dtype=z.dtype)
        # sums: up to 64 values of a thread at once and some for every part of a long row, 6 steps in a wave, 16 waves
        self.deep = 128 + vocab / 128
        s, top = z / temperature, 0
        if tokens is not None and soft > 0:
            top = tokens.shape[1]
            tokens = tokens.long()
            good = (tokens >= 0) & (tokens < vocab)
            scaled = torch.where(good, t / temperature, -math.inf)
            most = scaled.amax(1) if top else torch.full((rows,), -math.inf, dtype=z.dtype)
            self.taught = most > -math.inf
            e = torch.where(self.taught[:, None], torch.exp(scaled - torch.where(self.taught, most, 0.0)[:, None]), 0.0)
            p = e / e.sum(1, keepdim=True).clamp(min=1e-300)
            at = torch.where(good, tokens, 0)
            self.p.scatter_add_(1, at, torch.where(good, p, 0.0))
            lse = torch.logsumexp(s, 1)
            logq = torch.gather(s, 1, at) - lse[:, None]
            terms = torch.where(p > 0, p * (torch.log(p.clamp(min=1e-300)) - logq), 0.0)
            kl = torch.where(torch.isneginf(lse), math.inf, terms.sum(1))
            self.loss = self.loss + torch.where(self.taught, soft * temperature ** 2 * kl, 0.0)
            self.lse[:, 0] = torch.where(self.taught, lse, 0.0)
            self.lse_off[:, 0] = self.off_of_lse(s, lse)
            weight = torch.where(p > 0, p * ((scaled - most[:, None]).abs() + torch.gather(s, 1, at).abs()), 0.0).nan_to_num(0.0, 0.0, 0.0).sum(1)
            spread = torch.where(p > 0, (scaled - most[:, None]).abs(), 0.0).nan_to_num(0.0).amax(1) if top else 0.0
            p_log = torch.log(e.sum(1).clamp(min=1.0))
            self.loss_off = self.loss_off + soft * temperature ** 2 * (self.lse_off[:, 0] + U * (2 * top + 24 + 4 * spread) * (weight + 1) + 4 * U * (p_log + lse.abs().nan_to_num(0.0, 0.0, 0.0)))
            self.p_off = U * (2 * top + 24 + 8 * spread)
        if targets is not None and hard > 0:
            targets = targets.long()
            self.told = (targets >= 0) & (targets < vocab)
            at = torch.where(self.told, targets, 0)
            lse = torch.logsumexp(z, 1)
            ce = torch.where(torch.isneginf(lse), math.inf, lse - torch.gather(z, 1, at[:, None])[:, 0])
            self.loss = self.loss + torch.where(self.told, hard * ce, 0.0)
            self.lse[:, 1] = torch.where(self.told, lse, 0.0)
            self.lse_off[:, 1] = self.off_of_lse(z, lse)
            self.loss_off = self.loss_off + hard * (self.lse_off[:, 1] + 4 * U * (lse.abs() + torch.gather(z, 1, at[:, None])[:, 0].abs()).nan_to_num(0.0, 0.0, 0.0))
            self.one[torch.arange(rows), at] = torch.where(self.told, 1.0, 0.0).to(z.dtype)
        self.loss_off = self.loss_off + 4 * U * self.loss.abs().nan_to_num(0.0, 0.0, 0.0) + TINY[torch.float32]
        self.z, self.s = z, s

    def off_of_lse(self, s, lse):
        """Arguments of exponentials are off by a few U of their size, weighted by the exponentials; then the sum, its logarithm, and lse itself."""
        q = torch.exp(s - torch.where(torch.isneginf(lse), 0.0, lse)[:, None])
        far = torch.where(q > 0, q * (s.amax(1, keepdim=True) - s), 0.0).nan_to_num(0.0, 0.0, 0.0).sum(1)
        return U * (4 * far + self.deep + 12 + 4 * lse.abs().nan_to_num(0.0, 0.0, 0.0) + 2 * s.amax(1).abs().nan_to_num(0.0, 0.0, 0.0))

    def gradient(self, dloss, scale=1.0, from_lse=False):
        """(dlogits, how far off before their own rounding)"""
        g = scale * dloss
        void = ~(self.taught | self.told) | (g == 0)
        out, off = torch.zeros_like(self.z), torch.zeros_like(self.z)
        for there, s, p, lse, weight in ((self.taught, self.s, self.p, self.lse[:, :1], self.soft * self.tau), (self.told, self.z, self.one, self.lse[:, 1:], self.hard)):
            w = torch.where(there, g * weight, 0.0)[:, None]
            q = torch.exp(s - torch.where(torch.isneginf(lse), 0.0, lse))
            arg = (s.amax(1, keepdim=True) - s).nan_to_num(0.0, 0.0, 0.0) + (2 * (s.abs() + lse.abs()).nan_to_num(0.0, 0.0, 0.0) if from_lse else 0.0)
            p_off = self.p_off if p is self.p and hasattr(self, "p_off") else torch.zeros(len(s), dtype=s.dtype)
            out += torch.where(w == 0, 0.0, w * (q - p))
            off += torch.where(w == 0, 0.0, w.abs() * (q * U * (4 * arg + self.deep + 24) + p * (torch.as_tensor(p_off).reshape(-1, 1) + 8 * U)))
        out[void] = 0.0
        off[void] = 0.0
        return out, off + 4 * U * out.abs() + TINY[torch.float32]
