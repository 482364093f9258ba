"""The pieces between the matrix products of a learner's training step, measured.

A case is one call of one operator on one GPU, with its plain form (elementary torch operations in 32 bits) beside it:

  dropout           y = [residual +] D(x), with a mask that a counter-based generator makes and nothing stores
  norm_forward      z = [residual +] D(x), y = layer norm of z; single tokens (serving) and whole mini-batches (training)
  norm_backward     gradients of z and x, and those of gamma and beta summed over all rows
  softmax_forward   probabilities of attention scores with a learned relative position bias, masks and dropout
  softmax_backward  gradients of the scores and of the bias table

The generator is Philox-4x32 with 7 rounds: key = seed, counter = (column / 8, row, stream low, stream high); the four words
are eight halves, low half first, one for each of 8 columns.  With T = floor(p * 65536 + 1/2) a value is kept where its half
is at least T, and multiplied by 65536 / (65536 - T).

Widths come from the repository's own layer tables (hidden layers of 500 and 4096, an LSTM of 512 with its 577 inputs, 5999
outputs of a speech DNN) and are generic otherwise.
"""
import math

import torch

own = False
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-5
SCALE = 0.125   # 1 / sqrt(64), of scores that are products of 64 channels
MOST_NORM = 1 << 26      # rows * cols of a drawn case
MOST_SCORES = 1 << 28    # scores of a drawn case


def listed():
    return [
        # The hidden layer of the MNIST-sized network over a mini-batch of 100: the smallest call, latency counts.
        {"name": "dropout_hidden_500", "op": "dropout", "rows": 100, "cols": 500, "type": "f32", "p": 0.5, "residual": False, "pad": 0},
        # The residual sum of a block as wide as the speech DNN, 16384 frames.
        {"name": "dropout_residual_4096", "op": "dropout", "rows": 16384, "cols": 4096, "type": "bf16", "p": 0.1, "residual": True, "pad": 0},
        # An odd width (the speech DNN's outputs) inside wider rows, another type and rate.
        {"name": "dropout_odd_5999", "op": "dropout", "rows": 5003, "cols": 5999, "type": "f16", "p": 0.25, "residual": False, "pad": 17},
        # Serving: one token, nothing kept for a backward pass.
        {"name": "norm_token_4096", "op": "norm_forward", "rows": 1, "cols": 4096, "type": "bf16", "p": 0.0, "residual": False, "pad": 0, "keep": False},
        # A block's residual sum with dropout and its norm, with what the backward pass needs.
        {"name": "norm_block_4096", "op": "norm_forward", "rows": 16384, "cols": 4096, "type": "bf16", "p": 0.1, "residual": True, "pad": 0, "keep": True},
        # The LSTM's 577 inputs in 32 bits: rows that begin at odd places.
        {"name": "norm_odd_577", "op": "norm_forward", "rows": 6007, "cols": 577, "type": "f32", "p": 0.0, "residual": False, "pad": 0, "keep": True},
        # The backward pass of norm_block_4096, with the gradient that comes down the residual path.
        {"name": "norm_back_block_4096", "op": "norm_backward", "rows": 16384, "cols": 4096, "type": "bf16", "p": 0.1, "residual": True, "pad": 0},
        # The backward pass of norm_odd_577.
        {"name": "norm_back_odd_577", "op": "norm_backward", "rows": 6007, "cols": 577, "type": "f32", "p": 0.0, "residual": False, "pad": 0},
        # Serving: one new token in each of 32 sequences of up to 8193 tokens, each at its own place.
        {"name": "softmax_token_8193", "op": "softmax_forward", "batch": 32, "heads": 16, "queries": 1, "keys": 8193, "type": "bf16", "p": 0.0, "causal": True,
         "ragged": True, "mask": False, "buckets": 32, "distance": 128, "keep": False},
        # Training: sequences of 2048 tokens, causal, with dropout.
        {"name": "softmax_causal_2048", "op": "softmax_forward", "batch": 4, "heads": 16, "queries": 2048, "keys": 2048, "type": "bf16", "p": 0.1, "causal": True,
         "ragged": False, "mask": False, "buckets": 32, "distance": 128, "keep": True},
        # The backward pass over padded sequences that look both ways: the largest call.
        {"name": "softmax_back_2048", "op": "softmax_backward", "batch": 4, "heads": 16, "queries": 2048, "keys": 2048, "type": "bf16", "p": 0.1, "causal": False,
         "ragged": True, "mask": False, "buckets": 32, "distance": 128},
        # Odd lengths, 32 bits, a mask of single places that leaves some rows empty, anything at all in masked places.
        {"name": "softmax_back_odd_777", "op": "softmax_backward", "batch": 6, "heads": 5, "queries": 333, "keys": 777, "type": "f32", "p": 0.0, "causal": False,
         "ragged": True, "mask": True, "buckets": 64, "distance": 250},
    ]


def _log(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    op = rng.choice(("dropout", "norm_forward", "norm_backward", "softmax_forward", "softmax_backward"))
    case = {"op": op, "type": rng.choice(("f32", "bf16", "bf16", "f16")), "p": rng.choice((0.0, 0.1, round(rng.uniform(0.01, 0.6), 3)))}
    if not op.startswith("softmax"):
        if op == "dropout":
            case["p"] = case["p"] or 0.3
        cols = _log(rng, 16, 16384)
        rows = _log(rng, 1, 32768)
        while rows * cols > MOST_NORM:
            rows = (rows + 1) // 2
        case |= {"rows": rows, "cols": cols, "residual": rng.random() < 0.5, "pad": rng.choice((0, 0, 0, 8, rng.randint(1, 40)))}
        if op == "norm_forward":
            case["keep"] = rng.random() < 0.7
        return case
    batch, heads = _log(rng, 1, 32), rng.randint(1, 24)
    if rng.random() < 0.35:
        queries, keys = rng.choice((1, 1, 1, rng.randint(2, 8))), _log(rng, 1, 131072)
    else:
        queries = _log(rng, 16, 4096)
        keys = rng.choice((queries, queries, _log(rng, 16, 8192)))
    while batch * heads * queries * keys > MOST_SCORES:
        if batch > 1:
            batch = (batch + 1) // 2
        elif queries > 16:
            queries = (queries + 1) // 2
        else:
            heads = (heads + 1) // 2
    buckets, distance = rng.choice(((32, 128), (32, 128), (64, 250), (16, 40), (320, 800)))
    case |= {"batch": batch, "heads": heads, "queries": queries, "keys": keys, "causal": rng.random() < 0.5, "ragged": rng.random() < 0.5,
             "mask": rng.random() < 0.25, "buckets": buckets, "distance": distance}
    if op == "softmax_forward":
        case["keep"] = rng.random() < 0.7
    return case


# ---- inputs ---------------------------------------------------------------------------------------------------------

def _rows(g, case, scale=1.0, shift=0.0):
    """A [rows, cols] tensor, a part of wider rows where the case pads."""
    wide = torch.empty(case["rows"], case["cols"] + case["pad"], device=DEV).normal_(generator=g).mul_(scale).add_(shift).to(TYPES[case["type"]])
    return wide[:, :case["cols"]]


def bucket_map(buckets, distance, both_ways):
    """Bucket of every distance key - query in -distance .. distance: a bucket for each of the small ones, logarithmic ones up to
    `distance`; where both directions count, one half of the buckets for each."""
    out = []
    for d in range(-distance, distance + 1):
        count, first, n = buckets, 0, max(0, -d)
        if both_ways:
            count, first, n = buckets // 2, buckets // 2 if d > 0 else 0, abs(d)
        small = count // 2
        if n >= small:
            n = min(count - 1, small + int(math.log(n / small) / math.log(distance / small) * (count - small) + 1e-9))
        out.append(first + n)
    return out


def _inputs(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 1000003 + 17)
    t = TYPES[case["type"]]
    s = {"case": case, "seed": (seed * 0x9E3779B97F4A7C15 + 0x1234567) & (2 ** 63 - 1), "stream": 3 + (seed & 0xFFFF)}
    op = case["op"]
    if op in ("dropout", "norm_forward"):
        s["x"] = _rows(g, case)
        s["residual"] = _rows(g, case, 2.0, 0.25) if case["residual"] else None
    if op.startswith("norm"):
        s["gamma"] = torch.empty(case["cols"], device=DEV).normal_(generator=g).mul_(0.1).add_(1.0)
        s["beta"] = torch.empty(case["cols"], device=DEV).normal_(generator=g).mul_(0.1)
    if op == "norm_backward":
        s["z"] = _rows(g, case, 2.0, 0.25)
        z = s["z"].float()
        s["mean"] = z.mean(dim=1)
        s["rstd"] = torch.rsqrt((z - s["mean"][:, None]).square().mean(dim=1) + EPS)
        s["dy"] = _rows(g, case, 1e-2)
        s["dz_add"] = _rows(g, case, 1e-2) if case["residual"] else None
    if op.startswith("softmax"):
        b, h, q, k = case["batch"], case["heads"], case["queries"], case["keys"]
        s["table"] = torch.empty(case["buckets"], h, device=DEV).normal_(generator=g)
        s["map"] = torch.tensor(bucket_map(case["buckets"], case["distance"], not case["causal"]), dtype=torch.int32, device=DEV)
        s["scores"] = torch.empty(b, h, q, k, device=DEV, dtype=t).normal_(generator=g).mul_(8.0)
        s["lengths"] = s["starts"] = s["mask"] = None
        if case["ragged"]:
            low = max(1, k // 3) if q > 1 or k < 3 else 1
            s["lengths"] = torch.randint(low, k + 1, (b,), generator=g, device=DEV, dtype=torch.int32)
            s["lengths"][0] = k
            if case["causal"]:   # the last of a sequence's tokens are the new ones
                s["starts"] = s["lengths"] - q
        s["start"] = k - q if case["causal"] else 0
        if case["mask"]:   # one for all heads: single places, and now and then a whole row
            m = torch.rand(b, 1, q, k, generator=g, device=DEV) < 0.8
            m &= torch.rand(b, 1, q, 1, generator=g, device=DEV) < 0.95
            s["mask"] = m.to(torch.uint8)
            for part, value in ((0.5, float("nan")), (0.3, float("inf")), (0.2, torch.finfo(t).min)):   # padding holds anything
                wild = (torch.rand(b, 1, q, k, generator=g, device=DEV) < part) & ~m
                s["scores"].masked_fill_(wild, value)
        if op == "softmax_backward":
            s["dprobs"] = torch.empty(b, h, q, k, device=DEV, dtype=t).normal_(generator=g).mul_(1e-2)
            if case["mask"]:
                s["dprobs"].masked_fill_(~m, float("nan"))
            s["lse"] = _lse(s)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if not own:
        return s
    import paper_1712_02679_amd as A
    s["A"], op = A, case["op"]
    s["drop"] = A.Dropout(case["p"], s["seed"], s["stream"]) if case["p"] > 0 else None
    if op in ("dropout", "norm_forward"):
        s["y"] = torch.empty(case["rows"], case["cols"], device=DEV, dtype=TYPES[case["type"]])
        s["z_out"] = s["mean"] = s["rstd"] = None
        if op == "norm_forward" and case["keep"]:
            s["z_out"] = torch.empty_like(s["y"]) if case["residual"] or s["drop"] else None
            s["mean"], s["rstd"] = torch.empty(case["rows"], device=DEV), torch.empty(case["rows"], device=DEV)
    if op == "norm_backward":
        s["dz"] = torch.empty(case["rows"], case["cols"], device=DEV, dtype=TYPES[case["type"]])
        s["dx"] = torch.empty_like(s["dz"]) if s["drop"] else None
        s["dgamma"], s["dbeta"] = torch.empty(case["cols"], device=DEV), torch.empty(case["cols"], device=DEV)
        s["ws"] = torch.empty(A.adacomp_norm_workspace_bytes(case["rows"], case["cols"]), dtype=torch.uint8, device=DEV)
    if op.startswith("softmax"):
        s["bias"] = A.RelativeBias(s["table"], s["map"])
        s["out"] = torch.empty_like(s["scores"])
        s["lse_out"] = torch.empty(s["scores"].shape[:3], device=DEV) if case.get("keep") else None
        s["dtable"] = torch.empty_like(s["table"])
        n = A.adacomp_bias_softmax_workspace_bytes(case["batch"], case["heads"], case["queries"], case["keys"], case["distance"])
        s["ws"] = torch.empty(n, dtype=torch.uint8, device=DEV)
    return s


# ---- the framework's calls ------------------------------------------------------------------------------------------

def _calls(s):
    A, case = s["A"], s["case"]
    op = case["op"]
    if op == "dropout":
        A.adacomp_dropout(s["x"], s["y"], s["drop"], residual=s["residual"])
        return [s["y"]]
    if op == "norm_forward":
        A.adacomp_norm_forward(s["x"], s["gamma"], s["beta"], s["y"], residual=s["residual"], dropout=s["drop"], z=s["z_out"], mean=s["mean"],
                               rstd=s["rstd"], eps=EPS)
        return [v for v in (s["y"], s["z_out"], s["mean"], s["rstd"]) if v is not None]
    if op == "norm_backward":
        A.adacomp_norm_backward(s["dy"], s["z"], s["mean"], s["rstd"], s["gamma"], s["dz"], s["dgamma"], s["dbeta"], s["ws"], dz_add=s["dz_add"],
                                dropout=s["drop"], dx=s["dx"])
        return [v for v in (s["dz"], s["dx"], s["dgamma"], s["dbeta"]) if v is not None]
    if op == "softmax_forward":
        A.adacomp_bias_softmax_forward(s["scores"], s["bias"], s["out"], s["ws"], lse=s["lse_out"], scale=SCALE, causal=case["causal"],
                                       query_start=s["start"], query_starts=s["starts"], key_lengths=s["lengths"], mask=s["mask"], dropout=s["drop"])
        return [v for v in (s["out"], s["lse_out"]) if v is not None]
    A.adacomp_bias_softmax_backward(s["scores"], s["bias"], s["lse"], s["dprobs"], s["out"], s["dtable"], s["ws"], scale=SCALE, causal=case["causal"],
                                    query_start=s["start"], query_starts=s["starts"], key_lengths=s["lengths"], mask=s["mask"], dropout=s["drop"])
    return [s["out"], s["dtable"]]


# ---- the plain forms ------------------------------------------------------------------------------------------------

def _kept(rows, cols, s):
    """(truth values [rows, cols], factor) of the generator."""
    low = 0xFFFFFFFF
    k0, k1 = s["seed"] & low, s["seed"] >> 32
    c0 = torch.arange((cols + 7) // 8, device=DEV)[None, :]
    c1 = torch.arange(rows, device=DEV)[:, None]
    c2 = torch.full((1, 1), s["stream"] & low, dtype=torch.int64, device=DEV)
    c3 = torch.full((1, 1), s["stream"] >> 32, dtype=torch.int64, device=DEV)
    for _ in range(7):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((b >> 32) & low) ^ c1 ^ k0, b & low, ((a >> 32) & low) ^ c3 ^ k1, a & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    halves = torch.stack([half for w in (c0, c1, c2, c3) for half in (w & 0xFFFF, w >> 16)], dim=-1)
    t = math.floor(s["case"]["p"] * 65536 + 0.5)
    return halves.reshape(rows, -1)[:, :cols] >= t, 65536.0 / (65536.0 - t)


def _drop(x, s):
    """D(x) of a tensor whose last dimension are the columns."""
    if not s["case"]["p"] > 0:
        return x
    keep, factor = _kept(x.numel() // x.shape[-1], x.shape[-1], s)
    return torch.where(keep.view(x.shape), x * factor, 0.0)


def _admitted(s):
    """(places key - query, truth values of what a row may look at), both broadcast over [batch, heads, queries, keys]."""
    case = s["case"]
    i, j = torch.arange(case["queries"], device=DEV)[:, None], torch.arange(case["keys"], device=DEV)[None, :]
    start = s["starts"].long()[:, None, None, None] if s["starts"] is not None else s["start"]
    d = (j - i)[None, None] - start
    ok = torch.ones_like(d, dtype=torch.bool)
    if case["causal"]:
        ok = ok & (d <= 0)
    if s["lengths"] is not None:
        ok = ok & (j < s["lengths"][:, None, None, None])
    if s["mask"] is not None:
        ok = ok & (s["mask"] != 0)
    return d, ok


def _biased(s):
    """(scores with their bias, -inf where not admitted; buckets)"""
    case = s["case"]
    d, ok = _admitted(s)
    bucket = s["map"].long()[d.clamp(-case["distance"], case["distance"]) + case["distance"]]   # [batch or 1, 1, queries, keys]
    bias = s["table"][bucket[:, 0]].permute(0, 3, 1, 2)
    return torch.where(ok, s["scores"].float() * SCALE + bias, -torch.inf), bucket


def _lse(s):
    """Logarithm of every row's sum of exponentials; -inf for a row without any."""
    t, _ = _biased(s)
    top = t.amax(dim=-1, keepdim=True)
    top = torch.where(torch.isinf(top) & (top < 0), 0.0, top)
    return (torch.log(torch.exp(t - top).sum(dim=-1, keepdim=True)) + top)[..., 0]


def _plain(s):
    case = s["case"]
    op, t = case["op"], TYPES[case["type"]]
    if op in ("dropout", "norm_forward"):
        z = _drop(s["x"].float(), s)
        if s["residual"] is not None:
            z = s["residual"].float() + z
        if op == "dropout":
            return [z.to(t)]
        mean = z.mean(dim=1, keepdim=True)
        centred = z - mean
        rstd = torch.rsqrt(centred.square().mean(dim=1, keepdim=True) + EPS)
        out = [(centred * rstd * s["gamma"] + s["beta"]).to(t)]
        if case["keep"]:
            out += [z.to(t)] if case["residual"] or case["p"] > 0 else []
            out += [mean[:, 0], rstd[:, 0]]
        return out
    if op == "norm_backward":
        dy, h = s["dy"].float(), (s["z"].float() - s["mean"][:, None]) * s["rstd"][:, None]
        g = dy * s["gamma"]
        dz = s["rstd"][:, None] * (g - g.mean(dim=1, keepdim=True) - h * (g * h).mean(dim=1, keepdim=True))
        if s["dz_add"] is not None:
            dz = dz + s["dz_add"].float()
        out = [dz.to(t)] + ([_drop(dz, s).to(t)] if case["p"] > 0 else [])
        return out + [(dy * h).sum(dim=0), dy.sum(dim=0)]
    if op == "softmax_forward":
        x, _ = _biased(s)
        top = x.amax(dim=-1, keepdim=True)
        top = torch.where(torch.isinf(top) & (top < 0), 0.0, top)
        e = torch.exp(x - top)
        total = e.sum(dim=-1, keepdim=True)
        probs = torch.where(total > 0, e / total, 0.0)
        out = [_drop(probs, s).to(t)]
        return out + ([(torch.log(total) + top)[..., 0]] if case["keep"] else [])
    x, bucket = _biased(s)
    lse = s["lse"][..., None]
    probs = torch.where(torch.isinf(lse) & (lse < 0), 0.0, torch.exp(x - lse))
    dp = torch.where(probs > 0, _drop(s["dprobs"].float(), s), 0.0)
    ds = probs * (dp - (probs * dp).sum(dim=-1, keepdim=True))
    dtable = [torch.where(bucket == n, ds, 0.0).sum(dim=(0, 2, 3)) for n in range(case["buckets"])]
    return [(ds * SCALE).to(t), torch.stack(dtable)]


def run(state):
    return _calls(state) if own else _plain(state)


# ---- what a pass cannot do without ----------------------------------------------------------------------------------

def _share(case):
    """The share of the scores that causal rows admit."""
    q, k = case["queries"], case["keys"]
    if not case["causal"]:
        return 1.0
    return sum(max(0, min(k, k - q + i + 1)) for i in range(q)) / (q * k)


def work(case):
    size = 4 if case["type"] == "f32" else 2
    if not case["op"].startswith("softmax"):
        n, cols, rows = case["rows"] * case["cols"], case["cols"], case["rows"]
        streams = {"dropout": 2 + case["residual"], "norm_forward": 2 + case["residual"], "norm_backward": 3 + case["residual"] + (case["p"] > 0)}[case["op"]]
        more = 0
        if case["op"] == "norm_forward":
            more = 8 * cols
            if case["keep"]:
                streams += bool(case["residual"] or case["p"] > 0)
                more += 8 * rows
        if case["op"] == "norm_backward":
            more = 12 * cols + 8 * rows
        return {"bytes": n * size * streams + more, "flops": n * {"dropout": 2, "norm_forward": 9, "norm_backward": 16}[case["op"]]}
    rows = case["batch"] * case["heads"] * case["queries"]
    n = rows * case["keys"]
    read = n * _share(case) * (2 / 3 if case["ragged"] else 1.0)   # padding is not read: two thirds of the places on average
    back = case["op"] == "softmax_backward"
    total = int(read * size * (2 if back else 1)) + n * size + (4 * rows if back or case["keep"] else 0)
    if case["mask"]:
        total += n // case["heads"]
    return {"bytes": total, "flops": int(read * (12 if back else 7))}


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------

def _halves64(rows, cols, s):
    """The generator once more, with products in 16-bit parts: factors [rows, cols] that are 0 or the survivors'."""
    p = s["case"]["p"]
    if not p > 0:
        return 1.0

    def product(m, c):
        """High and low word of m * c."""
        mh, ml, ch, cl = m >> 16, m & 65535, c >> 16, c & 65535
        low, cross = ml * cl, mh * cl + (ml * ch & 65535) * 1
        mid = (low >> 16) + (cross & 65535)
        high = mh * ch + (ml * ch >> 16) + (cross >> 16) + (mid >> 16)
        return high & 0xFFFFFFFF, ((mid & 65535) << 16) | (low & 65535)

    col, row = torch.arange(cols, device=DEV), torch.arange(rows, device=DEV)
    x = [(col // 8).repeat(rows, 1)[:, ::8].contiguous(), row[:, None], torch.tensor(s["stream"] % 2 ** 32, device=DEV), torch.tensor(s["stream"] // 2 ** 32, device=DEV)]
    for r in range(7):
        key = [(s["seed"] % 2 ** 32 + r * 0x9E3779B9) % 2 ** 32, (s["seed"] // 2 ** 32 + r * 0xBB67AE85) % 2 ** 32]
        (h0, l0), (h2, l2) = product(0xD2511F53, x[0]), product(0xCD9E8D57, x[2])
        x = [h2 ^ x[1] ^ key[0], l2, h0 ^ x[3] ^ key[1], l0]
    t = int(p * 65536 + 0.5)
    out = torch.empty(rows, cols, dtype=torch.float64, device=DEV)
    for c in range(min(8, cols)):
        word = x[c // 2] >> 16 * (c % 2) & 65535
        out[:, c::8] = torch.where(word < t, 0.0, 65536.0 / (65536 - t))[:, :out[:, c::8].shape[1]]
    return out


def exact(case, seed):
    s = _inputs(case, seed)
    op = case["op"]
    if not op.startswith("softmax"):
        n, factor = case["cols"], _halves64(case["rows"], case["cols"], s)
        if op == "norm_backward":
            dy, z = s["dy"].double(), s["z"].double()
            h = (z - s["mean"].double().unsqueeze(1)) * s["rstd"].double().unsqueeze(1)
            g = s["gamma"].double() * dy
            inner = n * g - g.sum(1, True) - h * (g * h).sum(1, True)
            dz = inner * (s["rstd"].double() / n).unsqueeze(1)
            if s["dz_add"] is not None:
                dz += s["dz_add"].double()
            return [dz] + ([dz * factor] if case["p"] > 0 else []) + [(dy * h).sum(0), dy.sum(0)]
        z = s["x"].double() * factor + (0.0 if s["residual"] is None else s["residual"].double())
        if op == "dropout":
            return [z]
        var, mean = torch.var_mean(z, dim=1, correction=0)
        rstd = 1.0 / torch.sqrt(var + EPS)
        out = [torch.addcmul(s["beta"].double(), (z - mean[:, None]) * rstd[:, None], s["gamma"].double())]
        if case["keep"]:
            out += [z] if case["residual"] or case["p"] > 0 else []
            out += [mean, rstd]
        return out
    b, h, q, k = (case[n] for n in ("batch", "heads", "queries", "keys"))
    first = torch.empty(b, h, q, k, dtype=torch.float64, device=DEV)
    lse = torch.empty(b, h, q, dtype=torch.float64, device=DEV)
    dtable = torch.zeros(case["buckets"], h, dtype=torch.float64, device=DEV)
    key, far = torch.arange(k, device=DEV), case["distance"]
    for n in range(b):
        at = (int(s["starts"][n]) if s["starts"] is not None else s["start"]) + torch.arange(q, device=DEV)
        away = key.unsqueeze(0) - at.unsqueeze(1)
        hidden = torch.zeros(q, k, dtype=torch.bool, device=DEV)
        if case["causal"]:
            hidden |= away > 0
        if s["lengths"] is not None:
            hidden |= (key >= int(s["lengths"][n])).unsqueeze(0)
        if s["mask"] is not None:
            hidden |= s["mask"][n, 0] == 0
        which = s["map"].long()[torch.where(away < -far, -far, torch.where(away > far, far, away)) + far]
        for m in range(h):
            t = SCALE * s["scores"][n, m].double() + s["table"][:, m].double()[which]
            t[hidden] = -math.inf
            lse[n, m] = torch.logsumexp(t, dim=1)
            if op == "softmax_forward":
                first[n, m] = torch.nan_to_num(torch.softmax(t, dim=1), nan=0.0)
                continue
            probs = torch.exp(t - s["lse"][n, m].double().unsqueeze(1))
            probs[torch.isneginf(s["lse"][n, m])] = 0.0
            first[n, m] = probs
    factor = _halves64(b * h * q, k, s) if case["p"] > 0 else None
    if op == "softmax_forward":
        if factor is not None:
            first *= factor.view(b, h, q, k)
        return [first] + ([lse] if case["keep"] else [])
    for n in range(b):
        at = (int(s["starts"][n]) if s["starts"] is not None else s["start"]) + torch.arange(q, device=DEV)
        which = s["map"].long()[(key.unsqueeze(0) - at.unsqueeze(1)).clamp_(-far, far) + far].flatten()
        for m in range(h):
            up = s["dprobs"][n, m].double()
            up[first[n, m] == 0] = 0.0
            if factor is not None:
                up = up * factor.view(b, h, q, k)[n, m]
            up = (up - (up * first[n, m]).sum(1, True)) * first[n, m]
            first[n, m] = up * SCALE
            dtable[:, m] += torch.bincount(which, weights=up.flatten(), minlength=case["buckets"])
    return [first, dtable]
