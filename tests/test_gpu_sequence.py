"""Embedding, gated linear recurrence and distillation on the GPU against their formulas in 64 bits (sequence_reference.py), at the sizes,
types, strides and masks where a kernel can go wrong.  Every bound follows from the arithmetic."""
import numpy as np
import pytest
import torch

import sequence_reference as S
from layers_reference import HALF_STEP, TINY, U, within

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16, F16 = TYPES = [torch.float32, torch.bfloat16, torch.float16]


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
    wide = part._base
    assert torch.all(wide[..., :lead] == 3.0) and torch.all(wide[..., wide.shape[-1] - pad:] == 3.0)


def room(n):
    """A workspace with what an earlier call may have left."""
    return torch.full((n,), 0xA5, dtype=torch.uint8, device=DEV)


def rounded(value, off, dtype):
    return off + HALF_STEP[dtype] * 1.01 * value.abs() + TINY[dtype]


# ---- embedding ------------------------------------------------------------------------------------------------------

def tokens_of(rows, vocab, seed, skew=1.0):
    """Tokens of falling frequencies, a few that are none."""
    g = torch.Generator().manual_seed(seed)
    t = (torch.rand(rows, generator=g, dtype=torch.float64) ** skew * vocab).long().clamp(max=vocab - 1)
    for i, none in zip(range(3, rows, 17), (-1, vocab, -100, 2 ** 31 - 1, -2 ** 31)):
        t[i] = none
    return t


def embed_room(A, rows, vocab, cols):
    return room(A.adacomp_embed_workspace_bytes(rows, vocab, cols))


EMBED_SIZES = [(1, 1, 1, 0, 0), (1, 5999, 4096, 0, 0), (5, 3, 7, 0, 0), (64, 65, 8, 0, 0), (1000, 65, 512, 0, 0), (333, 1000, 577, 3, 1), (2049, 257, 65, 0, 0),
               (300, 70000, 33, 0, 0), (4097, 511, 1001, 1, 2), (130, 40, 2056, 0, 0), (77, 9, 9000, 0, 0), (20000, 7, 16, 0, 0)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab,cols,pad,lead", EMBED_SIZES)
def test_embed_forward(A, rows, vocab, cols, pad, lead, dtype):
    table, scale = rand((vocab, cols), F32, 1), float(np.float32(5.7))
    for index, drop in ((torch.int64, None), (torch.int32, (0.3, 2 ** 62 + 5, 2 ** 33 + 1))):
        tokens = tokens_of(rows, vocab, 2).to(index)
        y = on_gpu(torch.zeros(rows, cols, dtype=dtype), pad, lead)
        A.adacomp_embed_forward(tokens.to(DEV), table.to(DEV), y, scale=scale, dropout=A.Dropout(*drop) if drop else None)
        want = S.embed_forward(tokens, table.double(), scale, drop)
        within(y, want, rounded(want, 4 * U * want.abs(), dtype), (index, drop))
        if pad or lead:
            untouched(y, pad, lead)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab,cols,pad,lead", EMBED_SIZES)
def test_embed_backward(A, rows, vocab, cols, pad, lead, dtype):
    dy, scale = rand((rows, cols), dtype, 3), float(np.float32(0.37))
    gdy, ws = on_gpu(dy, pad, lead), embed_room(A, rows, vocab, cols)
    for index, drop, skew in ((torch.int64, None, 1.0), (torch.int32, (0.3, 2 ** 62 + 5, 2 ** 33 + 1), 6.0)):
        tokens = tokens_of(rows, vocab, 4, skew).to(index)
        want, size, count = S.embed_backward(tokens, dy.double(), vocab, scale, drop)
        for accumulate in (False, True):
            before = rand((vocab, cols), F32, 5)
            got = before.to(DEV)
            A.adacomp_embed_backward(tokens.to(DEV), gdy, got, ws, scale=scale, dropout=A.Dropout(*drop) if drop else None, accumulate=accumulate)
            total = want + before.double() if accumulate else want
            bound = U * ((count + 8).double()[:, None] * size + 2 * total.abs()) + TINY[F32]
            within(got, total, bound, (index, drop, accumulate))
            if accumulate:
                assert torch.equal(got.cpu()[count == 0], before[count == 0])
            else:
                assert torch.all(got.cpu()[count == 0] == 0)


def test_embed_backward_of_one_token_and_of_none(A):
    """All places hold one token, or none do, or there are no places."""
    dy = rand((5000, 40), BF16, 6)
    for tokens, what in ((torch.full((5000,), 11), "one"), (torch.full((5000,), -1), "none")):
        got = torch.full((300, 40), 9.0, device=DEV)
        A.adacomp_embed_backward(tokens.to(DEV), dy.to(DEV), got, embed_room(A, 5000, 300, 40))
        want, size, _ = S.embed_backward(tokens, dy.double(), 300, 1.0)
        within(got, want, U * 5010 * size + TINY[F32], what)
    got = torch.full((300, 40), 9.0, device=DEV)
    A.adacomp_embed_backward(torch.zeros(0, dtype=torch.int64, device=DEV), torch.zeros(0, 40, device=DEV), got, embed_room(A, 0, 300, 40))
    assert torch.all(got == 0)
    A.adacomp_embed_backward(torch.zeros(0, dtype=torch.int64, device=DEV), torch.zeros(0, 40, device=DEV), got.fill_(2.0), embed_room(A, 0, 300, 40), accumulate=True)
    assert torch.all(got == 2.0)
    A.adacomp_embed_forward(torch.zeros(0, dtype=torch.int64, device=DEV), got, torch.zeros(0, 40, device=DEV))


def test_embed_calls_repeat_bit_for_bit(A):
    tokens, dy = tokens_of(30000, 900, 7, 4.0).to(DEV), rand((30000, 200), F32, 8).to(DEV)
    ws, first = embed_room(A, 30000, 900, 200), None
    for _ in range(4):
        got = torch.empty(900, 200, device=DEV)
        A.adacomp_embed_backward(tokens, dy, got, ws)
        first = got if first is None else first
        assert torch.equal(got, first)


def test_embed_into_the_flat_gradient_and_of_shaped_tokens(A):
    """The table and its gradient are parts of flat buffers at odd places; tokens have two dimensions."""
    vocab, cols = 123, 45
    flat, grad = rand(vocab * cols + 11, F32, 9).to(DEV), torch.full((vocab * cols + 11,), 4.0, device=DEV)
    table, dtable = flat[5:5 + vocab * cols].view(vocab, cols), grad[5:5 + vocab * cols].view(vocab, cols)
    tokens, y, dy = tokens_of(60, vocab, 10).view(4, 15), torch.empty(4, 15, cols, dtype=F16, device=DEV), rand((4, 15, cols), F16, 11)
    A.adacomp_embed_forward(tokens.to(DEV), table, y)
    want = S.embed_forward(tokens, table.cpu().double(), 1.0)
    within(y, want, rounded(want, 4 * U * want.abs(), F16), "y")
    A.adacomp_embed_backward(tokens.to(DEV), dy.to(DEV), dtable, embed_room(A, 60, vocab, cols))
    want, size, count = S.embed_backward(tokens, dy.double(), vocab, 1.0)
    within(dtable, want, U * ((count + 8).double()[:, None] * size) + TINY[F32], "dtable")
    assert torch.all(grad[:5] == 4.0) and torch.all(grad[-6:] == 4.0)


def test_embed_dropped_values_may_be_anything(A):
    dy = torch.full((50, 64), float("nan"))
    f = S.drop_factors(50, 64, (0.5, 3, 4))
    dy[f != 0] = 1.0
    tokens = tokens_of(50, 9, 12)
    got = torch.empty(9, 64, device=DEV)
    A.adacomp_embed_backward(tokens.to(DEV), dy.to(DEV), got, embed_room(A, 50, 9, 64), dropout=A.Dropout(0.5, 3, 4))
    want, size, count = S.embed_backward(tokens, dy.double(), 9, 1.0, (0.5, 3, 4))
    within(got, want, U * (count + 8).double()[:, None] * size + TINY[F32], "dtable")


def test_embed_refusals(A):
    table, y, tokens, ws = torch.zeros(10, 8, device=DEV), torch.zeros(4, 8, device=DEV), torch.zeros(4, dtype=torch.int64, device=DEV), room(4096)
    for args in ((tokens.cpu(), table, y), (tokens.float(), table, y), (tokens, table.half(), y), (tokens, table.cpu(), y), (tokens, table.t(), y), (tokens, table, y[:, :7]),
                 (tokens[:3], table, y), (tokens, table, y.double()), (tokens, table, torch.zeros(8, 4, device=DEV).t()), (tokens.repeat(2)[::2], table, y)):
        with pytest.raises(A.AdacompError):
            A.adacomp_embed_forward(*args)
        with pytest.raises(A.AdacompError):
            A.adacomp_embed_backward(args[0], args[2], args[1], ws)
    with pytest.raises(A.AdacompError):
        A.adacomp_embed_backward(tokens, y, table, ws[:16])
    with pytest.raises(A.AdacompError):
        A.adacomp_embed_backward(tokens, y, table, ws.cpu())


# ---- gated linear recurrence ----------------------------------------------------------------------------------------

def recurrence_case(b, n, c, dtype, gate, bias, first, ragged, resets, seed, spread=1.0):
    x, forget, out = (rand((b, n, c), dtype, seed + i, spread) for i in range(3))
    g = torch.Generator().manual_seed(seed + 9)
    s = {"x": x, "forget": forget, "out": out if gate else None, "bias": rand((c,), F32, seed + 3, 1.5, 2.0) if bias else None,
         "first": rand((b, c), F32, seed + 4) if first else None, "lengths": None, "resets": None}
    if ragged:
        s["lengths"] = torch.randint(0, n + 1, (b,), generator=g, dtype=torch.int32)
        s["lengths"][0] = n
        if b > 1:
            s["lengths"][1] = min(1, n)
        if b > 2:
            s["lengths"][2] = 0
    if resets:
        s["resets"] = (torch.rand(b, n, generator=g) < 0.1).to(torch.uint8)
    return s


def wide(s):
    return {k: v.double() if v is not None and v.dtype.is_floating_point else v for k, v in s.items()}


def run_forward(A, s, dtype, pad=0, lead=0):
    b, n, c = s["x"].shape
    put = lambda name: on_gpu(s[name], pad, lead) if name in ("x", "forget", "out") else on_gpu(s[name])
    g = {name: put(name) for name in s}
    g["y"] = on_gpu(torch.full((b, n, c), float("nan"), dtype=dtype), pad, lead)
    g["last"] = torch.full((b, c), float("nan"), device=DEV)
    g["states"] = torch.full((b, A.adacomp_recurrence_kept(n), c), float("nan"), device=DEV)
    g["ws"] = room(A.adacomp_recurrence_workspace_bytes(b, n, c))
    A.adacomp_recurrence_forward(g["x"], g["forget"], g["y"], g["ws"], out=g["out"], bias=g["bias"], first=g["first"], last=g["last"], states=g["states"],
                                 lengths=g["lengths"], resets=g["resets"])
    return g


def check_states(got, r):
    want, off = r.states()
    within(got, want, off + 4 * U * want.abs(), "states")


def check_both(A, s, dtype, pad=0, lead=0, accumulate=False):
    b, n, c = s["x"].shape
    r = S.Recurrence(**wide(s))
    g = run_forward(A, s, dtype, pad, lead)
    within(g["y"], r.y, r.y_bound(dtype), "y")
    within(g["last"], r.last, r.last_bound(), "last")
    check_states(g["states"], r)
    dy, dlast = rand((b, n, c), dtype, 77), rand((b, c), F32, 78)
    want = r.backward(dy.double(), dlast.double())
    fresh = lambda: on_gpu(torch.full((b, n, c), float("nan"), dtype=dtype), pad, lead)
    got = {"dx": fresh(), "dforget": fresh(), "dout": fresh() if s["out"] is not None else None, "dfirst": torch.full((b, c), float("nan"), device=DEV)}
    before = rand((c,), F32, 79)
    got["dbias"] = before.to(DEV)
    A.adacomp_recurrence_backward(on_gpu(dy, pad, lead), g["x"], g["forget"], g["states"], got["dx"], got["dforget"], g["ws"], out=g["out"], dout=got["dout"],
                                  bias=g["bias"], dbias=got["dbias"], dlast=on_gpu(dlast), dfirst=got["dfirst"], lengths=g["lengths"], resets=g["resets"],
                                  accumulate=accumulate)
    for name, (value, off) in want.items():
        if name == "dbias" and accumulate:
            value = value + before.double()
        within(got[name], value, rounded(value, off, dtype if name in ("dx", "dforget", "dout") else F32), name)
    if pad or lead:
        for t in (g["y"], got["dx"], got["dforget"]):
            untouched(t, pad, lead)
    return g, got


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("length", [1, 2, 3, 7, 8, 9, 15, 16, 17, 31, 33, 63, 64, 65, 100, 127, 128, 129, 255, 256, 257, 300, 513])
def test_recurrence_lengths(A, length, dtype):
    check_both(A, recurrence_case(3, length, 70, dtype, True, True, True, False, False, length), dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("channels", [1, 2, 3, 4, 5, 7, 8, 15, 16, 60, 63, 64, 65, 67, 128, 130, 577])
def test_recurrence_channels(A, channels, dtype):
    check_both(A, recurrence_case(2, 75, channels, dtype, channels % 2 == 1, True, True, channels % 3 == 0, channels % 4 == 1, channels), dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("batch,length,channels", [(3, 1, 1), (3, 1, 2), (5, 2, 3), (4, 5, 5), (3, 12, 67), (7, 11, 130), (700, 13, 6), (3400, 66, 5)])
def test_recurrence_place_by_place(A, batch, length, channels, dtype):
    """Calls whose threads take sequences from their first place to the last: short ones, and very many."""
    check_both(A, recurrence_case(batch, length, channels, dtype, channels % 2 == 1, True, True, channels != 2, channels in (1, 5, 67), 21), dtype, pad=channels % 3, lead=channels % 2)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("gate,bias,first,ragged,resets", [(False, False, False, False, False), (True, False, True, False, False), (False, True, False, True, False),
                                                           (True, True, True, True, True), (False, True, True, False, True)])
def test_recurrence_forms(A, gate, bias, first, ragged, resets, dtype):
    for b, n, c, pad, lead in ((5, 150, 66, 3, 1), (4, 40, 12, 0, 0), (1, 700, 33, 0, 0)):
        check_both(A, recurrence_case(b, n, c, dtype, gate, bias, first, ragged, resets, 5), dtype, pad, lead, accumulate=bias)


@pytest.mark.parametrize("batch,length,channels", [(1, 4000, 64), (1, 9000, 20), (2, 2500, 130), (40, 200, 100), (300, 20, 70)])
def test_recurrence_shapes(A, batch, length, channels):
    """Long sequences of few channels, many sequences of few places."""
    check_both(A, recurrence_case(batch, length, channels, BF16, True, True, True, batch > 2, length == 2500, 6), BF16)
    check_both(A, recurrence_case(batch, length, channels, F32, False, True, False, True, length == 9000, 7), F32)


def test_recurrence_of_gates_side_by_side(A):
    """x, forget and out as one product leaves them, their gradients into one buffer, and time before batch."""
    b, n, c = 3, 90, 40
    wide_, grads = rand((b, n, 3 * c), BF16, 1).to(DEV), torch.full((b, n, 3 * c), float("nan"), dtype=BF16, device=DEV)
    x, forget, out = wide_.chunk(3, dim=2)
    plain = [t.contiguous() for t in (x, forget, out)]
    dy = rand((n, b, c), BF16, 2).to(DEV).transpose(0, 1)
    ws = room(A.adacomp_recurrence_workspace_bytes(b, n, c))
    results = []
    for parts, ds in (((x, forget, out), grads.chunk(3, dim=2)), (plain, [torch.empty_like(t) for t in plain])):
        y, states = torch.empty(n, b, c, dtype=BF16, device=DEV).transpose(0, 1), torch.empty(b, 2, c, device=DEV)
        A.adacomp_recurrence_forward(parts[0], parts[1], y, ws, out=parts[2], states=states)
        A.adacomp_recurrence_backward(dy, parts[0], parts[1], states, ds[0], ds[1], ws, out=parts[2], dout=ds[2])
        results.append([y, *ds])
    for one, other in zip(*results):
        assert torch.equal(one, other)


def test_recurrence_in_place(A):
    """y over x, the gradients over the gates, the state over itself."""
    for c in (64, 70, 3):
        s = recurrence_case(2, 200, c, F32, True, True, True, False, False, 8)
        g, want = check_both(A, s, F32)
        x, first = s["x"].to(DEV), s["first"].to(DEV)
        A.adacomp_recurrence_forward(x, g["forget"], x, g["ws"], out=g["out"], bias=g["bias"], first=first, last=first)
        assert torch.equal(x, g["y"]) and torch.equal(first, g["last"])
        x, forget, out, dy, dlast = g["x"].clone(), g["forget"].clone(), g["out"].clone(), rand((2, 200, c), F32, 77).to(DEV), rand((2, c), F32, 78).to(DEV)
        A.adacomp_recurrence_backward(dy, x, forget, g["states"], x, forget, g["ws"], out=out, dout=out, bias=g["bias"], dlast=dlast, dfirst=dlast)
        for got, name in ((x, "dx"), (forget, "dforget"), (out, "dout"), (dlast, "dfirst")):
            assert torch.equal(got, want[name]), name


@pytest.mark.parametrize("batch,length,channels", [(25, 1000, 509), (3, 3000, 67), (200, 300, 131), (300, 20, 66)])
def test_recurrence_states_over_themselves(A, batch, length, channels):
    """The last state over the first one, of sequences in parts and in one, with incomplete groups of channels that slabs share: as in separate buffers."""
    s = recurrence_case(batch, length, channels, BF16, True, True, True, False, False, 16)
    g = run_forward(A, s, BF16)
    first, y = g["first"].clone(), torch.empty_like(g["y"])
    A.adacomp_recurrence_forward(g["x"], g["forget"], y, g["ws"], out=g["out"], bias=g["bias"], first=first, last=first)
    assert torch.equal(y, g["y"]) and torch.equal(first, g["last"])
    dy, dlast = rand((batch, length, channels), BF16, 17).to(DEV), rand((batch, channels), F32, 18).to(DEV)
    results = []
    for over in (False, True):
        d, dfirst = [torch.empty_like(dy) for _ in range(3)], torch.empty_like(dlast)
        start = dlast.clone()
        dfirst = start if over else dfirst
        A.adacomp_recurrence_backward(dy, g["x"], g["forget"], g["states"], d[0], d[1], g["ws"], out=g["out"], dout=d[2], bias=g["bias"], dlast=start, dfirst=dfirst)
        results.append([*d, dfirst])
    for one, other in zip(*results):
        assert torch.equal(one, other)


def test_recurrence_token_by_token_is_the_whole_sequence(A):
    """Serving: single tokens with the state carried along, against the sequence at once; some sequences get no token now and then."""
    b, n, c = 5, 70, 130
    s = recurrence_case(b, n, c, F32, True, True, True, False, False, 9)
    r = S.Recurrence(**wide(s))
    g = {k: on_gpu(v) for k, v in s.items()}
    state, ws = g["first"].clone(), room(A.adacomp_recurrence_workspace_bytes(b, 1, c))
    y, done = torch.empty(b, 1, c, device=DEV), [0] * b
    for turn in range(200):
        if min(done) == n:
            break
        take = [int(done[i] < n and (turn + i) % 3 != 0) for i in range(b)]
        pick = lambda t: torch.stack([t[i, min(done[i], n - 1)] for i in range(b)])[:, None]
        A.adacomp_recurrence_forward(pick(g["x"]), pick(g["forget"]), y, ws, out=pick(g["out"]), bias=g["bias"], first=state, last=state,
                                     lengths=torch.tensor(take, dtype=torch.int32, device=DEV))
        for i in range(b):
            if take[i]:
                within(y[i, 0], r.y[i, done[i]], r.y_bound(F32)[i, done[i]], (turn, i))
                done[i] += 1
            else:
                assert torch.all(y[i] == 0)
    assert min(done) == n
    within(state, r.last, r.last_bound(), "state")


def test_recurrence_padding_may_be_anything(A):
    """NaN and infinities behind the sequences' ends, and before a document's first place, do not spread."""
    b, n, c = 3, 150, 20
    s = recurrence_case(b, n, c, BF16, True, True, True, True, False, 10)
    s["lengths"] = torch.tensor([100, 7, 0], dtype=torch.int32)
    clean_y, clean = check_both(A, s, BF16)
    for name in ("x", "forget", "out"):
        for i, end in enumerate(s["lengths"].tolist()):
            s[name][i, end:] = torch.tensor([float("nan"), float("inf"), -float("inf"), torch.finfo(BF16).min])[torch.arange((n - end) * c).view(n - end, c) % 4].to(BF16)
    g, got = run_forward(A, s, BF16), {}
    dy = rand((b, n, c), BF16, 77)
    for i, end in enumerate(s["lengths"].tolist()):
        dy[i, end:] = float("nan")
    grads = [torch.empty(b, n, c, dtype=BF16, device=DEV) for _ in range(3)]
    dbias = rand((c,), F32, 79).to(DEV)
    A.adacomp_recurrence_backward(dy.to(DEV), g["x"], g["forget"], g["states"], grads[0], grads[1], g["ws"], out=g["out"], dout=grads[2], bias=g["bias"], dbias=dbias,
                                  dlast=rand((b, c), F32, 78).to(DEV), lengths=g["lengths"])
    assert torch.equal(g["y"], clean_y["y"]) and torch.equal(g["last"], clean_y["last"])
    for t, name in zip((*grads, dbias), ("dx", "dforget", "dout", "dbias")):
        assert torch.equal(t, clean[name]), name
    s = recurrence_case(1, n, c, F32, False, True, True, False, True, 11)
    s["resets"].zero_()
    s["resets"][0, 60] = 1
    s["x"][0, 20] = float("nan")
    g = run_forward(A, s, F32)
    assert torch.all(torch.isnan(g["y"][0, 20:60])) and torch.all(torch.isfinite(g["y"][0, 60:])) and torch.all(torch.isfinite(g["last"]))
    dx, df = torch.empty(1, n, c, device=DEV), torch.empty(1, n, c, device=DEV)
    dy = torch.zeros(1, n, c)
    dy[0, 100] = float("nan")
    A.adacomp_recurrence_backward(dy.to(DEV), g["x"], g["forget"], g["states"], dx, df, g["ws"], bias=g["bias"], resets=g["resets"])
    assert torch.all(torch.isnan(dx[0, 60:101])) and torch.all(dx[0, :60] == 0) and torch.all(dx[0, 101:] == 0)


@pytest.mark.parametrize("dtype", TYPES)
def test_recurrence_of_extreme_gates(A, dtype):
    """Gates that are shut or open as far as the type goes: a state that stays for ever, one that is new at every place."""
    s = recurrence_case(2, 140, 9, dtype, True, False, True, False, False, 12)
    big = torch.finfo(dtype).max
    values = torch.tensor([0.0, 30.0, -30.0, 79.0, -79.0, 200.0, -200.0, big, -big], dtype=torch.float64)
    for name in ("forget", "out"):
        s[name] = values[(torch.arange(2 * 140 * 9) * (5 if name == "out" else 1) + torch.arange(2 * 140 * 9) // 9).view(2, 140, 9) % 9].to(dtype)
    check_both(A, s, dtype)


def test_recurrence_of_nothing(A):
    ws = room(4096)
    for shape in ((0, 5, 8), (3, 0, 8), (3, 5, 0)):
        b, n, c = shape
        x, y = torch.empty(shape, device=DEV), torch.empty(shape, device=DEV)
        first, last, dbias = rand((b, c), F32, 1).to(DEV), torch.zeros(b, c, device=DEV), torch.full((c,), 5.0, device=DEV)
        states = torch.empty(b, A.adacomp_recurrence_kept(n), c, device=DEV)
        A.adacomp_recurrence_forward(x, x, y, ws, first=first, last=last, states=states)
        assert n or torch.equal(first, last)
        last.zero_()
        A.adacomp_recurrence_backward(x, x, x, states, y, y, ws, dbias=dbias, dlast=first, dfirst=last)
        assert n or torch.equal(first, last)
        assert torch.all(dbias == 0)


def test_recurrence_calls_repeat_bit_for_bit(A):
    s = recurrence_case(2, 3000, 100, BF16, True, True, True, False, False, 13)
    _, first = check_both(A, s, BF16)
    for _ in range(3):
        _, again = check_both(A, s, BF16)
        for name in first:
            assert torch.equal(first[name], again[name]), name


def test_recurrence_refusals(A):
    x, ws = torch.zeros(2, 6, 8, device=DEV), room(4096)
    y, states = torch.zeros_like(x), torch.zeros(2, 1, 8, device=DEV)
    ok = dict(x=x, forget=x, y=y, workspace=ws)
    A.adacomp_recurrence_forward(**ok)
    vec = torch.zeros(2, 8, device=DEV)
    for bad in (dict(x=x[0]), dict(x=x.double()), dict(x=x.cpu()), dict(forget=x.half()), dict(forget=x[:, :5]), dict(out=x[:, :, :7]), dict(y=y.expand(2, 6, 8)[:, :1].expand(2, 6, 8)),
                dict(y=torch.zeros(2, 8, 6, device=DEV).transpose(1, 2)), dict(bias=vec), dict(bias=vec[0].half()), dict(first=vec[:1]), dict(last=vec.cpu()), dict(states=states[:1]),
                dict(lengths=torch.zeros(2, dtype=torch.int64, device=DEV)), dict(lengths=torch.zeros(3, dtype=torch.int32, device=DEV)), dict(resets=torch.zeros(2, 5, dtype=torch.uint8, device=DEV)),
                dict(resets=torch.zeros(2, 6, device=DEV)), dict(resets=torch.zeros(2, 12, dtype=torch.uint8, device=DEV)[:, ::2]), dict(workspace=ws[:128])):
        with pytest.raises(A.AdacompError):
            A.adacomp_recurrence_forward(**(ok | bad))
    ok = dict(dy=x, x=x, forget=x, states=states, dx=y, dforget=torch.zeros_like(x), workspace=ws)
    A.adacomp_recurrence_backward(**ok)
    for bad in (dict(dy=x.half()), dict(states=None), dict(out=x), dict(dout=x), dict(dx=None), dict(dbias=vec), dict(dlast=vec[:1]), dict(workspace=ws[:128])):
        with pytest.raises(A.AdacompError):
            A.adacomp_recurrence_backward(**(ok | bad))


# ---- distillation ---------------------------------------------------------------------------------------------------

def distill_case(rows, vocab, top, dtype, seed, padding=True):
    g = torch.Generator().manual_seed(seed)
    z = rand((rows, vocab), dtype, seed, 3.0)
    s = {"z": z, "tokens": torch.randint(0, vocab, (rows, top), generator=g), "t": rand((rows, top), F32, seed + 1, 3.0), "targets": torch.randint(0, vocab, (rows,), generator=g)}
    if padding:
        for i in range(rows):
            if i % 7 == 1:
                s["tokens"][i] = -1
            if i % 7 in (1, 2):
                s["targets"][i] = -100
            if i % 7 == 3 and top:
                s["tokens"][i, 0] = vocab
                s["t"][i, 0] = float("nan")
            if i % 7 == 4 and top > 1:
                s["tokens"][i, -1] = s["tokens"][i, 0]     # twice
                s["targets"][i] = s["tokens"][i, 0]
            if i % 7 == 5 and top:
                s["t"][i, 0] = -float("inf")
            if i % 7 == 6:
                s["t"][i] = -float("inf")                  # no teacher either
    return s


def check_distill(A, s, dtype, temperature, soft, hard, index=torch.int64, tdtype=None, pad=0, lead=0, scale=1.0):
    rows, vocab = s["z"].shape
    tdtype = tdtype or dtype
    t = s["t"].to(tdtype)
    tau, soft32, hard32, scale32 = (float(np.float32(v)) for v in (temperature, soft, hard, scale))
    d = S.Distill(s["z"].double(), s["tokens"] if soft else None, t.double(), s["targets"] if hard else None, tau, soft32, hard32)
    dloss = torch.where(torch.arange(rows) % 5 == 4, 0.0, rand((rows,), F32, 90))
    z = on_gpu(s["z"], pad, lead)
    args = dict(teacher_tokens=s["tokens"].to(index).to(DEV), teacher_logits=t.to(DEV), targets=s["targets"].to(index).to(DEV), temperature=temperature, soft=soft, hard=hard)
    loss, lse = torch.full((rows,), float("nan"), device=DEV), torch.full((rows, 2), float("nan"), device=DEV)
    A.adacomp_distill_forward(z, loss, lse=lse, **args)
    within(loss, d.loss, d.loss_off, "loss")
    within(lse, d.lse, torch.where(d.lse == 0, 0.0, d.lse_off), "lse")
    for at_once in (True, False):
        got = on_gpu(torch.full((rows, vocab), float("nan"), dtype=dtype), pad, lead)
        if at_once:
            again = torch.full((rows,), float("nan"), device=DEV)
            A.adacomp_distill_forward(z, again, dlogits=got, dloss=dloss.to(DEV), scale=scale, **args)
            assert torch.equal(again, loss)
        else:
            A.adacomp_distill_backward(z, lse, got, dloss=dloss.to(DEV), scale=scale, **args)
        want, off = d.gradient(dloss.double(), scale32, from_lse=not at_once)
        within(got, want, rounded(want, off, dtype), ("dlogits", at_once))
        if pad or lead:
            untouched(got, pad, lead)
    return loss, lse, got


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [1, 2, 7, 8, 9, 65, 255, 256, 257, 1000, 1024, 1025, 2048, 4096, 4097, 5999, 8192, 8200, 16391, 32768, 32769, 50001, 65536, 70001, 131072, 140003])
def test_distill_vocabularies(A, vocab, dtype):
    rows, top = (45 if vocab < 5000 else 9), min(20, vocab)
    s = distill_case(rows, vocab, top, dtype, vocab)
    check_distill(A, s, dtype, 1.0, 1.0, 0.0)
    check_distill(A, s, dtype, 2.0, 0.7, 0.3, scale=1.7)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("temperature,soft,hard", [(1.0, 0.5, 0.5), (1.0, 0.0, 1.0), (3.3, 1.0, 0.0), (0.6, 0.4, 0.6), (5.0, 0.0, 1.0)])
def test_distill_terms(A, temperature, soft, hard, dtype):
    for rows, vocab, top, pad, lead in ((40, 65, 7, 3, 1), (23, 3001, 33, 0, 0), (9, 9001, 100, 5, 2)):
        s = distill_case(rows, vocab, top, dtype, 3)
        check_distill(A, s, dtype, temperature, soft, hard, index=torch.int32, tdtype=BF16, pad=pad, lead=lead)


@pytest.mark.parametrize("vocab,top", [(300, 256), (50, 256), (200, 127), (200, 128), (6000, 256), (40000, 1), (9, 9)])
def test_distill_top_tokens(A, vocab, top):
    """As many top tokens as there can be, more than the vocabulary has, and one."""
    check_distill(A, distill_case(30, vocab, top, F32, 4), F32, 1.5, 0.8, 0.2)


@pytest.mark.parametrize("rows,vocab", [(4096, 1025), (4100, 2047), (4097, 8191), (4096, 8193), (513, 9000), (511, 16385), (4099, 1024)])
def test_distill_many_rows(A, rows, vocab):
    """Rows enough for a wave each, and the sizes where that ends; the first and the last of them against the formula, all against one another."""
    g = torch.Generator().manual_seed(12)
    few = distill_case(24, vocab, 30, BF16, 13)
    pick = torch.randint(0, 24, (rows,), generator=g)
    pick[:24], pick[-24:] = torch.arange(24), torch.arange(24)
    args = dict(temperature=1.5, soft=0.6, hard=0.4)
    part = lambda i: dict(teacher_tokens=few["tokens"][i].to(DEV), teacher_logits=few["t"][i].to(DEV), targets=few["targets"][i].to(DEV))
    loss, lse, grad = torch.empty(rows, device=DEV), torch.empty(rows, 2, device=DEV), torch.empty(rows, vocab, dtype=BF16, device=DEV)
    z = few["z"].to(DEV)[pick.to(DEV)]
    A.adacomp_distill_forward(z, loss, lse=lse, dlogits=grad, **part(pick), **args)
    d = S.Distill(few["z"].double(), few["tokens"], few["t"].double(), few["targets"], *(float(np.float32(v)) for v in (1.5, 0.6, 0.4)))
    want, off = d.gradient(torch.ones(24, dtype=torch.float64))
    within(loss[:24], d.loss, d.loss_off, "loss")
    within(grad[:24], want, rounded(want, off, BF16), "dlogits")
    assert torch.equal(loss, loss[:24][pick.to(DEV)]) and torch.equal(lse, lse[:24][pick.to(DEV)]) and torch.equal(grad, grad[:24][pick.to(DEV)])
    back = torch.empty_like(grad)
    A.adacomp_distill_backward(z, lse, back, **part(pick), **args)
    want, off = d.gradient(torch.ones(24, dtype=torch.float64), from_lse=True)
    within(back[:24], want, rounded(want, off, BF16), "dlogits from lse")
    assert torch.equal(back, back[:24][pick.to(DEV)])


def test_distill_without_a_teacher_is_cross_entropy(A):
    z, targets = rand((200, 65), F32, 5, 3.0), torch.randint(0, 65, (200,), generator=torch.Generator().manual_seed(6))
    d = S.Distill(z.double(), targets=targets)
    loss, lse, grad = torch.empty(200, device=DEV), torch.empty(200, 2, device=DEV), torch.empty(200, 65, device=DEV)
    A.adacomp_distill_forward(z.to(DEV), loss, lse=lse, targets=targets.to(DEV), dlogits=grad)
    within(loss, d.loss, d.loss_off, "loss")
    within(loss, torch.nn.functional.cross_entropy(z.double(), targets, reduction="none"), d.loss_off, "cross entropy")
    want, off = d.gradient(torch.ones(200, dtype=torch.float64))
    within(grad, want, rounded(want, off, F32), "dlogits")
    for what in (dict(), dict(targets=targets.to(DEV), hard=0.0), dict(teacher_tokens=torch.zeros(200, 0, dtype=torch.int64, device=DEV), teacher_logits=torch.zeros(200, 0, device=DEV))):
        A.adacomp_distill_forward(z.to(DEV), loss.fill_(3.0), dlogits=grad.fill_(3.0), **what)   # no term: all rows are padding
        assert torch.all(loss == 0) and torch.all(grad == 0)


def test_distill_in_place_and_of_shaped_rows(A):
    """The gradient over the logits, at once and from the lse; rows in two dimensions, of wider tensors; logits as a teacher's topk left them."""
    for vocab in (65, 3000, 40001):
        s = distill_case(12, vocab, 10, BF16, 7)
        _, lse, want = check_distill(A, s, BF16, 2.0, 0.5, 0.5)
        dloss = torch.where(torch.arange(12) % 5 == 4, 0.0, rand((12,), F32, 90)).to(DEV)
        wide_t, wide_k = torch.zeros(3, 4, 16, dtype=BF16, device=DEV), torch.zeros(3, 4, 13, dtype=torch.int64, device=DEV)
        wide_t[..., :10], wide_k[..., 2:12] = s["t"].to(BF16).view(3, 4, 10).to(DEV), s["tokens"].view(3, 4, 10).to(DEV)
        args = dict(teacher_tokens=wide_k[..., 2:12], teacher_logits=wide_t[..., :10], targets=s["targets"].view(3, 4).to(DEV), temperature=2.0, soft=0.5, hard=0.5, dloss=dloss.view(3, 4))
        z = s["z"].to(DEV).view(3, 4, vocab).clone()
        A.adacomp_distill_backward(z, lse, z, **args)
        assert torch.equal(z.view(12, vocab), want)
        z, out = s["z"].to(DEV).view(3, 4, vocab).clone(), torch.empty(12, vocab, dtype=BF16, device=DEV)
        loss = torch.empty(3, 4, device=DEV)
        A.adacomp_distill_forward(z.clone(), loss, dlogits=out.view(3, 4, vocab), **args)
        A.adacomp_distill_forward(z, loss, dlogits=z, **args)
        assert torch.equal(z.view(12, vocab), out)


def test_distill_of_padding_that_holds_anything(A):
    """Rows that count for nothing hold NaN and infinities; places that are no token hold NaN in the teacher's logits."""
    for vocab in (40, 3000, 40001):
        s = distill_case(14, vocab, 6, F32, 8)
        void = torch.arange(14) % 7 == 1
        s["z"][void] = torch.tensor([float("nan"), float("inf"), -float("inf")])[torch.arange(vocab) % 3]
        s["t"][void] = float("nan")
        rows = torch.nonzero(~void)[:, 0]
        loss, lse, grad = torch.empty(14, device=DEV), torch.empty(14, 2, device=DEV), torch.full((14, vocab), 5.0, device=DEV)
        args = dict(teacher_tokens=s["tokens"].to(DEV), teacher_logits=s["t"].to(DEV), targets=s["targets"].to(DEV), temperature=2.0, soft=0.5, hard=0.5)
        d = S.Distill(s["z"][rows].double(), s["tokens"][rows], s["t"][rows].double(), s["targets"][rows], 2.0, 0.5, 0.5)
        want, off = d.gradient(torch.ones(len(rows), dtype=torch.float64))
        A.adacomp_distill_forward(s["z"].to(DEV), loss, lse=lse, dlogits=grad, **args)
        for _ in range(2):
            assert torch.all(loss[void] == 0) and torch.all(lse[void] == 0) and torch.all(grad[void] == 0)
            within(loss[~void], d.loss, d.loss_off, "loss")
            within(grad[~void], want, rounded(want, off + U * 100 * want.abs(), F32), "dlogits")
            A.adacomp_distill_backward(s["z"].to(DEV), lse, grad.fill_(5.0), **args)


def test_distill_of_tokens_that_cannot_be(A):
    """-infinity among the logits: nothing for q; at the target or a top token an infinite loss, and a finite gradient."""
    inf = float("inf")
    for vocab in (50, 2000, 33000):
        z = rand((6, vocab), F32, 9)
        z[0, 10:] = -inf
        z[1, 5] = -inf
        z[2, 5] = -inf
        z[3] = -inf
        z[4] = torch.finfo(F32).min
        tokens, t = torch.tensor([[3, 4], [5, 6], [7, 8], [1, 2], [3, 4], [5, 5]]), rand((6, 2), F32, 10)
        targets = torch.tensor([2, 6, 5, 0, 9, 8])
        for temperature in (1.0, 2.0):
            args = dict(teacher_tokens=tokens.to(DEV), teacher_logits=t.to(DEV), targets=targets.to(DEV), temperature=temperature, soft=0.5, hard=0.5)
            loss, lse, grad = torch.empty(6, device=DEV), torch.empty(6, 2, device=DEV), torch.empty(6, vocab, device=DEV)
            A.adacomp_distill_forward(z.to(DEV), loss, lse=lse, dlogits=grad, **args)
            assert torch.isfinite(loss[[0, 5]]).all() and torch.all(loss[[1, 2, 3]] == inf) and torch.isfinite(loss[4])
            assert torch.isfinite(grad).all()
            assert torch.all(grad[0, 10:] == 0) and torch.all(torch.isneginf(lse[3]))
            d = S.Distill(z[[0, 5]].double(), tokens[[0, 5]], t[[0, 5]].double(), targets[[0, 5]], temperature, 0.5, 0.5)
            want, off = d.gradient(torch.ones(2, dtype=torch.float64))
            within(grad[[0, 5]], want, rounded(want, off, F32), "dlogits")
            p = torch.softmax(t[3].double() / temperature, 0)   # q is 0 everywhere
            row = torch.zeros(vocab, dtype=torch.float64)
            row[tokens[3]] = -0.5 * temperature * p
            row[0] -= 0.5
            within(grad[3], row, U * 64 * row.abs() + TINY[F32], "row of nothing")
            even = 1.0 / vocab   # all logits alike, however low
            assert abs(grad[4, 11].item() - 0.5 * (temperature + 1) * even) <= U * 400 * even * (temperature + 1)
            again = torch.empty_like(grad)
            A.adacomp_distill_backward(z.to(DEV), lse, again, **args)
            rows = [0, 3, 5]
            assert torch.isfinite(again[:4]).all() and torch.all(again[0, 10:] == 0)
            within(again[3], row, U * 64 * row.abs() + TINY[F32], "row of nothing, from the lse")
            want, off = d.gradient(torch.ones(2, dtype=torch.float64), from_lse=True)
            within(again[[0, 5]], want, rounded(want, off, F32), "dlogits from the lse")


def test_distill_nan_stays_in_its_row(A):
    for vocab in (50, 2000, 33000):
        z = rand((4, vocab), BF16, 11)
        z[1, vocab // 2] = float("nan")
        z[2, 3] = float("inf")
        targets = torch.tensor([1, 2, 3, 4], device=DEV)
        loss, lse, grad = torch.empty(4, device=DEV), torch.empty(4, 2, device=DEV), torch.empty(4, vocab, dtype=BF16, device=DEV)
        A.adacomp_distill_forward(z.to(DEV), loss, lse=lse, dlogits=grad, targets=targets)
        assert torch.isfinite(loss[[0, 3]]).all() and torch.isnan(loss[1]) and torch.isnan(loss[2])
        assert torch.isfinite(grad[[0, 3]]).all() and torch.isnan(grad[1]).all() and torch.isnan(grad[2]).all()


def test_distill_of_logits_beyond_the_range(A):
    """z / temperature beyond float32: a row with +infinity there is NaN, loss and gradient, in either way; one with -infinity at all places has q = 0; and the
    target's term, at a temperature of 1, is what it is in a row without a teacher."""
    for vocab in (50, 2000, 33000):
        z = rand((3, vocab), F32, 19)
        z[0, 7] = 3e38
        z[1] = torch.finfo(F32).min
        z[2, 7] = 3e38
        tokens, t, targets = torch.tensor([[3, 4], [3, 4], [-1, -1]]), rand((3, 2), F32, 20), torch.tensor([1, 1, 7])
        args = dict(teacher_tokens=tokens.to(DEV), teacher_logits=t.to(DEV), targets=targets.to(DEV), temperature=0.5, soft=0.5, hard=0.5)
        loss, lse, grad = torch.empty(3, device=DEV), torch.empty(3, 2, device=DEV), torch.empty(3, vocab, device=DEV)
        A.adacomp_distill_forward(z.to(DEV), loss, lse=lse, dlogits=grad, **args)
        back = torch.empty_like(grad)
        A.adacomp_distill_backward(z.to(DEV), lse, back, **args)
        assert torch.isnan(loss[0]) and loss[1] == float("inf") and loss[2] == 0
        for g in (grad, back):
            assert torch.isnan(g[0]).all() and torch.isfinite(g[1:]).all() and torch.all(g[2] == 0)


def test_distill_refusals(A):
    z, loss, lse, grad = torch.zeros(4, 9, device=DEV), torch.zeros(4, device=DEV), torch.zeros(4, 2, device=DEV), torch.zeros(4, 9, device=DEV)
    k, t, targets = torch.zeros(4, 3, dtype=torch.int64, device=DEV), torch.zeros(4, 3, device=DEV), torch.zeros(4, dtype=torch.int64, device=DEV)
    ok = dict(teacher_tokens=k, teacher_logits=t, targets=targets)
    A.adacomp_distill_forward(z, loss, **ok)
    for bad in (dict(teacher_tokens=None), dict(teacher_logits=None), dict(teacher_tokens=k[:3]), dict(teacher_logits=t[:, :2]), dict(teacher_tokens=k.float()), dict(teacher_logits=t.double()),
                dict(targets=targets[:3]), dict(targets=targets.cpu()), dict(targets=targets.float()), dict(teacher_tokens=k.cpu()), dict(temperature=0.0), dict(temperature=-1.0),
                dict(temperature=float("nan")), dict(soft=-1.0), dict(hard=float("inf")), dict(scale=float("nan")), dict(dlogits=grad.half()), dict(dlogits=grad[:, :8]), dict(dloss=loss[:2]),
                dict(lse=loss), dict(teacher_tokens=torch.zeros(4, 300, dtype=torch.int64, device=DEV), teacher_logits=torch.zeros(4, 300, device=DEV))):
        with pytest.raises(A.AdacompError):
            A.adacomp_distill_forward(z, loss, **(ok | bad))
    for args in ((z, None, grad), (z, lse, None), (z.cpu(), lse, grad), (z, lse, grad[:1].expand(4, 9))):
        with pytest.raises(A.AdacompError):
            A.adacomp_distill_backward(*args, **ok)
    with pytest.raises(A.AdacompError):
        A.adacomp_distill_forward(z, None, **ok)
    none = torch.zeros(0, 9, device=DEV)
    A.adacomp_distill_forward(none, loss[:0], dlogits=none, targets=targets[:0])


# ---- graphs, streams, large calls -----------------------------------------------------------------------------------

def everything(A, seed, rows=(4, 300), vocab=500, c=70, top=9):
    """One call of each kind on buffers of its own: (a function that makes the calls, the results, the inputs that may change)."""
    b, n = rows
    g = lambda shape, k, dtype=BF16: rand(shape, dtype, seed + k).to(DEV)
    tokens = tokens_of(b * n, vocab, seed).view(b, n).to(DEV)
    table, x, forget, out, dy, z = g((vocab, c), 1, F32), g((b, n, c), 2), g((b, n, c), 3), g((b, n, c), 4), g((b, n, c), 5), g((b, n, vocab), 6)
    k, t, targets = torch.randint(0, vocab, (b, n, top), device=DEV), g((b, n, top), 7), torch.randint(0, vocab, (b, n), device=DEV)
    y, dtable, r, states, last = torch.empty_like(x), torch.empty_like(table), torch.empty_like(x), torch.empty(b, A.adacomp_recurrence_kept(n), c, device=DEV), torch.empty(b, c, device=DEV)
    dx, df, do, dbias, bias = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x), torch.empty(c, device=DEV), g((c,), 8, F32)
    loss, lse, dz, dz2 = torch.empty(b, n, device=DEV), torch.empty(b, n, 2, device=DEV), torch.empty_like(z), torch.empty_like(z)
    ws = room(max(A.adacomp_embed_workspace_bytes(b * n, vocab, c), A.adacomp_recurrence_workspace_bytes(b, n, c)))
    terms = dict(teacher_tokens=k, teacher_logits=t, targets=targets, temperature=2.0, soft=0.5, hard=0.5)

    def calls():
        A.adacomp_embed_forward(tokens, table, y, dropout=A.Dropout(0.2, 9, 10))
        A.adacomp_embed_backward(tokens, dy, dtable, ws, dropout=A.Dropout(0.2, 9, 10))
        A.adacomp_recurrence_forward(x, forget, r, ws, out=out, bias=bias, states=states, last=last)
        A.adacomp_recurrence_backward(dy, x, forget, states, dx, df, ws, out=out, dout=do, bias=bias, dbias=dbias)
        A.adacomp_distill_forward(z, loss, lse=lse, dlogits=dz, **terms)
        A.adacomp_distill_backward(z, lse, dz2, **terms)
    return calls, [y, dtable, r, states, last, dx, df, do, dbias, loss, lse, dz, dz2], [x, forget, dy, z, table]


def capture(calls):
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            calls()
    return graph


def test_captured_and_replayed(A):
    """Two graphs with a workspace of their own each, replayed in turn with eager work between, on inputs that change."""
    pairs = [everything(A, 20), everything(A, 40, rows=(1, 3000), vocab=5000, c=40)]
    graphs = []
    for calls, _, _ in pairs:
        calls()
        torch.cuda.synchronize()
        graphs.append(capture(calls))
    for turn in range(4):
        for (calls, results, inputs), graph in zip(pairs, graphs):
            for t in inputs:
                t.mul_(0.9)
            calls()
            eager = [r.clone() for r in results]
            for r in results:
                r.fill_(7.0)
            graph.replay()
            torch.cuda.synchronize()
            for i, (got, want) in enumerate(zip(results, eager)):
                assert torch.equal(got, want), (turn, i)


def test_embed_step_in_memory(A):
    """A captured lookup and its gradient draw another mask when the number in memory has changed, the same one in both."""
    tokens, table, dy = tokens_of(200, 30, 22).to(DEV), rand((30, 45), F32, 23).to(DEV), rand((200, 45), F32, 24).to(DEV)
    y, dtable, ws, step = torch.empty(200, 45, device=DEV), torch.empty(30, 45, device=DEV), embed_room(A, 200, 30, 45), torch.zeros(1, dtype=torch.int64, device=DEV)
    drop = A.Dropout(0.4, 5, 100, step)

    def calls():
        A.adacomp_embed_forward(tokens, table, y, dropout=drop)
        A.adacomp_embed_backward(tokens, dy, dtable, ws, dropout=drop)
    calls()
    torch.cuda.synchronize()
    graph = capture(calls)
    for number in (0, 3, 3, 9):
        step.fill_(number)
        graph.replay()
        torch.cuda.synchronize()
        f = (0.4, 5, 100 + number)
        want = S.embed_forward(tokens.cpu(), table.cpu().double(), 1.0, f)
        within(y, want, rounded(want, 4 * U * want.abs(), F32), ("y", number))
        want, size, count = S.embed_backward(tokens.cpu(), dy.cpu().double(), 30, 1.0, f)
        within(dtable, want, U * ((count + 8).double()[:, None] * size + 2 * want.abs()) + TINY[F32], ("dtable", number))


def test_on_other_streams_at_once(A):
    """Calls of two streams at the same time, each with its workspace, give what they give alone."""
    pairs = [everything(A, 60, rows=(3, 900)), everything(A, 80, rows=(2, 1500), vocab=3000)]
    alone = []
    for calls, results, _ in pairs:
        calls()
        alone.append([r.clone() for r in results])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for (calls, results, _), stream in zip(pairs, streams):
        with torch.cuda.stream(stream):
            for r in results:
                r.fill_(7.0)
            for _ in range(5):
                calls()
    torch.cuda.synchronize()
    for (_, results, _), want in zip(pairs, alone):
        for i, (got, w) in enumerate(zip(results, want)):
            assert torch.equal(got, w), i


def test_embed_rows_beyond_32_bits(A):
    """A table and an output of more than 2^32 bytes, and more than 2^31 values: rows at their ends."""
    vocab, cols = (1 << 19) + 3, 4100
    table = torch.zeros(vocab, cols, device=DEV)
    ends = [0, 1, vocab // 2, vocab - 2, vocab - 1]
    rows = rand((len(ends), cols), F32, 1)
    table[torch.tensor(ends, device=DEV)] = rows.to(DEV)
    tokens = torch.tensor(ends, device=DEV).repeat(3)
    y = torch.empty(len(tokens), cols, dtype=F32, device=DEV)
    A.adacomp_embed_forward(tokens, table, y)
    assert torch.equal(y.cpu(), rows.repeat(3, 1))
    A.adacomp_embed_backward(tokens, y, table.fill_(5.0), embed_room(A, len(tokens), vocab, cols))
    want = (rows + rows) + rows
    assert torch.equal(table[torch.tensor(ends, device=DEV)].cpu(), want)
    table[torch.tensor(ends, device=DEV)] = 0
    assert not table.any()
    del table
    torch.cuda.empty_cache()
    rows = (1 << 20) + 5
    y = torch.full((rows, cols), 3.0, dtype=BF16, device=DEV)
    small = rand((7, cols), F32, 2)
    tokens = torch.arange(rows, device=DEV) % 8   # the eighth is none
    A.adacomp_embed_forward(tokens, small.to(DEV), y)
    for first in (0, (1 << 19) - 2, rows - 9):
        want = S.embed_forward(tokens[first:first + 9].cpu(), small.double(), 1.0)
        within(y[first:first + 9], want, rounded(want, 0.0 * want, BF16), first)
    got = torch.empty(7, cols, device=DEV)
    A.adacomp_embed_backward(tokens, y.fill_(0.5), got, embed_room(A, rows, 7, cols))
    assert torch.equal(got.cpu(), (torch.bincount(tokens.cpu(), minlength=8)[:7].float() * 0.5)[:, None].expand(7, cols))
    del y
    torch.cuda.empty_cache()


def test_recurrence_and_distill_beyond_32_bits(A):
    """Tensors of more than 2^32 bytes: sequences far apart, rows at both ends."""
    b, n, c, stride = 3, 70, 66, 1 << 30   # 2^31 bytes between bf16 sequences, which are 70 rows of 2^24 bytes long
    s = recurrence_case(b, n, c, BF16, True, True, True, False, False, 14)
    room_ = torch.zeros(2 * stride + n * (1 << 23) + 4096, dtype=BF16, device=DEV)
    far = room_.as_strided((b, n, c), (stride, 1 << 23, 1))   # rows 2^24 bytes apart
    far.copy_(s["x"])
    near = run_forward(A, s, BF16)
    y = torch.empty(b, n, c, dtype=BF16, device=DEV)
    A.adacomp_recurrence_forward(far, near["forget"], y, near["ws"], out=near["out"], bias=near["bias"], first=near["first"])
    assert torch.equal(y, near["y"])
    A.adacomp_recurrence_forward(far, near["forget"], far, near["ws"], out=near["out"], bias=near["bias"], first=near["first"])
    assert torch.equal(far, near["y"])
    del room_, far
    torch.cuda.empty_cache()
    rows, vocab = 40000, 70001
    z = torch.full((rows, vocab), 1.0, dtype=BF16, device=DEV)
    few = distill_case(8, vocab, 12, BF16, 15)
    at = torch.tensor([0, 1, 2, 3, rows - 4, rows - 3, rows - 2, rows - 1])
    z[at.to(DEV)] = few["z"].to(DEV)
    tokens, t, targets = torch.full((rows, 12), -1), torch.zeros(rows, 12), torch.full((rows,), -1)
    tokens[at], t[at], targets[at] = few["tokens"], few["t"], few["targets"]
    d = S.Distill(few["z"].double(), few["tokens"], few["t"].double(), few["targets"], 2.0, 0.5, 0.5)
    loss = torch.empty(rows, device=DEV)
    A.adacomp_distill_forward(z, loss, dlogits=z, teacher_tokens=tokens.to(DEV), teacher_logits=t.to(DEV), targets=targets.to(DEV), temperature=2.0, soft=0.5, hard=0.5)
    want, off = d.gradient(torch.ones(8, dtype=torch.float64))
    within(loss[at.to(DEV)], d.loss, d.loss_off, "loss")
    within(z[at.to(DEV)], want, rounded(want, off, BF16), "dlogits")
    assert not z[4:rows - 4].any() and not loss[4:rows - 4].any()
    del z
    torch.cuda.empty_cache()
