"""Several documents in a sequence of the gated linear recurrence: what is not finite lasts to the end of its document and no further, in both
directions, however the sequence is shared out among threads, waves and parts, and whatever the gates are."""
import pytest
import torch

import sequence_reference as S
from test_gpu_sequence import A, BF16, DEV, F16, F32, TYPES, on_gpu, rand, recurrence_case, room, rounded, run_forward, wide  # noqa: F401

pytestmark = pytest.mark.gpu
NAN, INF = float("nan"), float("inf")


def agree(got, want, off, what):
    """Finite at the same places, and within the bound there."""
    got = got.cpu().double()
    finite = torch.isfinite(want)
    assert torch.equal(torch.isfinite(got), finite), (what, torch.nonzero(torch.isfinite(got) != finite)[:5].tolist())
    off = torch.where(torch.isnan(off), 0.0, off)   # 0 times NaN: behind a reset at the first place its gradient is 0, exactly
    assert torch.all(((got - want).abs() <= off)[finite]), what


def backward(A, g, dy, dlast, dtype):
    got = {k: torch.full(dy.shape, 7.0, dtype=dtype, device=DEV) for k in ("dx", "dforget", "dout")}
    if g["out"] is None:
        got["dout"] = None
    got["dfirst"], got["dbias"] = torch.full(dlast.shape, 7.0, device=DEV), torch.full(dlast.shape[1:], 7.0, device=DEV)
    A.adacomp_recurrence_backward(dy.to(DEV), g["x"], g["forget"], g["states"], got["dx"], got["dforget"], g["ws"], out=g["out"], dout=got["dout"], bias=g["bias"],
                                  dlast=dlast.to(DEV), dfirst=got["dfirst"], dbias=got["dbias"], lengths=g["lengths"], resets=g["resets"])
    return {k: v for k, v in got.items() if v is not None}


def check(A, s, dtype, dy, dlast):
    r = S.Recurrence(**wide(s))
    g = run_forward(A, s, dtype)
    agree(g["y"], r.y, r.y_bound(dtype), "y")
    agree(g["last"], r.last, r.last_bound(), "last")
    want, off = r.states()
    agree(g["states"], want, off + 4 * S.U * want.abs(), "states")
    got, want = backward(A, g, dy, dlast, dtype), r.backward(dy.double(), dlast.double())
    for name in {"dx", "dforget", "dout"} & set(want):   # zeros behind the end, where the formula has 0 times what is not finite
        want[name] = tuple(torch.where(r.inside, v, 0.0) for v in want[name])
    df, off = want["dforget"]
    want["dbias"] = (df.sum((0, 1)), off.sum((0, 1)) + S.U * (r.n + df.shape[0] + 64) * df.abs().sum((0, 1)))
    for name, (value, off) in want.items():
        agree(got[name], value, rounded(value, off, dtype if name in ("dx", "dforget", "dout") else F32), name)


# sequences of few places, of one block, of several, and in parts (few sequences of few channels)
SHAPES = [(3, 12, 9), (300, 100, 66), (260, 150, 64), (3, 300, 20), (2, 1500, 67), (1, 4000, 8)]


def documents(b, n, seed):
    """A reset every 40 places or so, and a sequence with none where there are three."""
    g = torch.Generator().manual_seed(seed)
    resets = (torch.rand(b, n, generator=g) < 0.025).to(torch.uint8)
    if b > 2:
        resets[2] = 0
    return resets


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("where,gate,shut", [(w, g, not g) for w in ("forget", "x", "x infinite", "dy") for g in (True, False)] + [("out", True, False), ("out", True, True)])
@pytest.mark.parametrize("batch,length,channels", SHAPES)
def test_what_is_not_finite_stays_in_its_document(A, batch, length, channels, where, gate, shut, dtype):
    """shut: gates that are nearly shut, whose product over a few places is below what float32 can hold."""
    s = recurrence_case(batch, length, channels, dtype, gate, True, True, False, False, 31)
    s["resets"] = documents(batch, length, 32)
    s["bias"] = torch.full((channels,), -12.0) if shut else s["bias"]
    dy, dlast = rand((batch, length, channels), dtype, 77), rand((batch, channels), F32, 78)
    at = torch.rand(batch, length, generator=torch.Generator().manual_seed(33)) < 0.015   # about as many as documents, in some channels
    at[0, min(50, length - 2)], s["resets"][0, min(60, length - 1)] = True, 1
    some = at[..., None] & (torch.arange(channels) % 3 != 1)
    t = dy if where == "dy" else s[where.split()[0]]
    t[some] = INF if "infinite" in where else NAN
    check(A, s, dtype, dy, dlast)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("batch,length,channels", SHAPES)
def test_documents_of_ragged_sequences(A, batch, length, channels, dtype):
    """NaN and resets behind the ends too, where they change nothing."""
    s = recurrence_case(batch, length, channels, dtype, True, True, True, True, False, 39)
    s["resets"] = documents(batch, length, 40) * 200   # any number but 0
    dy, dlast = rand((batch, length, channels), dtype, 77), rand((batch, channels), F32, 78)
    g = torch.Generator().manual_seed(41)
    for t in (s["x"], s["forget"], s["out"], dy):
        t[torch.rand(t.shape, generator=g) < 0.001] = NAN
        for i, end in enumerate(s["lengths"].tolist()):
            t[i, end:] = NAN
    for i, end in enumerate(s["lengths"].tolist()):
        s["resets"][i, end:] = 1
    check(A, s, dtype, dy, dlast)


@pytest.mark.parametrize("place,reset", [(50, 60), (58, 60), (59, 60), (60, 60), (60, 61), (63, 64), (64, 127), (130, 383), (500, 515), (0, 1023)])
def test_a_gate_that_is_nan_and_a_document_behind_it(A, place, reset):
    """Within the run of a thread, a wave, a block and a part, and across their ends."""
    for b, n, c in ((1, 1100, 20), (260, 1100, 5)):
        for dtype in (BF16, F32):
            s = recurrence_case(b, n, c, dtype, True, True, True, False, False, 34)
            s["resets"] = torch.zeros(b, n, dtype=torch.uint8)
            s["resets"][:, reset] = 1
            s["forget"][:, place] = NAN
            g = run_forward(A, s, dtype)
            y = torch.isnan(g["y"])
            if place < reset:
                assert not y[:, :place].any() and y[:, place:reset].all() and not y[:, reset:].any()
            else:   # the place that begins a document is the one
                assert not y[:, :place].any() and y[:, place:].all()
            got = backward(A, g, rand((b, n, c), dtype, 77), rand((b, c), F32, 78), dtype)
            dx = torch.isnan(got["dx"])
            # gradients come from behind up to the document's beginning: through the gate to all places before it, but not through a reset
            if place < reset:
                assert dx[:, :place + 1].all() and not dx[:, place + 1:].any()
            else:
                assert not dx[:, :place].any() and dx[:, place].all() and not dx[:, place + 1:].any()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shut", [False, True])
@pytest.mark.parametrize("batch,length,channels", SHAPES)
def test_resets_that_are_all_zero_are_none(A, batch, length, channels, shut, dtype):
    """Bit for bit, with values that are not finite and gates that are nearly shut."""
    s = recurrence_case(batch, length, channels, dtype, True, True, True, True, False, 35)
    if shut:
        s["bias"] = torch.full((channels,), -12.0)
    s["x"][0, length // 3] = NAN
    s["x"][-1, length // 4] = INF
    dy, dlast = rand((batch, length, channels), dtype, 77), rand((batch, channels), F32, 78)
    dy[0, length // 2] = NAN
    results = []
    for resets in (None, torch.zeros(batch, length, dtype=torch.uint8)):
        s["resets"] = resets
        g = run_forward(A, s, dtype)
        results.append([g["y"], g["last"], g["states"], *backward(A, g, dy, dlast, dtype).values()])
    for i, (one, other) in enumerate(zip(*results)):
        assert torch.all((one == other) | (torch.isnan(one) & torch.isnan(other))), i


@pytest.mark.parametrize("shut", [False, True])
def test_the_whole_sequence_is_not_finite_where_its_tokens_are(A, shut):
    """At once, in parts and blocks, and a few places at a time with the state carried along."""
    b, n, c = 2, 1300, 12
    s = recurrence_case(b, n, c, F32, False, True, True, False, False, 36)
    s["resets"] = documents(b, n, 37)
    if shut:
        s["bias"] = torch.full((c,), -12.0)
    at = torch.rand(b, n, generator=torch.Generator().manual_seed(38)) < 0.01
    s["forget"][at] = NAN
    s["x"][at.roll(5, 1)] = NAN
    whole = run_forward(A, s, F32)
    state, ws, rows = whole["first"].clone(), room(A.adacomp_recurrence_workspace_bytes(b, 10, c)), []
    for t in range(0, n, 10):
        y = torch.empty(b, 10, c, device=DEV)
        A.adacomp_recurrence_forward(whole["x"][:, t:t + 10], whole["forget"][:, t:t + 10], y, ws, bias=whole["bias"], first=state, last=state, resets=whole["resets"][:, t:t + 10])
        rows.append(y)
    assert torch.equal(torch.isfinite(torch.cat(rows, 1)), torch.isfinite(whole["y"])) and torch.equal(torch.isfinite(state), torch.isfinite(whole["last"]))
