"""Gradient of the embedding where every sum is exact, whatever its order: whole numbers, and a scale and a factor that are powers of two.  No place may be
lost, doubled or given to another token, of frequent tokens either, whose places lie in many pieces."""
import pytest
import torch

import sequence_reference as S
from test_gpu_sequence import DEV, TYPES, embed_room, on_gpu, tokens_of

pytestmark = pytest.mark.gpu

# (rows, vocabulary, columns, skew of the tokens, more columns behind and before)
CASES = [(1, 1, 1, 1.0, 0, 0), (64, 3, 8, 1.0, 0, 0), (5000, 300, 40, 1.0, 0, 0), (20000, 7, 16, 6.0, 0, 0), (20000, 7, 13, 6.0, 3, 1), (12800, 65, 512, 2.0, 0, 0), (30001, 900, 201, 4.0, 1, 2),
         (140000, 50, 33, 8.0, 0, 0), (40000, 20000, 65, 3.0, 0, 0), (3000, 2, 2056, 1.0, 0, 0)]


def whole_numbers(shape, dtype, seed):
    return torch.randint(-7, 8, shape, generator=torch.Generator().manual_seed(seed)).to(dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab,cols,skew,pad,lead", CASES)
def test_every_place_counts_once(rows, vocab, cols, skew, pad, lead, dtype):
    import paper_1712_02679_amd as A
    dy, before, ws = whole_numbers((rows, cols), dtype, 1), whole_numbers((vocab, cols), torch.float32, 2), embed_room(A, rows, vocab, cols)
    gdy = on_gpu(dy, pad, lead)
    for tokens in (tokens_of(rows, vocab, 3, skew), torch.full((rows,), vocab - 1)):
        for drop in (None, (0.5, 2 ** 62 + 5, 2 ** 33 + 1)):   # half of 65536 is kept: a factor of 2
            want, size, _ = S.embed_backward(tokens, dy.double(), vocab, 0.25, drop)
            assert size.max() * 4 < 2 ** 24   # every sum on the way is a whole number of float32 too
            for accumulate in (False, True):
                got = before.to(DEV)
                A.adacomp_embed_backward(tokens.to(DEV), gdy, got, ws, scale=0.25, dropout=A.Dropout(*drop) if drop else None, accumulate=accumulate)
                assert torch.equal(got.cpu().double(), want + before.double() if accumulate else want), (drop, accumulate)
