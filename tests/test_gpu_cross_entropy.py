"""Cross entropy, the distillation calls with targets alone, over rows of all lengths: losses, both at once, and the gradient from the logarithms that were kept."""
import numpy as np
import pytest
import torch

import sequence_reference as S
from layers_reference import within
from test_gpu_sequence import BF16, DEV, F32, TYPES, on_gpu, rand, rounded, untouched

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab,pad,lead", [(1, 1, 0, 0), (40, 7, 0, 0), (200, 65, 3, 1), (45, 256, 0, 0), (45, 257, 0, 0), (33, 1001, 1, 2), (23, 1024, 0, 0), (20, 1025, 0, 0), (9, 5999, 0, 0), (5, 16384, 0, 0),
                                                 (5, 16385, 3, 1), (3, 50001, 0, 0), (2, 131072, 0, 0), (1, 200003, 0, 0)])
def test_targets_alone(rows, vocab, pad, lead, dtype):
    import paper_1712_02679_amd as A
    z, targets = rand((rows, vocab), dtype, 50, 3.0), torch.randint(0, vocab, (rows,), generator=torch.Generator().manual_seed(51))
    targets[1::7], targets[2::11], targets[0] = -100, vocab, vocab - 1
    dloss, hard, scale = torch.where(torch.arange(rows) % 5 == 4, 0.0, rand((rows,), F32, 52)), float(np.float32(0.3)), float(np.float32(1.7))
    # the temperature is the teacher's: without one it does nothing
    for index, temperature in ((torch.int64, 1.0), (torch.int32, 2.5)):
        d = S.Distill(z.double(), targets=targets, hard=hard)
        gz, args = on_gpu(z, pad, lead), dict(targets=targets.to(index).to(DEV), temperature=temperature, hard=hard)
        loss, lse, again = (torch.full(s, float("nan"), device=DEV) for s in ((rows,), (rows, 2), (rows,)))
        A.adacomp_distill_forward(gz, loss, lse=lse, **args)
        within(loss, d.loss, d.loss_off, "loss")
        within(lse, d.lse, torch.where(d.lse == 0, 0.0, d.lse_off), "lse")
        told = torch.nn.functional.cross_entropy(z.double(), torch.where(d.told, targets, -100), reduction="none", ignore_index=-100) * hard
        within(loss, told, d.loss_off, "cross entropy")
        for at_once in (True, False):
            got = on_gpu(torch.full((rows, vocab), float("nan"), dtype=dtype), pad, lead)
            if at_once:
                A.adacomp_distill_forward(gz, again, dlogits=got, dloss=dloss.to(DEV), scale=scale, **args)
                assert torch.equal(again, loss)
            else:
                A.adacomp_distill_backward(gz, lse, got, dloss=dloss.to(DEV), scale=scale, **args)
            want, off = d.gradient(dloss.double(), scale, from_lse=not at_once)
            within(got, want, rounded(want, off, dtype), ("dlogits", at_once))
            if pad or lead:
                untouched(got, pad, lead)


@pytest.mark.parametrize("rows,vocab", [(4096, 1025), (4097, 5000), (4100, 8192), (4096, 8193), (600, 20000)])
def test_many_rows(rows, vocab):
    """The forms of many rows: the first rows against the formula, all against one another."""
    import paper_1712_02679_amd as A
    few, g = rand((16, vocab), BF16, 53, 3.0), torch.Generator().manual_seed(54)
    target, pick = torch.randint(0, vocab, (16,), generator=g), torch.randint(0, 16, (rows,), generator=g)
    target[3], pick[:16], pick[-16:] = -1, torch.arange(16), torch.arange(16)
    z, targets = few.to(DEV)[pick.to(DEV)], target[pick].to(DEV)
    loss, lse, grad, back = torch.empty(rows, device=DEV), torch.empty(rows, 2, device=DEV), torch.empty_like(z), torch.empty_like(z)
    A.adacomp_distill_forward(z, loss, lse=lse, targets=targets, dlogits=grad)
    A.adacomp_distill_backward(z, lse, back, targets=targets)
    d = S.Distill(few.double(), targets=target)
    within(loss[:16], d.loss, d.loss_off, "loss")
    for got, from_lse in ((grad, False), (back, True)):
        want, off = d.gradient(torch.ones(16, dtype=torch.float64), from_lse=from_lse)
        within(got[:16], want, rounded(want, off, BF16), ("dlogits", from_lse))
        assert torch.equal(got, got[:16][pick.to(DEV)])
    assert torch.equal(loss, loss[:16][pick.to(DEV)]) and torch.equal(lse, lse[:16][pick.to(DEV)])
