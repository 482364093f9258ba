"""The steps of the example's recurrent student: its learners' gradients, packed and applied by the CPU oracle in place of the library, lead to the same weights bit for bit."""
import os
import sys

import numpy as np
import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def E():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import recurrent_student
    return recurrent_student


@pytest.mark.parametrize("learners", [1, 3])
def test_steps_are_adam_on_the_sum_of_all_packets(E, learners):
    import oracle
    orc, f32 = oracle.Oracle(), np.float32
    steps, batch, length, vocab, dim, top, rate, lr, seed = 4, 3, 30, 17, 24, 4, 0.1, 5e-3, 2
    losses, weights, layout = E.train(steps, learners, batch, length, vocab, dim, top, rate, lr, seed)
    text, table, n = E.Text(vocab, seed), layout.table, layout.total
    inside = np.zeros(n, bool)
    for at, count, _ in table:
        inside[at:at + count] = True
    w = E.initial_weights(layout, seed).cpu().numpy()
    start, m, v = w.copy(), np.zeros(n, f32), np.zeros(n, f32)
    residues, moved = [np.zeros(n, f32) for _ in range(learners)], 0
    students = [E.Student(layout, batch, length, rate, seed * 1000 + k) for k in range(learners)]
    dloss = torch.full((batch, length), 1.0 / (batch * (length - 1)), device=E.DEV)
    for step in range(1, steps + 1):
        packets, total = [], 0.0
        on_gpu = torch.from_numpy(w).to(E.DEV)
        for k, student in enumerate(students):
            tokens, targets, teacher_tokens, teacher_logits = text.batch(batch, length, top, (seed * 100003 + step) * 64 + k)
            total = total + (student.forward(tokens, on_gpu, step, teacher_tokens, teacher_logits, targets, dloss) * dloss).sum()
            grad = torch.zeros_like(on_gpu)
            student.backward(on_gpu, grad, step)
            packets.append(orc.compress(table, grad.cpu().numpy(), residues[k]))
        assert losses[step - 1] == (total / learners).item()
        dense = orc.unpack_accumulate(table, packets, n)
        dense[~inside] = 0
        moved += int(np.count_nonzero(dense))
        orc.update_adam(table, dense, learners, w, m, v, float(f32(lr)), 0.9, 0.999, 1e-8, float(f32(1.0 - 0.9 ** step)), float(f32(1.0 - 0.999 ** step)))
    assert moved > 0 and not np.array_equal(w, start)
    assert np.array_equal(weights.cpu().numpy().view(np.uint32), w.view(np.uint32))
