"""Distillation over fewer logits than a thread takes at once, with more top tokens than logits: the rule that picks a kernel, and its results."""
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

import sequence_reference as S
from layers_reference import within
from test_gpu_sequence import BF16, DEV, F16, F32, distill_case, rounded

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

FORMS = r"""
#include <cstdio>
#include "sequence_plan.h"
int main()
{
    using namespace adacomp;
    for (uint64_t rows : {1ull, 511ull, 512ull, 4095ull, 4096ull, 1ull << 30})
        for (uint32_t vocab = 1; vocab <= 20000; ++vocab)
            for (uint32_t top : {0u, 1u, 158u, 159u, 160u, ADACOMP_TEACHER_TOP_MAX}) {
                const DistillForm f = distill_form(rows, vocab, top);
                const uint32_t teams = f.threads > 256u ? 1u : 256u / f.threads, entries = (top + 4u) & ~3u;
                const bool fits = (!f.held || f.threads * f.groups * 8u >= vocab) && (vocab >= 8u || f.short_rows());   // groups of 8 are read from the end of a row that has them
                if (!fits || teams * entries * 12u > (64u << 10)) { std::printf("%llu rows of %u, %u top tokens: %u threads, held %u\n", (unsigned long long)rows, vocab, top, f.threads, f.held); return 1; }
            }
    std::printf("all forms ok\n");
    return 0;
}
"""


def test_forms_take_the_rows_that_they_are_given(tmp_path):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not (os.path.exists(hipcc) or shutil.which("hipcc")):
        pytest.skip("no hipcc")
    source, exe = tmp_path / "forms.hip", tmp_path / "forms"
    source.write_text(FORMS)
    subprocess.run([hipcc, "--offload-host-only", "-std=c++17", "-I" + os.path.join(ROOT, "include"), "-I" + os.path.join(ROOT, "paper_1712_02679_amd", "csrc"),
                    "-o", str(exe), str(source)], check=True, capture_output=True)
    res = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert res.returncode == 0 and "all forms ok" in res.stdout, res.stdout + res.stderr


def guarded(t, fill):
    """A copy on the GPU with other values right before and behind it."""
    flat = torch.full((t.numel() + 64,), fill, dtype=t.dtype, device=DEV)
    part = flat[32:32 + t.numel()].view(t.shape)
    part.copy_(t)
    return part, flat


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("top", [159, 160, 256])
@pytest.mark.parametrize("vocab", [1, 2, 3, 4, 5, 6, 7, 8, 255, 256])
def test_few_logits_and_many_top_tokens(vocab, top, dtype):
    import paper_1712_02679_amd as A
    rows, nan = 45, float("nan")
    s = distill_case(rows, vocab, top, dtype, 10 * vocab + top)
    z, _ = guarded(s["z"], nan)
    tau, soft, hard = 1.5, float(np.float32(0.7)), float(np.float32(0.3))
    d = S.Distill(s["z"].double(), s["tokens"], s["t"].double(), s["targets"], tau, soft, hard)
    args = dict(teacher_tokens=s["tokens"].to(DEV), teacher_logits=s["t"].to(DEV), targets=s["targets"].to(DEV), temperature=tau, soft=soft, hard=hard)
    loss, lse = torch.full((rows,), nan, device=DEV), torch.full((rows, 2), nan, device=DEV)
    A.adacomp_distill_forward(z, loss, lse=lse, **args)
    within(loss, d.loss, d.loss_off, "loss")
    within(lse, d.lse, torch.where(d.lse == 0, 0.0, d.lse_off), "lse")
    for at_once in (True, False):
        got, around = guarded(torch.full((rows, vocab), nan, dtype=dtype), 3.0)
        if at_once:
            again = torch.full((rows,), nan, device=DEV)
            A.adacomp_distill_forward(z, again, dlogits=got, **args)
            assert torch.equal(again, loss)
        else:
            A.adacomp_distill_backward(z, lse, got, **args)
        want, off = d.gradient(torch.ones(rows, dtype=torch.float64), from_lse=not at_once)
        within(got, want, rounded(want, off, dtype), ("dlogits", at_once))
        assert torch.all(around[:32] == 3.0) and torch.all(around[-32:] == 3.0)
