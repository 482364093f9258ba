"""Launches of the layer calls at the limits of their sizes."""
import os
import shutil
import subprocess

import pytest
import torch

import layers_reference as R
from layers_reference import DEEP, HALF_STEP, TINY, U, within

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
DEV = "cuda:0"

FORWARD_LAUNCHES = r"""
#include <cstdio>
#include "layers_plan.h"
int main()
{
    using namespace adacomp;
    for (uint32_t cols = 1; cols <= ADACOMP_NORM_COLS_MAX; ++cols) {
        const RowForm row = {norm_forward_threads(cols), 0};
        const uint64_t rows = norm_forward_rows(row), threads = (rows + row.teams() - 1u) / row.teams() * row.workgroup();
        if (rows == 0 || threads > UINT32_MAX || row.threads * 32u < cols) { std::printf("%u columns: %llu rows, %llu threads\n", cols, (unsigned long long)rows, (unsigned long long)threads); return 1; }
    }
    std::printf("all widths ok\n");
    return 0;
}
"""


def test_norm_forward_launches_have_fewer_than_2_to_the_32_threads(tmp_path):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not (os.path.exists(hipcc) or shutil.which("hipcc")):
        pytest.skip("no hipcc")
    source, exe = tmp_path / "launches.hip", tmp_path / "launches"
    source.write_text(FORWARD_LAUNCHES)
    subprocess.run([hipcc, "--offload-host-only", "-std=c++17", "-I" + os.path.join(ROOT, "include"), "-I" + os.path.join(ROOT, "paper_1712_02679_amd", "csrc"),
                    "-o", str(exe), str(source)], check=True, capture_output=True)
    res = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert res.returncode == 0 and "all widths ok" in res.stdout, res.stdout + res.stderr


@pytest.mark.gpu
def test_norm_forward_of_more_wide_rows_than_one_launch_takes():
    """1024 threads to each of more than 2^22 rows, 69 GB of them: one row read over and over, and told apart by its dropout."""
    import paper_1712_02679_amd as A
    rows, cols = (1 << 22) + 3, 8200
    x = torch.randn(1, cols, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    y = torch.empty(rows, cols, dtype=torch.bfloat16, device=DEV)
    mean, rstd = torch.full((rows,), float("nan"), device=DEV), torch.full((rows,), float("nan"), device=DEV)
    A.adacomp_norm_forward(x.to(DEV).expand(rows, cols), None, None, y, dropout=A.Dropout(0.5, 21, 22), mean=mean, rstd=rstd)
    assert torch.isfinite(mean).all() and torch.isfinite(rstd).all()
    for first in (0, (1 << 21) - 2, (1 << 22) - 2, rows - 4):
        z = x.double() * R.factors(4, cols, 0.5, 21, 22, first)
        want, m, r = R.norm_forward(z, 1.0, 0.0, float(torch.tensor(1e-5)))
        size = z.abs().mean(-1, keepdim=True) * r[:, None]
        bound = HALF_STEP[torch.bfloat16] * 1.01 * want.abs() + U * DEEP * (1 + size) ** 2 * (1 + want.abs()) + TINY[torch.bfloat16]
        within(y[first:first + 4], want, bound, ("y", first))
        within(mean[first:first + 4], m, U * DEEP * z.abs().mean(-1), ("mean", first))
    del y
    torch.cuda.empty_cache()
