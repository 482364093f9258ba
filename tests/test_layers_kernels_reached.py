"""The layer kernels that the library holds are those that calls reach: forms of rows shorter than a group of 8, inputs past the caches."""
import os
import re
import shutil
import subprocess

import pytest

from paper_1712_02679_amd import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SHORT_FORMS = r"""
#include <cstdio>
#include "layers_plan.h"
int main()
{
    for (uint32_t keys = 0; keys < 8; ++keys)
        for (uint32_t places = 1; places <= 2 * ADACOMP_BIAS_DISTANCE_MAX + 1; ++places) {
            const adacomp::SoftmaxForm f = adacomp::softmax_form(keys, places, true);
            std::printf("%u %u %u\n", f.row.threads, f.row.groups, f.parts);
        }
    return 0;
}
"""


@pytest.fixture(scope="module")
def kernels():
    if not os.path.exists(binding.LIB_PATH):
        from paper_1712_02679_amd import build
        build.build()
    return subprocess.run(["nm", "-D", "--defined-only", binding.LIB_PATH], capture_output=True, text=True, check=True).stdout


def test_backward_softmax_has_the_forms_that_short_rows_take(kernels, tmp_path):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not (os.path.exists(hipcc) or shutil.which("hipcc")):
        pytest.skip("no hipcc")
    source, exe = tmp_path / "forms.hip", tmp_path / "forms"
    source.write_text(SHORT_FORMS)
    subprocess.run([hipcc, "--offload-host-only", "-std=c++17", "-I" + os.path.join(ROOT, "include"), "-I" + os.path.join(ROOT, "paper_1712_02679_amd", "csrc"),
                    "-o", str(exe), str(source), "-L" + os.path.dirname(binding.LIB_PATH), "-ladacomp", "-Wl,-rpath," + os.path.dirname(binding.LIB_PATH)], check=True, capture_output=True)
    lines = set(subprocess.run([str(exe)], capture_output=True, text=True, check=True, timeout=60).stdout.split("\n")) - {""}
    taken = {tuple(int(n) for n in line.split()) for line in lines}
    assert all(parts == 1 for _, _, parts in taken)
    # forms of 8 threads look at the row's length themselves
    wanted = {(threads, groups) for threads, groups, _ in taken if threads > 8}
    for dtype in ("f", "DF16b", "DF16_"):
        built = {(int(t), int(g)) for t, g in re.findall(r"k_softmax_backwardI%sLi(\d+)ELi(\d+)ELi0ELi2E" % dtype, kernels)}
        assert built == wanted, dtype


def test_only_16_bit_dropout_goes_past_the_caches(kernels):
    built = set(re.findall(r"k_dropoutI(f|DF16b|DF16_)Lb([01])E", kernels))
    assert built == {("f", "0"), ("DF16b", "0"), ("DF16b", "1"), ("DF16_", "0"), ("DF16_", "1")}
