"""Launches of the recurrence at the limits of their sizes."""
import os
import shutil
import subprocess

import pytest
import torch

import sequence_reference as S
from layers_reference import within
from test_gpu_sequence import DEV, F32, rand, room, rounded

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

LAUNCHES = r"""
#include <cstdio>
#include "sequence_plan.h"
int main()
{
    using namespace adacomp;
    for (uint32_t channels : {1u, 64u, 65u, 4096u, 8191u, 1u << 20})
        for (uint64_t batch : {1ull, 255ull, 256ull, (1ull << 22) - 1, 1ull << 22, (1ull << 22) + 1, (1ull << 23) - 1, 1ull << 23, (1ull << 23) + 1, (1ull << 31) - 1})
            for (uint32_t length : {1u, 33u, 1000u, 65536u, (1u << 31) - 1u}) {
                if (batch * length >= 1ull << 31) continue;
                const RecurrenceForm form = recurrence_form(uint32_t(batch), length, channels);
                const uint64_t of_one = uint64_t((channels + kSlab - 1u) / kSlab) * form.segments, step = recurrence_sequences(uint32_t(of_one));
                if (step == 0 || of_one > UINT32_MAX || step * of_one * kRecurrenceThreads > UINT32_MAX) {
                    std::printf("%llu x %u x %u: %llu sequences of %llu workgroups\n", (unsigned long long)batch, length, channels, (unsigned long long)step, (unsigned long long)of_one);
                    return 1;
                }
            }
    std::printf("all launches ok\n");
    return 0;
}
"""


def test_recurrence_launches_have_fewer_than_2_to_the_32_threads(tmp_path):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not (os.path.exists(hipcc) or shutil.which("hipcc")):
        pytest.skip("no hipcc")
    source, exe = tmp_path / "launches.hip", tmp_path / "launches"
    source.write_text(LAUNCHES)
    subprocess.run([hipcc, "--offload-host-only", "-std=c++17", "-I" + os.path.join(ROOT, "include"), "-I" + os.path.join(ROOT, "paper_1712_02679_amd", "csrc"),
                    "-o", str(exe), str(source)], check=True, capture_output=True)
    res = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert res.returncode == 0 and "all launches ok" in res.stdout, res.stdout + res.stderr


@pytest.mark.gpu
def test_recurrence_of_more_sequences_than_one_launch_takes():
    """2^23 sequences and one more, of one channel, in 32 bits with a gate: 512 threads to each in the backward pass. All read the same values, and begin and end with their own states."""
    import paper_1712_02679_amd as A
    b, n = (1 << 23) + 1, 33
    one = {name: rand((1, n, 1), F32, 40 + i) for i, name in enumerate(("x", "forget", "out", "dy"))}
    g = {name: t.to(DEV).expand(b, n, 1) for name, t in one.items()}
    first, dlast = (torch.randn(b, 1, generator=torch.Generator(device=DEV).manual_seed(k), device=DEV) for k in (44, 45))
    ws, nan = room(A.adacomp_recurrence_workspace_bytes(b, n, 1)), float("nan")
    y, last, states = torch.full((b, n, 1), nan, device=DEV), torch.full((b, 1), nan, device=DEV), torch.full((b, 1, 1), nan, device=DEV)
    A.adacomp_recurrence_forward(g["x"], g["forget"], y, ws, out=g["out"], first=first, last=last, states=states)
    assert torch.equal(states[:, 0], first) and torch.isfinite(y).all() and torch.isfinite(last).all()
    dx, df, do, dfirst = (torch.full(s, nan, device=DEV) for s in ((b, n, 1),) * 3 + ((b, 1),))
    A.adacomp_recurrence_backward(g["dy"], g["x"], g["forget"], states, dx, df, ws, out=g["out"], dout=do, dlast=dlast, dfirst=dfirst)
    for t in (dx, df, do, dfirst):
        assert torch.isfinite(t).all()
    for at in (0, (1 << 22) - 4, (1 << 23) - 7):   # the launches' ends
        some = slice(at, at + 8)
        wide = {name: t.double().expand(8, n, 1) for name, t in one.items()}
        r = S.Recurrence(wide["x"], wide["forget"], wide["out"], None, first[some].cpu().double())
        within(y[some], r.y, r.y_bound(F32), ("y", at))
        within(last[some], r.last, r.last_bound(), ("last", at))
        want = r.backward(wide["dy"], dlast[some].cpu().double())
        for name, got in (("dx", dx), ("dforget", df), ("dout", do), ("dfirst", dfirst)):
            within(got[some], want[name][0], rounded(*want[name], F32), (name, at))
    del y, dx, df, do
    torch.cuda.empty_cache()
