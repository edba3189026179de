"""The join's plan of its backward pass, on the CPU (tests/sanitize/join_plan.cpp): the sizes of
test_gpu_join_units.py run every form of the kernel, each with workgroups that have no unit in the
last turn, and the workspace holds all workgroups' and units' sums."""
import os
import re
import subprocess

import pytest

from test_gpu_join_units import UNITS

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SAN, CSRC = os.path.join(ROOT, "tests", "sanitize"), os.path.join(ROOT, "paper_1903_06681_amd", "csrc")
HIPCC, CLANG = "/opt/rocm/bin/hipcc", "/opt/rocm/lib/llvm/bin/clang"


def _run(cmd):
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, (cmd[0], r.stdout[-3000:], r.stderr[-3000:])
    return r


@pytest.mark.skipif(not (os.path.exists(HIPCC) and os.path.exists(CLANG) and os.path.isdir(SAN)), reason="ROCm toolchain or sources missing")
def test_sizes_with_idle_workgroups(tmp_path):
    sources = [os.path.join(CSRC, "join_fwd.hip"), os.path.join(CSRC, "join_bwd.hip"), os.path.join(SAN, "join_plan.cpp")]
    objs = [str(tmp_path / (os.path.basename(s) + ".o")) for s in sources]
    jobs = [subprocess.Popen([HIPCC, "-x", "hip", "--offload-host-only", "-O1", "-std=c++17", "-fPIC", "-I", os.path.join(ROOT, "include"),
                              "-I", CSRC, "-w", "-c", s, "-o", o]) for s, o in zip(sources, objs)]
    assert [j.wait() for j in jobs] == [0] * len(jobs)
    fat = sorted(set(re.findall(r"\b(__hip_fatbin_[0-9a-f]+)\b", _run(["nm", "-u", *objs]).stdout)))
    (tmp_path / "fatbins.c").write_text("".join(f"char {s}[16];\n" for s in fat))
    exe = str(tmp_path / "join_plan")
    _run([CLANG, "-O1", "-DSTUB_ATTR_CUS=1", "-DSTUB_ATTR_LDS=2", "-o", exe, os.path.join(SAN, "hip_stub.c"), str(tmp_path / "fatbins.c"),
          *objs, "-lstdc++", "-lm"])
    sizes = [(form, s) for form, some in UNITS.items() for s in some]
    lines = "".join(f"{N} {H * W} {C} {int(form[0] == 'rows')} 1\n" for form, (N, C, H, W) in sizes)
    out = subprocess.run([exe], input=lines, capture_output=True, text=True, check=True).stdout.split("\n")
    for (form, shape), line in zip(sizes, out):
        lpx, held, grid, units, need = map(int, line.split())
        assert (lpx, held) == form[1:], shape
        assert units % grid, shape                       # the last turn has workgroups without a unit
        width = -(-shape[1] // 32) * 32
        assert need >= 4 * width * (4 * grid + units), shape
    forms = set(re.findall(r"join_bwd_kernel<(\d+), (\d+), (true|false)>", open(os.path.join(CSRC, "join_bwd.hip")).read()))
    assert {("true" if k == "rows" else "false", str(lpx), str(held)) for k, lpx, held in UNITS} == {(cl, lpx, r) for lpx, r, cl in forms}
