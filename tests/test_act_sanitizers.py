"""AddressSanitizer / UndefinedBehaviorSanitizer build of the host code of the operators
between two convolutions, against the stub HIP runtime, on the CPU (tests/sanitize/act_checks.c)."""
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SAN = os.path.join(ROOT, "tests", "sanitize")
CSRC = os.path.join(ROOT, "paper_1903_06681_amd", "csrc")
HIPCC, CLANG = "/opt/rocm/bin/hipcc", "/opt/rocm/lib/llvm/bin/clang"
FLAGS = ["-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-fno-omit-frame-pointer"]


def _run(cmd, **kw):
    r = subprocess.run(cmd, capture_output=True, text=True, **kw)
    assert r.returncode == 0, (cmd[0], r.stdout[-3000:], r.stderr[-3000:])
    return r


@pytest.mark.skipif(not (os.path.exists(HIPCC) and os.path.exists(CLANG)), reason="ROCm toolchain missing")
def test_host_code_of_the_block_operators(tmp_path):
    units = [f for f in sorted(os.listdir(CSRC)) if f.endswith((".hip", ".cpp")) and f.startswith(("act_", "ckpt", "norm", "linear"))]
    host_san = [a for flag in FLAGS for a in ("-Xarch_host", flag)]
    jobs = [(f, subprocess.Popen([HIPCC, "-x", "hip", "--offload-host-only", "-O1", "-g", "-std=c++17", "-fPIC",
                                  "-I", os.path.join(ROOT, "include"), "-I", CSRC, *host_san, "-w",
                                  "-c", os.path.join(CSRC, f), "-o", str(tmp_path / (f + ".o"))])) for f in units]
    assert [f for f, j in jobs if j.wait() != 0] == []
    objs = [str(tmp_path / (f + ".o")) for f in units]
    fat = sorted(set(re.findall(r"\b(__hip_fatbin_[0-9a-f]+)\b", _run(["nm", "-u", *objs]).stdout)))
    (tmp_path / "fatbins.c").write_text("".join(f"char {s}[16];\n" for s in fat))
    exe = str(tmp_path / "act_checks")
    _run([CLANG, "-O1", "-g", *FLAGS, "-DSTUB_ATTR_CUS=1", "-DSTUB_ATTR_LDS=2", "-I", os.path.join(ROOT, "include"), "-o", exe,
          os.path.join(SAN, "act_checks.c"), os.path.join(SAN, "hip_stub.c"), str(tmp_path / "fatbins.c"), *objs,
          "-lstdc++", "-lm", "-lpthread"])
    r = _run([exe], env=dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=1",
                             UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1"))
    assert "launches" in r.stdout
    print(r.stdout)
