"""AddressSanitizer / UndefinedBehaviorSanitizer build of the host code of a gated residual
block's operators, against the stub HIP runtime, on the CPU (tests/sanitize/block_checks.c)."""
import os
import re
import subprocess

import pytest

from test_act_sanitizers import CLANG, CSRC, FLAGS, HIPCC, ROOT, SAN, _run


@pytest.mark.skipif(not (os.path.exists(HIPCC) and os.path.exists(CLANG)), reason="ROCm toolchain missing")
def test_host_code_of_the_gated_block(tmp_path):
    units = [f for f in sorted(os.listdir(CSRC)) if f.endswith((".hip", ".cpp")) and f.startswith(("block_", "drop", "gate", "join"))]
    host_san = [a for flag in FLAGS for a in ("-Xarch_host", flag)]
    jobs = [(f, subprocess.Popen([HIPCC, "-x", "hip", "--offload-host-only", "-O1", "-g", "-std=c++17", "-fPIC",
                                  "-I", os.path.join(ROOT, "include"), "-I", CSRC, *host_san, "-w",
                                  "-c", os.path.join(CSRC, f), "-o", str(tmp_path / (f + ".o"))])) for f in units]
    assert [f for f, j in jobs if j.wait() != 0] == []
    objs = [str(tmp_path / (f + ".o")) for f in units]
    fat = sorted(set(re.findall(r"\b(__hip_fatbin_[0-9a-f]+)\b", _run(["nm", "-u", *objs]).stdout)))
    (tmp_path / "fatbins.c").write_text("".join(f"char {s}[16];\n" for s in fat))
    exe = str(tmp_path / "block_checks")
    _run([CLANG, "-O1", "-g", *FLAGS, "-DSTUB_ATTR_CUS=1", "-DSTUB_ATTR_LDS=2", "-I", os.path.join(ROOT, "include"), "-o", exe,
          os.path.join(SAN, "block_checks.c"), os.path.join(SAN, "hip_stub.c"), str(tmp_path / "fatbins.c"), *objs,
          "-lstdc++", "-lm", "-lpthread"])
    r = _run([exe], env=dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=1",
                             UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1"))
    assert "launches" in r.stdout
    print(r.stdout)
