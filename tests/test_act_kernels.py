"""The layer norm's kernels in the library are those that its plan picks: nothing is compiled
that no call reaches.  Reads the names of the library's own kernels; no GPU."""
import os
import re
import shutil
import subprocess

import pytest

import paper_1903_06681_amd as dc

LIB = os.path.join(os.path.dirname(dc.__file__), "libdc.so")


def plan(M, C, cl, backward):
    """(pixels of a wave, blocks a lane holds, rows of channels), as the planner's comments have it."""
    blocks = -(-C // 32)
    waves = -(-M // 64) * blocks
    lpx = (4 if blocks >= 16 else 16) if cl else 64 if blocks <= 16 and waves >= 2048 else 16
    side = 64 // lpx
    nw = min(-(-blocks // side), 8)
    held = -(-blocks // (nw * side))
    return lpx, 1 if held <= 1 else 2 if held == 2 and not cl and not (backward and lpx == 16) else 0, cl


@pytest.mark.skipif(not shutil.which("nm"), reason="no nm")
def test_every_norm_kernel_is_picked_for_some_size():
    names = subprocess.run(["nm", LIB], capture_output=True, text=True, check=True).stdout
    for kernel, types, backward in (("norm_fwd_kernel", 2, False), ("norm_bwd_kernel", 6, True)):
        want = {plan(M, C, cl, backward) for M in (1, 300, 5000, 70000, 1 << 20) for C in (1, 32, 64, 256, 512, 544, 1024, 1056, 4096, 4128, 9000)
                for cl in (False, True)}
        found = set(re.findall(rf"\d{kernel}I(\w+?)Li(\d+)ELi(\d+)ELb([01])E", names))
        assert {(int(lpx), int(held), cl == "1") for _, lpx, held, cl in found} == want, kernel
        assert len(found) == types * len(want)
