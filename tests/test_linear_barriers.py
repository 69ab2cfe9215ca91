"""The tiles of the linear operators write LDS anew behind hand-placed barriers: in the compiled kernels no LDS access of
a wave may still be under way where it reaches one. Read from the compiler's own assembly, so no GPU is needed."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2609_05255_amd import build as gsbuild


def accesses_under_way(text):
    """(kernel, line) of the barriers that have LDS accesses before them without a wait for all of them between."""
    out, kernel, under_way, barriers = [], None, 0, 0
    for number, line in enumerate(text.splitlines(), 1):
        label = re.match(r"(_Z\w*k_gemm\w*):", line)
        if line.startswith("_Z"):
            kernel, under_way = (label.group(1) if label else None), 0
        if kernel is None:
            continue
        line = line.strip()
        if line.startswith("ds_"):
            under_way += 1
        wait = re.match(r"s_waitcnt.*lgkmcnt\((\d+)\)", line)
        if wait:
            under_way = min(under_way, int(wait.group(1)))
        if line.startswith("s_barrier"):
            barriers += 1
            if under_way:
                out.append((kernel, number))
    assert barriers > 0
    return out


@pytest.mark.skipif(shutil.which(gsbuild.HIPCC) is None, reason="no hipcc")
def test_no_lds_access_is_under_way_at_a_barrier(tmp_path):
    src, asm = os.path.join(gsbuild.CSRC, "linear_f32.hip"), str(tmp_path / "linear.s")
    subprocess.run([gsbuild.HIPCC, *gsbuild.COMMON, "-S", "--offload-device-only", src, "-o", asm], check=True,
                   capture_output=True)
    assert accesses_under_way(open(asm).read()) == []
