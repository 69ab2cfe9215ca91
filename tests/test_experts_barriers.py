"""The tiles of the experts' products, as those of the linear operators: no LDS access of a wave may still be under way
where it reaches a barrier. Read from the compiler's own assembly, so no GPU is needed."""
import os
import shutil
import subprocess

import pytest

from paper_2609_05255_amd import build as gsbuild
from test_linear_barriers import accesses_under_way


@pytest.mark.skipif(shutil.which(gsbuild.HIPCC) is None, reason="no hipcc")
@pytest.mark.parametrize("name", ["experts_f32", "experts_bf16"])
def test_no_lds_access_is_under_way_at_a_barrier(tmp_path, name):
    src, asm = os.path.join(gsbuild.CSRC, name + ".hip"), str(tmp_path / "experts.s")
    subprocess.run([gsbuild.HIPCC, *gsbuild.COMMON, "-S", "--offload-device-only", src, "-o", asm], check=True,
                   capture_output=True)
    text = open(asm).read()
    assert "k_gemm_pair" in text and accesses_under_way(text) == []
