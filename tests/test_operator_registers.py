"""The kernels around the step that keep their working set in registers (a row of scores, the parts of a merge, a block's words) fit them: no form
of the shared-prefix attention, of its merge or of the logits' kernels spills."""
import os
import re
import subprocess

import pytest

from paper_2604_02047_b200 import build


@pytest.mark.parametrize("source,kernels", [("tree_attn_shared.cu", 4), ("adjust_logits.cu", 4)])
def test_no_spills(tmp_path, source, kernels):
    cmd = [build._nvcc()] + build.NVCC_FLAGS + ["-Xptxas", "-v", "-c", os.path.join(build.CSRC, source), "-o", str(tmp_path / "x.o")]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    found = re.findall(r"Compiling entry function '(\w+)'.*?(\d+) bytes spill stores, (\d+) bytes spill loads", r.stdout + r.stderr, re.S)
    assert len(found) == kernels
    assert all((stores, loads) == ("0", "0") for _, stores, loads in found), found
