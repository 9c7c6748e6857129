"""The kernels of the paged cache, looked at without a GPU: those that keep their working set in registers do not spill, a wait that runs out is followed by one for
the block's own copies, and the limits that the kernels count on are those of the header."""
import os
import re
import subprocess

import pytest

from paper_2604_02047_b200 import build


def _source(name):
    with open(os.path.join(build.CSRC, name)) as f:
        return re.sub(r"//.*", "", f.read())


@pytest.mark.parametrize("source,kernels", [("chunk_attn.cu", 2), ("kv_weights.cu", 2), ("evict_kv.cu", 4)])
def test_no_spills(tmp_path, source, kernels):
    cmd = [build._nvcc()] + build.NVCC_FLAGS + ["-Xptxas", "-v", "-c", os.path.join(build.CSRC, source), "-o", str(tmp_path / "x.o")]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    found = re.findall(r"Compiling entry function '(\w+)'.*?(\d+) bytes spill stores, (\d+) bytes spill loads", r.stdout + r.stderr, re.S)
    assert len(found) == kernels
    assert all((stores, loads) == ("0", "0") for _, stores, loads in found), found


@pytest.mark.parametrize("source,drains", [("chunk_attn.cu", [r"\bdrain\("]), ("kv_weights.cu", [r"\bdrain\(", r"cp_async_wait_all\("])])
def test_a_wait_that_ran_out_is_followed_by_a_drain(source, drains):
    text = _source(source)
    behind = text[text.index("GOOSE_ST_TIMEOUT"):]
    for d in drains:
        assert len(re.findall(d, behind)) > 1 or d.startswith("cp"), (source, d)
        assert re.search(d, behind), (source, d)


def test_the_register_split_is_what_a_block_is_launched_with():
    """setmaxnreg.inc draws on the registers of the launch: more than those would be waited for for good."""
    text = _source("chunk_attn.cu")
    few, many = map(int, re.search(r"kRegsFew = (\d+), kRegsMany = (\d+)", text).groups())
    threads = int(re.search(r"kChunkThreads = (\d+)", text).group(1))
    at_launch = 65536 // threads // 8 * 8
    assert threads == 384 and few + 2 * many <= 3 * at_launch and few % 8 == many % 8 == 0
    assert "setmaxnreg" not in _source("kv_weights.cu")


def test_a_selecting_block_has_its_words_in_shared_memory():
    with open(os.path.join(build.INCLUDE, "goose.h")) as f:
        rows = int(re.search(r"GOOSE_MAX_PAGED_ROWS (\d+)", f.read()).group(1))
    smem = int(re.search(r"kSelectSmem = (\d+)", _source("evict_kv.cu")).group(1))
    words = rows // 32 + 1
    assert 2 * 4 * words < smem and smem + 4 * 2048 + 1024 <= 232448
