"""Arrivals that one lane makes for its whole warp, in the kernels' sources: an mbarrier arrival orders what its own thread did before it, and
nothing else.  What the other lanes did (zeros behind the last key, a tile's P, a segment's description) is only in front of it where
__syncwarp() stands between; that a warp has come together again behind a loop or a branch is its habit, not a promise."""
import os
import re

import pytest

from paper_2604_02047_b200 import build


def _statements(name):
    """(line number, code without comments) of the lines that have any."""
    with open(os.path.join(build.CSRC, name)) as f:
        text = f.read()
    text = re.sub(r"/\*.*?\*/", lambda m: re.sub(r"[^\n]", " ", m.group()), text, flags=re.S)
    return [(i, re.sub(r"//.*", "", line).strip()) for i, line in enumerate(text.split("\n"), 1) if re.sub(r"//.*", "", line).strip()]


@pytest.mark.parametrize("name", sorted(n for n in os.listdir(build.CSRC) if n.endswith((".cu", ".cuh"))))
def test_a_lane_arrives_for_its_warp_behind_a_syncwarp(name):
    lines = _statements(name)
    for (_, before), (i, line) in zip(lines, lines[1:]):
        if re.match(r"if \(lane == 0\)\s*\{?\s*(mbar_arrive|arrive_at)\(", line):
            assert before.endswith("__syncwarp();"), "%s:%d: %s" % (name, i, line)


def test_the_look_finds_them():
    lines = _statements("tree_attn_shared.cu")
    assert sum(bool(re.match(r"if \(lane == 0\)\s*\{?\s*(mbar_arrive|arrive_at)\(", line)) for _, line in lines) == 5
