"""A wait on copies that runs out: the kernel reports it and waits once more, with a limit again, for its own copies in flight before it returns, so that none
lands in shared memory that is another block's by then.  Looked for in the sources (no test makes a copy that does not arrive)."""
import os
import re

import pytest

from paper_2604_02047_b200 import build


@pytest.mark.parametrize("source,drains", [("adjust_logits.cu", r"mbar_wait_bounded\("), ("node_topk.cu", r"mbar_wait_bounded\("),
                                           ("tree_attn_shared.cu", r"drain\("), ("tree_attn_umma.cu", r"mbar_drain\(")])
def test_a_wait_that_ran_out_is_followed_by_a_drain(source, drains):
    with open(os.path.join(build.CSRC, source)) as f:
        text = re.sub(r"//.*", "", f.read())
    reported = text.index("GOOSE_ST_TIMEOUT")
    behind = text[reported:]
    if source in ("adjust_logits.cu", "node_topk.cu"):         # in the branch itself
        behind = behind[:behind.index("return")]
    assert re.search(drains, behind), source
