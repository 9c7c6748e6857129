"""After a wait that ran out, a block of the paged kernels waits once more, with a limit, for its own copies in flight.  Looked for in the sources, barrier by
barrier: every one that copies arrive at is drained in the branch behind its role's loop.  And the parities of those waits, as a model: the phase of the
last copy that began, wherever the role gave up.  That the look notices is shown on texts that lack a drain."""
import os
import random
import re

import pytest

from paper_2604_02047_b200 import build


def _source(name):
    with open(os.path.join(build.CSRC, name)) as f:
        return re.sub(r"//.*", "", f.read())


def _block(text, at):
    """The statement or braces behind position ``at``."""
    depth = 0
    for i in range(at, len(text)):
        depth += {"{": 1, "}": -1, "(": 1, ")": -1}.get(text[i], 0)
        if depth == 0 and text[i] in ";}":
            return text[at:i + 1]
    raise AssertionError("no end")


def _copied(text):
    """Barriers that expect the bytes of copies, by name."""
    names = set()
    for target in re.findall(r"mbar_expect_tx\(([^,]+),", text):
        if "hd->" in target:
            names |= set(re.findall(r"hd->(\w+)", target))
        else:                                                  # a pointer: what it is set to
            for value in re.findall(r"\*\s*(?:const\s+)?%s = ([^;]+);" % re.escape(target.strip()), text):
                names |= set(re.findall(r"hd->(\w+full)\b", value))
    return names


def _drained(text):
    """Barriers that are drained where a role has given up, and whether its 16-byte copies are waited for."""
    names, copies = set(), False
    for m in re.finditer(r"if \(!ok\)\s*", text):
        block = _block(text, m.end())
        names |= set(re.findall(r"\bdrain\(&hd->(\w+)", block))
        copies |= "cp_async_wait_all()" in block
    return names, copies


def _look(text):
    names, copies = _drained(text)
    assert _copied(text) and _copied(text) <= names, _copied(text) - names
    assert copies or "cp_async_16(" not in text, "16-byte copies"


@pytest.mark.parametrize("source,barriers", [("chunk_attn.cu", {"kv_full", "pair_full", "single_full"}), ("kv_weights.cu", {"q_full"})])
def test_every_barrier_of_a_copy_is_drained(source, barriers):
    text = _source(source)
    assert _copied(text) == barriers
    _look(text)
    drains = re.findall(r"drain\(&hd->\w+\[[^;]+;|cp_async_wait_all\(\);", text)
    assert len(drains) == len(barriers) + (source == "kv_weights.cu")
    for d in drains:
        with pytest.raises(AssertionError):
            _look(text.replace(d, ";"))


def test_the_waits_are_bounded():
    for source in ("chunk_attn.cu", "kv_weights.cu"):
        text = _source(source)
        m = re.search(r"void drain\([^)]*\)\s*", text)
        assert re.search(r"clock64\(\) - t0 < kWaitCycles", _block(text, m.end()))


def test_parities_of_the_last_copies():
    """The producer of chunk_attn_kernel, giving up at any place: stages by who has them, the queries' places of pairs and of single tiles in turn."""
    for seed in range(3000):
        r = random.Random(seed)
        began = {}                                             # copies that a barrier has been given
        phases, users, pairs, singles, tile0, stage = {}, {}, 0, 0, 0, 0
        sg_n, single, asked = 0, False, set()

        def start(name, began=began):
            began[name] = began.get(name, 0) + 1

        def load_q(b):
            start(("single" if single else "pair", b))
            asked.discard(b)

        try:
            for _ in range(r.randint(1, 8)):
                def step():
                    if r.random() < 0.03:
                        raise StopIteration
                for b in sorted(asked):
                    step()
                    load_q(b)
                if sg_n > 0:
                    singles, pairs, sg_n = singles + single, pairs + (not single), 0
                step()
                sg_n, single = r.randint(1, 5), r.random() < 0.5
                asked.update({singles & 1} if single else {0, 1})
                for i in range(sg_n):
                    for _ in range(2):
                        while asked and r.random() < 0.4:
                            load_q(r.choice(sorted(asked)))
                        step()
                        user = (tile0 + i) & 1 if single else 2
                        start(("kv", user, stage))
                        phases[user, stage] = phases.get((user, stage), 0) ^ 1
                        users[stage] = user
                        stage = (stage + 1) % 5
                tile0 += sg_n
        except StopIteration:
            pass
        for at, user in users.items():                         # what the branch waits for
            assert phases[user, at] ^ 1 == (began["kv", user, at] - 1) & 1
        if sg_n > 0 and single and not asked:
            singles += 1
        for b in range(2):
            of_pairs, of_singles = pairs + (sg_n > 0 and not single and b not in asked), (singles + 1 - b) >> 1
            assert of_pairs == began.get(("pair", b), 0) and of_singles == began.get(("single", b), 0)
