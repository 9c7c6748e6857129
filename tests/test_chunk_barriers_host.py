"""The barriers of chunk_attn_kernel as a model: those of the shared-prefix attention, and what is different here: the lanes of a single M tile join what
they have through tensor memory, and a segment's pages are checked behind its publication.  That the model notices is shown with mistakes planted in it."""
import random

import pytest

from test_shared_barriers_host import SEGMENTS, STAGES, Barrier, Kernel, _segments


class Chunk(Kernel):
    def __init__(self, segments, seed, mistake=None):
        super().__init__(segments, seed, None)
        self.wrong = mistake
        self.checked, self.verdict = [Barrier(1) for _ in range(SEGMENTS)], [None] * SEGMENTS
        self.other_full, self.other = Barrier(4), [None] * 4

    def planner(self):
        for k in range(len(self.segments) + 1):
            at, turn = k % SEGMENTS, k // SEGMENTS
            while not self.seg_empty[at].done(turn - 1, turn & 1 ^ 1):
                yield
            self.seg[at] = (k,) + (self.segments[k] if k < len(self.segments) else (False, 0, False))
            self.seg_full[at].arrive()
            if k == len(self.segments):
                return
            for _ in range(self.r.randrange(60)):              # the look at the pages
                yield
            self.verdict[at] = k
            self.checked[at].arrive()

    def softmax(self, l, warp):
        ops = segs = tile0 = joins = 0
        for k in range(len(self.segments) + 1):
            at = k % SEGMENTS
            while not self.seg_full[at].done(k // SEGMENTS, k // SEGMENTS & 1):
                yield
            _, single, n, ragged = self.seg[at]
            if n == 0:
                return
            turn = tile0 & 1 ^ l if single else l
            first, has_rows = True, (k + warp) % 3 > 0          # (some warps of some segments have no rows)
            for t in range(turn if single else 0, n, 2 if single else 1):
                while not self.s_full[l].done(ops, ops & 1):
                    yield
                assert self.S[l][warp] == ("S", k, t)
                yield
                if ragged and t == n - 1:
                    stage = (2 * (tile0 + t) + 1) % STAGES
                    while not self.v_there[l].done(ops, ops & 1):
                        yield
                    assert self.kv[stage] == (k, t, 1)
                    self.zeros[stage][l].add(warp)
                for h in range(2) if has_rows else ():
                    self.S[l][warp] = ("P", k, t, h)
                    self.p_ready[l][h].arrive()
                    yield
                if not has_rows:
                    self.S[l][warp] = ("P", k, t, 1)
                    self.p_ready[l][0].arrive()
                    self.p_ready[l][1].arrive()
                first, ops = False, ops + 1
            while self.wrong != "nobody waits for the check" and not self.checked[at].done(k // SEGMENTS, k // SEGMENTS & 1):
                yield
            assert self.verdict[at] == k, "not checked"
            two = single and n > 1
            if not first:
                while not self.o_full[l].done(segs, segs & 1):
                    yield
                segs += 1
                assert self.O[l][0] == k
            if not first and two and turn != (n - 1) % 2:
                assert self.other[warp] is None, "still to be read"
                self.other[warp] = k
                yield
                self.other_full.arrive()
                if self.wrong == "a lane frees its own accumulators":
                    self.o_free[l].arrive()
            elif not first:
                if two:
                    while not self.other_full.done(joins, joins & 1):
                        yield
                    assert self.other[warp] == k
                    self.other[warp] = None
                    for _ in range(self.r.randrange(20)):
                        yield
                    assert self.O[l ^ 1][0] == k, "the other lane's accumulators are another segment's"
                    self.results[k, 1 - turn, warp] = list(self.O[l ^ 1][1])
                self.results[k, turn, warp] = list(self.O[l][1])
                yield
                self.o_free[l].arrive()
                if two and self.wrong != "a lane frees its own accumulators":
                    self.o_free[l ^ 1].arrive()
            joins += two
            tile0 += n
            self.seg_empty[at].arrive()


@pytest.mark.parametrize("block", range(4))
def test_every_schedule_runs_through(block):
    for seed in range(100 * block, 100 * block + 100):
        Chunk(_segments(random.Random(seed)), seed).run()


@pytest.mark.parametrize("mistake,told", [("a lane frees its own accumulators", "are another segment's"), ("nobody waits for the check", "not checked")])
def test_the_model_notices(mistake, told):
    for seed in range(400):
        try:
            Chunk(_segments(random.Random(seed)), seed, mistake).run()
        except AssertionError as e:
            assert told in str(e), e
            return
    pytest.fail("not noticed")
