"""The barriers of tree_attn_shared_kernel as a model: planner, producer, the two issuers and the eight softmax warps as roles that make the
kernel's waits and arrivals in its order, copies that land in any order, products and their arrivals in order of issue but at any time, all of it under random
schedules.

A wait names a parity, and a parity tells two neighbouring phases apart, not three.  So every wait of the model also says which phase it
means, and the model holds that the barrier is in that phase or just behind it, that the parity is that phase's, that every role finds what the
others should have left (queries, key tiles, scores, P, zeros behind the last key, O), that every key tile reaches every lane's result once and in
order, and that nothing is under way when all roles have ended.  That the model notices is shown with mistakes planted in it."""
import random

import pytest

STAGES, SEGMENTS = 5, 6


class Barrier:
    def __init__(self, count):
        self.count = self.pending = count
        self.phase = self.bytes = 0                            # phases completed, copies expected and not there

    def arrive(self, copies=0):
        self.bytes += copies
        assert self.pending > 0, "more arrivals than the phase has"
        self.pending -= 1
        self.look()

    def landed(self):
        self.bytes -= 1
        self.look()

    def look(self):
        if self.pending == 0 and self.bytes == 0:
            self.phase += 1
            self.pending = self.count

    def done(self, phase, parity):
        """A look by parity at the barrier for the end of its `phase`-th phase (-1: the one before the first)."""
        assert parity == phase & 1, "not that phase's parity"
        assert phase <= self.phase <= phase + 1, "phase %d is looked for in phase %d" % (phase, self.phase)
        return (self.phase - 1) & 1 == parity


class Kernel:
    """segments: (single M tile, key tiles, does its last tile end ragged)."""

    def __init__(self, segments, seed, mistake=None):
        self.r, self.segments, self.mistake = random.Random(seed), segments, mistake
        bars = lambda n, count: [Barrier(count) for _ in range(n)]  # noqa: E731
        self.kv_full = [bars(STAGES, 1) for _ in range(3)]      # lane 0, lane 1, pairs
        if mistake == "one barrier a stage":
            self.kv_full = [self.kv_full[2]] * 3
        self.kv_empty = bars(STAGES, 2)
        self.seg_full, self.seg_empty = bars(SEGMENTS, 1), bars(SEGMENTS, 3 + 8)
        self.pair_full, self.pair_empty, self.single_full, self.single_empty = bars(2, 1), bars(2, 1), bars(2, 1), bars(2, 2)
        self.s_full, self.v_there, self.o_full, self.o_free = bars(2, 1), bars(2, 1), bars(2, 1), bars(2, 4)
        self.p_ready = [bars(2, 4), bars(2, 4)]
        self.seg, self.q, self.kv = [None] * SEGMENTS, [None, None], [None] * STAGES
        self.S, self.O = [[None] * 4, [None] * 4], [None, None]  # noqa: E741
        self.zeros = {}                                        # warps whose zeros are in the V tile of a stage, by lane
        self.results = {}
        self.copies, self.products, self.stores = [], [[], []], []

    # ------------------------------------------------------------------------------------------------ roles
    def planner(self):
        for k in range(len(self.segments) + 1):
            at, turn = k % SEGMENTS, k // SEGMENTS
            while not self.seg_empty[at].done(turn - 1, turn & 1 ^ 1):
                yield
            self.seg[at] = (k,) + (self.segments[k] if k < len(self.segments) else (False, 0, False))
            self.seg_full[at].arrive()

    def producer(self):
        pairs = singles = tile = load = 0
        asked, sg = set(), None
        pair_free = lambda b: self.pair_empty[b].done(pairs - 1, pairs & 1 ^ 1)  # noqa: E731
        single_free = lambda b: self.single_empty[b].done((singles + 1 - b >> 1) - 1, singles + 1 - b >> 1 & 1 ^ 1)  # noqa: E731

        def load_q(b):
            bar, what = (self.single_full if sg[1] else self.pair_full)[b], (sg[0], 0 if sg[1] else b)
            bar.arrive(copies=1)
            self.q[b] = "on its way"
            asked.discard(b)

            def land():
                self.q[b] = what
                bar.landed()
            self.copies.append(land)

        def free(stage_load):
            return self.kv_empty[stage_load % STAGES].done(stage_load // STAGES - 1, stage_load // STAGES & 1 ^ 1)

        for k in range(len(self.segments) + 1):
            for b in sorted(asked):
                while not pair_free(b):
                    yield
                while not single_free(b):
                    yield
                load_q(b)
            if sg:
                singles, pairs = singles + sg[1], pairs + (not sg[1])
            at = k % SEGMENTS
            while not self.seg_full[at].done(k // SEGMENTS, k // SEGMENTS & 1):
                yield
            sg = self.seg[at]
            self.seg_empty[at].arrive()
            if sg[2] == 0:
                break
            asked = {singles & 1} if sg[1] else {0, 1}
            for i in range(sg[2]):
                for kv in range(2):
                    while True:
                        for b in sorted(asked):
                            if pair_free(b) and single_free(b):
                                load_q(b)
                        yield
                        if free(load):
                            break
                    bar, stage, what = self.kv_full[tile + i & 1 if sg[1] else 2][load % STAGES], load % STAGES, (sg[0], i, kv)
                    bar.arrive(copies=1)
                    self.kv[stage], self.zeros[stage] = "on its way", [set(), set()]

                    def land(stage=stage, what=what, bar=bar):
                        self.kv[stage] = what
                        bar.landed()
                    self.copies.append(land)
                    load += 1
            tile += sg[2]
        if self.mistake != "nobody waits for the last arrivals":
            for i in range(STAGES):
                while not free(load + i):
                    yield
            for b in range(2):
                while not pair_free(b):
                    yield
                while not single_free(b):
                    yield

    def issuer(self, l):
        ops = segs = tile0 = pairs = singles = 0
        seen = {}                                              # phases followed, by barrier
        issue = self.products[l].append

        def stage_full(load, single):
            bar = self.kv_full[l if single else 2][load % STAGES]
            n = load // STAGES if self.mistake == "one barrier a stage" else seen.get(bar, 0)
            if not bar.done(n, n & 1):
                return False
            seen[bar] = n + 1
            return True

        for k in range(len(self.segments) + 1):
            at = k % SEGMENTS
            while not self.seg_full[at].done(k // SEGMENTS, k // SEGMENTS & 1):
                yield
            _, single, n, ragged = self.seg[at]
            self.seg_empty[at].arrive()
            if n == 0:
                return
            place, before = (singles & 1, singles >> 1) if single else (l, pairs)
            q_full, q_empty = (self.single_full, self.single_empty) if single else (self.pair_full, self.pair_empty)
            while not q_full[place].done(before, before & 1):
                yield
            step, end = 2 if single else 1, tile0 + n

            def release(load):
                issue(self.kv_empty[load % STAGES].arrive)
                if single:
                    self.kv_empty[load % STAGES].arrive()

            def scores(t, base=tile0, k=k, place=place, single=single):
                def product():
                    assert self.q[place] == (k, 0 if single else l) and self.kv[2 * t % STAGES] == (k, t - base, 0)
                    self.S[l] = [("S", k, t - base)] * 4
                issue(product)
                issue(self.s_full[l].arrive)

            t = tile0 + (tile0 & 1 ^ l if single else 0)
            any_ = t < end
            if any_:
                while not stage_full(2 * t, single):
                    yield
                scores(t)
                release(2 * t)
            if t + step >= end:
                if any_:
                    issue(q_empty[place].arrive)
                else:
                    q_empty[place].arrive()
            if any_ and segs > 0:
                while not self.o_free[l].done(segs - 1, segs - 1 & 1):
                    yield
            first = True
            while t < end:
                more = t + step < end
                while not stage_full(2 * t + 1, single):
                    yield
                self.v_there[l].arrive()
                if more and not single:
                    while not stage_full(2 * (t + step), single):
                        yield
                for h in range(2):
                    while not self.p_ready[l][h].done(ops, ops & 1):
                        yield

                    def product(h=h, t=t, first=first, base=tile0, k=k, last=ragged and t == end - 1):
                        stage = (2 * t + 1) % STAGES
                        assert self.kv[stage] == (k, t - base, 1)
                        assert all(s in (("P", k, t - base, h), ("P", k, t - base, 1)) for s in self.S[l])
                        assert not last or self.zeros[stage][l] == {0, 1, 2, 3}, "rows behind the last key in a product"
                        if h == 0:
                            self.O[l] = (k, [] if first else self.O[l][1])
                            assert self.O[l][0] == k
                            self.O[l][1].append(t - base)
                    issue(product)
                ops += 1
                if more:
                    if single:
                        while not stage_full(2 * (t + step), single):
                            yield
                    scores(t + step)
                else:
                    issue(self.o_full[l].arrive)
                release(2 * t + 1)
                if more:
                    release(2 * (t + step))
                    if t + 2 * step >= end:
                        issue(q_empty[place].arrive)
                t, first = t + step, False
            segs += any_
            singles, pairs, tile0 = singles + single, pairs + (not single), end

    def softmax(self, l, warp):
        ops = segs = tile0 = 0
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
                    write = lambda stage=stage: self.zeros[stage][l].add(warp)  # noqa: E731
                    if self.mistake == "an arrival ahead of the other lanes" and not has_rows:
                        self.stores.append(write)               # lane 0's own are there, the others' come when they come
                    else:
                        write()
                if has_rows:
                    for h in range(2):
                        self.S[l][warp] = ("P", k, t, h)
                        self.p_ready[l][h].arrive()
                        yield
                else:
                    self.S[l][warp] = ("P", k, t, 1)
                    self.p_ready[l][0].arrive()
                    self.p_ready[l][1].arrive()
                first, ops = False, ops + 1
            if not first:
                while not self.o_full[l].done(segs, segs & 1):
                    yield
                segs += 1
                assert self.O[l][0] == k
                self.results[k, turn, warp] = list(self.O[l][1])
                yield
                self.o_free[l].arrive()
            tile0 += n
            self.seg_empty[at].arrive()

    # ------------------------------------------------------------------------------------------------ a schedule
    def run(self):
        roles = [self.planner(), self.producer(), self.issuer(0), self.issuer(1)] + [self.softmax(l, w) for l in range(2) for w in range(4)]
        live, idle = list(roles), 0
        weight, newest = [self.r.choice([1, 1, 1, 5, 20]) for _ in range(16)], self.r.choice([0, 0, .9])
        while live:
            what = self.r.choices(range(16), weight)[0]
            if what < 12:
                if roles[what] in live:
                    try:
                        next(roles[what])
                    except StopIteration:
                        live.remove(roles[what])
            elif what == 12 and self.copies:
                self.copies.pop(-1 if self.r.random() < newest else self.r.randrange(len(self.copies)))()
            elif what == 13 and self.stores:
                self.stores.pop(self.r.randrange(len(self.stores)))()
            elif what > 13 and self.products[what - 14]:
                self.products[what - 14].pop(0)()
            idle += 1
            assert idle < 50000 * (10 + sum(n for _, n, _ in self.segments)), "nobody gets on"
        assert not self.copies and not any(self.products), "under way when all roles have ended"
        for k, (single, n, _) in enumerate(self.segments):
            for turn in range(2):
                want = list(range(turn, n, 2)) if single else list(range(n))
                for warp in range(4):
                    assert self.results.get((k, turn, warp), []) == want


def _segments(r):
    single, most, ragged = r.choice([0, .2, .5, .8, 1]), r.choice([1, 2, 3, 7]), r.choice([0, .5, 1])
    return [(r.random() < single, r.randint(1, most), r.random() < ragged) for _ in range(r.randint(1, 12))]


@pytest.mark.parametrize("block", range(4))
def test_every_schedule_runs_through(block):
    for seed in range(100 * block, 100 * block + 100):
        Kernel(_segments(random.Random(seed)), seed).run()


@pytest.mark.parametrize("mistake,told", [("one barrier a stage", "is looked for in phase"), ("nobody waits for the last arrivals", "under way"),
                                          ("an arrival ahead of the other lanes", "rows behind the last key")])
def test_the_model_notices(mistake, told):
    for seed in range(400):
        try:
            Kernel(_segments(random.Random(seed)), seed, mistake).run()
        except AssertionError as e:
            assert told in str(e), e
            return
    pytest.fail("not noticed")
