"""The barriers of kv_weights_kernel as a model: planner, the queries' warp, four warps of copies, the log-sum-exps' warp, the issuer and the warps of the
sums as roles that make the kernel's waits and arrivals in its order, copies that land in any order, products and their arrivals in order of issue but at any
time, all of it under random schedules.  Held: every wait finds its barrier in the phase that it means or just behind it; every product has its
key tile, its queries and its last step as they belong together; every key tile's sums get every Q tile once and in order; nothing is under way when all
roles have ended.  That the model notices is shown with mistakes planted in it."""
import random

import pytest

from test_shared_barriers_host import Barrier

RUN, STAGES, Q_STAGES, SEGMENTS, COPIES = 4, 4, 2, 6, 4


class Kernel:
    """segments: (Q tiles, key tiles)."""

    def __init__(self, segments, seed, mistake=None):
        self.r, self.segments, self.mistake = random.Random(seed), segments, mistake
        bars = lambda n, count: [Barrier(count) for _ in range(n)]  # noqa: E731
        self.k_full, self.k_empty = bars(STAGES, COPIES), bars(STAGES, 1)
        self.q_full, self.q_empty = bars(Q_STAGES, 1), bars(Q_STAGES, 1)
        self.lse_full, self.lse_empty = bars(Q_STAGES, 1), bars(Q_STAGES, 4 * RUN)
        self.seg_full, self.seg_empty = bars(SEGMENTS, 1), bars(SEGMENTS, 3 + 4 * RUN + COPIES)
        self.s_full, self.s_free = bars(RUN, 1), bars(RUN, 4)
        self.seg, self.k, self.q, self.step = [None] * SEGMENTS, [None] * STAGES, [None] * Q_STAGES, [None] * Q_STAGES
        self.S, self.sums = [None] * RUN, {}
        self.copies, self.products = [], []

    def segment(self, k):
        at = k % SEGMENTS
        while not self.seg_full[at].done(k // SEGMENTS, k // SEGMENTS & 1):
            yield
        return self.seg[at]

    def planner(self):
        for k in range(len(self.segments) + 1):
            at, turn = k % SEGMENTS, k // SEGMENTS
            while not self.seg_empty[at].done(turn - 1, turn & 1 ^ 1):
                yield
            self.seg[at] = self.segments[k] if k < len(self.segments) else (0, 0)
            self.seg_full[at].arrive()

    def queries(self):
        load = 0
        free = lambda i: self.q_empty[i % Q_STAGES].done(i // Q_STAGES - 1, i // Q_STAGES & 1 ^ 1)  # noqa: E731
        for k in range(len(self.segments) + 1):
            n, _ = yield from self.segment(k)
            self.seg_empty[k % SEGMENTS].arrive()
            for i in range(n):
                while not free(load):
                    yield
                bar, at = self.q_full[load % Q_STAGES], load % Q_STAGES
                bar.arrive(copies=1)
                self.q[at] = "on its way"

                def land(at=at, bar=bar, what=(k, i)):
                    self.q[at] = what
                    bar.landed()
                self.copies.append(land)
                load += 1
        if self.mistake != "nobody waits for the last arrivals":
            for i in range(Q_STAGES):
                while not free(load + i):
                    yield

    def keys(self, part):
        load = 0
        free = lambda i: self.k_empty[i % STAGES].done(i // STAGES - 1, i // STAGES & 1 ^ 1)  # noqa: E731
        for k in range(len(self.segments) + 1):
            _, run = yield from self.segment(k)
            self.seg_empty[k % SEGMENTS].arrive()
            for u in range(run):
                while not free(load):
                    yield
                at, bar = load % STAGES, self.k_full[load % STAGES]
                if self.k[at] is None or self.k[at][0] != (k, u):
                    self.k[at] = ((k, u), set())

                def land(at=at, bar=bar, what=(k, u)):         # the arrival comes with the copies
                    assert self.k[at][0] == what
                    self.k[at][1].add(part)
                    bar.arrive()
                self.copies.append(land)
                load += 1
        if self.mistake != "nobody waits for the last arrivals":
            for i in range(STAGES):
                while not free(load + i):
                    yield

    def steps(self):
        i = 0
        for k in range(len(self.segments) + 1):
            n, _ = yield from self.segment(k)
            self.seg_empty[k % SEGMENTS].arrive()
            for t in range(n):
                at = i % Q_STAGES
                while not self.lse_empty[at].done(i // Q_STAGES - 1, i // Q_STAGES & 1 ^ 1):
                    yield
                self.step[at] = (k, t)
                yield
                self.lse_full[at].arrive()
                i += 1

    def issuer(self):
        q = tile = 0
        used = [0] * RUN
        issue = self.products.append
        for k in range(len(self.segments) + 1):
            n, run = yield from self.segment(k)
            self.seg_empty[k % SEGMENTS].arrive()
            for t in range(n):
                at = q % Q_STAGES
                while not self.q_full[at].done(q // Q_STAGES, q // Q_STAGES & 1):
                    yield
                while self.mistake != "a product ahead of its last step" and not self.lse_full[at].done(q // Q_STAGES, q // Q_STAGES & 1):
                    yield
                for u in range(run):
                    load = tile + u
                    if t == 0:
                        while not self.k_full[load % STAGES].done(load // STAGES, load // STAGES & 1):
                            yield
                    while not self.s_free[u].done(used[u] - 1, used[u] & 1 ^ 1):
                        yield
                    used[u] += 1

                    def product(at=at, u=u, stage=load % STAGES, k=k, t=t):
                        assert self.q[at] == (k, t) and self.step[at] == (k, t), "not the Q tile's last step"
                        assert self.k[stage] == ((k, u), set(range(COPIES)))
                        self.S[u] = (k, t)
                    issue(product)
                    issue(self.s_full[u].arrive)
                    if t == n - 1:
                        issue(self.k_empty[load % STAGES].arrive)
                issue(self.q_empty[at].arrive)
                q += 1
            tile += run

    def sum(self, u, warp):
        q = used = 0
        for k in range(len(self.segments) + 1):
            n, run = yield from self.segment(k)
            if n == 0:
                return
            for t in range(n):
                at = q % Q_STAGES
                while (u < run or self.mistake != "idle warps do not wait") and not self.lse_full[at].done(q // Q_STAGES, q // Q_STAGES & 1):
                    yield
                if u < run:
                    while not self.s_full[u].done(used, used & 1):
                        yield
                    used += 1
                    assert self.S[u] == (k, t)
                    yield
                    assert self.S[u] == (k, t)
                    self.sums.setdefault((k, u, warp), []).append(t)
                    self.s_free[u].arrive()
                    yield
                    assert self.step[at] == (k, t)             # (which of its rows count)
                self.lse_empty[at].arrive()
                q += 1
            self.seg_empty[k % SEGMENTS].arrive()

    def run(self):
        roles = [self.planner(), self.queries(), self.steps(), self.issuer()] + [self.keys(p) for p in range(COPIES)] + \
            [self.sum(u, w) for u in range(RUN) for w in range(4)]
        live, idle = set(range(len(roles))), 0
        weight = [self.r.choice([1, 1, 1, 5, 20]) for _ in range(len(roles) + 2)]
        while live:
            what = self.r.choices(range(len(roles) + 2), weight)[0]
            if what in live:
                try:
                    next(roles[what])
                except StopIteration:
                    live.discard(what)
            elif what == len(roles) and self.copies:
                self.copies.pop(self.r.randrange(len(self.copies)))()
            elif what == len(roles) + 1 and self.products:
                self.products.pop(0)()
            idle += 1
            assert idle < 60000 * (10 + sum(n * run for n, run in self.segments)), "nobody gets on"
        assert not self.copies and not self.products, "under way when all roles have ended"
        for k, (n, run) in enumerate(self.segments):
            for u in range(RUN):
                for w in range(4):
                    assert self.sums.get((k, u, w), []) == (list(range(n)) if u < run else [])


def _segments(r):
    most, runs = r.choice([1, 2, 5]), r.choice([[1], [1, 2], [1, 2, 3, 4], [4]])
    return [(r.randint(1, most), r.choice(runs)) for _ in range(r.randint(1, 10))]


@pytest.mark.parametrize("block", range(4))
def test_every_schedule_runs_through(block):
    for seed in range(60 * block, 60 * block + 60):
        Kernel(_segments(random.Random(seed)), seed).run()


@pytest.mark.parametrize("mistake,told", [("a product ahead of its last step", "not the Q tile's last step"), ("idle warps do not wait", None),
                                          ("nobody waits for the last arrivals", "under way")])
def test_the_model_notices(mistake, told):
    for seed in range(400):
        try:
            Kernel(_segments(random.Random(seed)), seed, mistake).run()
        except AssertionError as e:
            assert told is None or told in str(e), e
            return
    pytest.fail("not noticed")
