"""The calls on a cache in pages with heads, lengths, pages and counts drawn at random, each against its definition with the tolerances of its own tests.  The draws
come from their seed alone; ``python tests/test_gpu_paged_random.py FIRST LAST`` goes through those of more seeds."""
import os
import random
import sys

sys.path[:0] = [os.path.dirname(os.path.abspath(__file__)), os.path.dirname(os.path.dirname(os.path.abspath(__file__)))]

import pytest  # noqa: E402

from test_gpu_append_pages import _run as append  # noqa: E402
from test_gpu_chunk_attn import Case as Chunk  # noqa: E402
from test_gpu_evict_kv import Case as Evict  # noqa: E402
from test_gpu_kv_weights import Case as Weights  # noqa: E402

pytestmark = pytest.mark.gpu
CALLS = 25                                                     # of a seed


def _goose():
    from paper_2604_02047_b200 import binding, build
    build.build()
    return binding.Goose(max_S=70, max_B=16, max_H=64)


@pytest.fixture(scope="module")
def goose():
    g = _goose()
    yield g
    g.close()


def _log(r, a, b):
    return int(round(a * (b / a) ** r.random()))


def _one(goose, r):
    """Draws a call, makes it and looks at what came of it; returns its kind."""
    H, Hkv = r.choice([(1, 1), (5, 5), (8, 2), (32, 8), (40, 40), (16, 1), (14, 2), (16, 2), (52, 52), (64, 4), (3, 1)])
    S, page = _log(r, 1, 70), r.choice([16, 16, 32, 64, 128, 256, 1024])
    B = r.choice([1, 1, 1, 2, 8, 17, 60, 128, 129, _log(r, 2, 300), _log(r, 100, 2000)])
    hi = _log(r, 1, 9000)
    while S * (hi + B) * Hkv > 1e6 or S * B * H > 1e5 or S * B * H * (hi + B) > 2e8:
        if S > 1:
            S = S * 3 // 4
        elif B > 1 and S * B * H > 1e5:
            B = B * 3 // 4
        else:
            hi, B = hi * 3 // 4, max(1, B * 9 // 10)
    lo = r.choice([0, hi])
    ctxs = [r.randint(lo, hi) for _ in range(S)]
    new = None if r.random() < 0.5 else [r.choice([0, 1, B, r.randint(0, B)]) for _ in range(S)]
    seed, kind = r.randrange(10 ** 6), r.choices(["chunk", "weights", "evict", "append"], [4, 3, 1, 2])[0]
    if kind == "chunk":
        Chunk(H, Hkv, B, ctxs, page, new=new, seed=seed).check(goose)
    elif kind == "weights":
        Weights(H, Hkv, B, ctxs, page, new=new, seed=seed).check(goose)
    elif kind == "append":
        S = min(S, 40)
        append(goose, H, Hkv, B, ctxs[:S], page, new=None if new is None else new[:S], norm=r.random() < 0.6, rot=r.choice([0, 16, 64, 128, 128]),
               interleaved=r.random() < 0.4, pos_off=r.choice([None, [r.randint(0, 5000) for _ in range(S)]]), seed=seed, in_place=r.random() < 0.3,
               arrays=r.choice(["wp", "wp", "w", "p", ""]))
    else:
        while sum(ctxs) * Hkv > 1e5:                           # (the definition is worked out row by row)
            ctxs = [x * 3 // 4 for x in ctxs]
        budget = max(1, int(max(ctxs + [1]) * r.uniform(0.1, 1)))
        sink = r.randint(0, min(16, budget))
        Evict(Hkv, ctxs, page, budget, sink, r.randint(0, budget - sink), off=[r.randint(0, 99) for _ in ctxs], seed=seed).check(goose)
    return kind


@pytest.mark.parametrize("seed", range(12))
def test_random_calls(goose, seed):
    r = random.Random(seed)
    for i in range(CALLS):
        state = r.getstate()
        try:
            _one(goose, r)
        except BaseException:
            print("seed %d, call %d" % (seed, i), state[1][-1])
            raise


if __name__ == "__main__":
    context, count = _goose(), {}
    for at in range(int(sys.argv[1]), int(sys.argv[2])):
        draws = random.Random(at)
        for _ in range(CALLS):
            k = _one(context, draws)
            count[k] = count.get(k, 0) + 1
    print("held:", count)
