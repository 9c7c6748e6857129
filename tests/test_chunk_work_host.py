"""The work partition of the attention over pages, compiled for the host from the kernel's own header and walked as the kernel's planner walks it:
every key tile of every item dealt once and in order, items that are cut named alike by all CTAs that have tiles of them, at most one segment of a CTA
that does not begin its item and one that does not end it, ranges of about equal cost."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

from paper_2604_02047_b200 import build

SOURCE = r"""
#include <algorithm>
#include <map>
#include <tuple>
#include <vector>
#include "chunk_work.cuh"
using namespace goose;
// 0, or what is wrong
template <typename Int>
static int walk_as(int S, int B, int Hkv, int t, int G, int room, const int32_t* ctx_len, const int32_t* n_new, double* worst) {
    ChunkWork<Int> wk{};
    wk.ctx_len = ctx_len; wk.n_new = n_new; wk.S = S; wk.B = B; wk.Hkv = Hkv; wk.G = G; wk.t = t; wk.room = room;
    Int sum = 0;
    bool several = false;
    for (int s = 0; s < S; ++s) {
        const ChunkSeq<Int> q = wk.seq(s);
        sum += q.before(q.pairs);
        several |= q.n > t;
    }
    wk.set(sum, several);
    std::map<std::tuple<int, int, int>, std::pair<int, int>> dealt;      // item -> (tiles so far, CTAs so far)
    long long longest = 0, all = 0;
    for (int c = 0; c < G; ++c) {
        const Int from = wk.start(c), to = wk.start(c + 1);
        if (from >= to) continue;
        ChunkCursor<Int> cu{};
        Int begin = 0; long long mine = 0;
        ChunkSeq<Int> q{};
        for (cu.s = 0; cu.s < S; ++cu.s) {
            q = wk.seq(cu.s);
            const Int all = Hkv * q.before(q.pairs);
            if (from < begin + all) break;
            begin += all;
        }
        if (cu.s == S) return 1;
        cu.enter(q, begin, from);
        if (cu.hk < 0 || cu.hk >= Hkv || cu.p < 0 || cu.p >= q.pairs || cu.w0 > from || cu.w0 + q.width(cu.p) <= from) return 2;
        int heads = 0, tails = 0;
        while (cu.w0 < to) {
            cu.look(wk, q, c, from, to);
            if (cu.T < 1 || cu.T != (q.keys(cu.p) + 127) / 128) return 3;
            if (cu.t1 > cu.t0) {
                auto& d = dealt[{cu.s, cu.hk, cu.p}];
                if (d.first != cu.t0) return 4;
                if (c != cu.c0 + d.second || c > cu.c1) return 5;
                d.first = cu.t1; d.second++;
                mine += cu.t1 - cu.t0;
                const bool starts = cu.t0 == 0, ends = cu.t1 == cu.T;
                if (starts != (c == cu.c0) || ends != (c == cu.c1)) return 6;
                heads += !starts; tails += starts && !ends;
            }
            if (!cu.next(wk, q)) {
                do { ++cu.s; q = cu.s < S ? wk.seq(cu.s) : ChunkSeq<Int>{}; } while (cu.s < S && q.pairs == 0);
                if (cu.s == S) break;
                cu.hk = cu.p = 0;
            }
        }
        if (heads > 1 || tails > 1) return 7;
        longest = std::max(longest, mine); all += mine;
    }
    for (int s = 0; s < S; ++s) {
        const ChunkSeq<Int> q = wk.seq(s);
        const int n = n_new ? (n_new[s] < 0 || n_new[s] > B ? 0 : n_new[s]) : B;
        if (q.n != n || q.pairs != (n + 2 * t - 1) / (2 * t)) return 8;
        long long rows = 0;
        for (int p = 0; p < q.pairs; ++p) {
            rows += std::min(n - p * q.step, q.step);
            for (int h = 0; h < Hkv; ++h) {
                auto it = dealt.find({s, h, p});
                if (it == dealt.end() || it->second.first != q.tiles(p)) return 9;
            }
        }
        if (rows != n) return 10;
    }
    *worst = all ? (double)longest * G / all : 0;
    return (double)wk.total <= ChunkWork<Int>::most(S, B, Hkv, t, room) ? 0 : 11;
}
extern "C" int walk(int S, int B, int Hkv, int t, int G, int room, const int32_t* ctx_len, const int32_t* n_new, double* worst) {
    const int rc = walk_as<long long>(S, B, Hkv, t, G, room, ctx_len, n_new, worst);
    if (rc) return rc;
    return ChunkWork<int>::most(S, B, Hkv, t, room) < kShortPlaces ? 100 * walk_as<int>(S, B, Hkv, t, G, room, ctx_len, n_new, worst) : 0;
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    at = tmp_path_factory.mktemp("chunk_work")
    (at / "walk.cu").write_text(SOURCE)
    out = at / "walk.so"
    subprocess.run([build._nvcc(), "-std=c++17", "-O1", "-Xcompiler", "-fPIC", "-shared", "-I", build.INCLUDE, "-I", build.CSRC, str(at / "walk.cu"), "-o", str(out)],
                   check=True, capture_output=True)
    return ctypes.CDLL(str(out))


def _walk(lib, B, Hkv, t, ctxs, new=None, G=148, room=2 ** 20):
    p = lambda a: None if a is None else np.ascontiguousarray(a, np.int32).ctypes.data_as(ctypes.c_void_p)  # noqa: E731
    ctx, cnt = np.ascontiguousarray(ctxs, np.int32), None if new is None else np.ascontiguousarray(new, np.int32)
    worst = ctypes.c_double()
    rc = lib.walk(len(ctxs), B, Hkv, t, G, room, p(ctx), p(cnt), ctypes.byref(worst))
    assert rc == 0, (rc, B, Hkv, t, ctxs, new, G)
    return worst.value


@pytest.mark.parametrize("seed", range(300))
def test_random_lists(lib, seed):
    r = np.random.default_rng(seed)
    S, Hkv, g = int(r.integers(1, 70)), int(r.choice([1, 2, 8, 40])), int(r.integers(1, 17))
    B = int(r.choice([1, 2, 17, 128, 129, 700, 5000]))
    ctxs = r.integers(-3, int(r.choice([2, 200, 5000, 60000])), S)
    new = None if r.random() < .4 else r.integers(-1, B + 2, S)
    _walk(lib, B, Hkv, 128 // g, ctxs, new, G=int(r.choice([1, 2, 132, 148, 256])), room=int(r.choice([100, 30000, 2 ** 20])))


def test_extremes(lib):
    big = 2 ** 20
    _walk(lib, big, 64, 8, [0], room=big)
    _walk(lib, big, 64, 8, [0, big, 5, big - 1, -2 ** 31, 2 ** 31 - 1], [big, 0, 1, 1, 7, 7], room=big)
    _walk(lib, 2 ** 31 - 1, 1, 128, [0], [big], room=big)
    _walk(lib, 1, 64, 128, [big - 1] * 70)
    _walk(lib, 1, 1, 32, [0])
    _walk(lib, 5, 2, 32, [3, 4], [0, 0])


@pytest.mark.parametrize("B,Hkv,t,ctxs,most", [(4096, 8, 32, [8192], 1.06), (1, 8, 32, list(range(500, 8192, 120)), 1.05), (1, 8, 32, [16384], 1.3)])
def test_ranges_are_alike(lib, B, Hkv, t, ctxs, most):
    """Tiles of the longest range over the mean."""
    assert _walk(lib, B, Hkv, t, ctxs) <= most
