"""The work partition of the shared-prefix attention, compiled for the host from the kernels' own header and walked as the main kernel
walks it: every key tile of every item dealt exactly once and in order, every lane's partial result in a place of its own inside
the workspace, and the merge reading exactly those."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

from paper_2604_02047_b200 import build

SOURCE = r"""
#include <algorithm>
#include <map>
#include <vector>
using std::max; using std::min;
#include "shared_work.cuh"
using namespace goose;
// what a warp does on the GPU, a sequence after the other: the list's length, and a place in it
static void measure(SharedWork& wk) {
    long long sum = 0;
    int live = 0;
    for (int s = 0; s < wk.S; ++s) {
        const int T = wk.tiles(s);
        sum += T;
        live += T > 0;
    }
    wk.set(sum, live);
}
static void seek(SharedCursor& cu, const SharedWork& wk, long long w0) {
    cu.w = w0; cu.s = -1; cu.T = wk.shared_tiles;
    if (w0 < wk.shared_total) { cu.enter(wk, w0); return; }
    long long rem = w0 - wk.shared_total;
    for (cu.s = 0; cu.s < wk.S; ++cu.s) {
        cu.T = wk.tiles(cu.s);
        const long long mine = (long long)wk.Hkv * wk.own_pairs() * wk.width(cu.s, cu.T);
        if (rem < mine) break;
        rem -= mine;
    }
    if (cu.s < wk.S) cu.enter(wk, rem);
}
// 0, or what is wrong
extern "C" int walk(int S, int B, int Hkv, int shared_tiles, int shared_m, int own_m, int G, int kv_rows, const int32_t* ctx_len,
                    const int32_t* n_nodes, long long* longest) {
    SharedWork wk{};
    wk.ctx_len = ctx_len; wk.n_nodes = n_nodes; wk.S = S; wk.B = B; wk.Hkv = Hkv; wk.kv_rows = kv_rows;
    wk.shared_tiles = shared_tiles; wk.shared_m = shared_m; wk.own_m = own_m; wk.G = G;
    measure(wk);
    std::map<int, std::pair<int, int>> written;             // slot -> (item, tiles of it)
    std::vector<int> dealt(wk.items(), 0);
    for (int cta = 0; cta < G; ++cta) {
        const long long w0 = wk.start(cta), w_end = wk.start(cta + 1);
        if (w0 > w_end) return 1;
        if (w0 == w_end) continue;
        SharedCursor cu;
        seek(cu, wk, w0);
        long long mine = 0;
        while (cu.w < w_end) {
            if (cu.s >= S || cu.s < -1 || cu.i < 0) return 2;
            const int pairs = cu.s < 0 ? wk.shared_pairs() : wk.own_pairs(), n_m = cu.s < 0 ? shared_m : own_m;
            if (cu.i >= Hkv * pairs || cu.T != (cu.s < 0 ? shared_tiles : wk.tiles(cu.s))) return 3;
            const int item = wk.item(cu.s, cu.i), n = cu.run(wk, w_end);
            const bool single = 2 * (cu.i % pairs) + 1 >= n_m;
            if (item < 0 || item >= wk.items() || n < 1 || cu.t != dealt[item] || cu.t + n > cu.T) return 4;
            for (int l = 0; l < 2; ++l) {
                const int tiles = single ? (n + 1 - l) / 2 : n;
                if (tiles == 0) continue;
                const int slot = wk.slot(item, cta, cu.t == 0, cu.t + n == cu.T, l);
                if (slot < 0 || slot >= wk.slots() || written.count(slot)) return 5;
                written[slot] = {item, tiles};
            }
            dealt[item] += n; mine += n * wk.places(cu.s);
            cu.skip(wk, n);
        }
        *longest = max(*longest, mine);
    }
    size_t read = 0;
    long long first = 0;
    for (int s = -1; s < S; ++s) {
        const int pairs = s < 0 ? wk.shared_pairs() : wk.own_pairs(), n_m = s < 0 ? shared_m : own_m;
        const int T = s < 0 ? shared_tiles : wk.tiles(s);
        for (int i = 0; i < Hkv * pairs; ++i) {
            if (T == 0) continue;
            if (dealt[wk.item(s, i)] != T) return 6;
            for (int m = 2 * (i % pairs); m < min(n_m, 2 * (i % pairs) + 2); ++m) {
                SharedParts ps;
                ps.set(wk, s, i, first + (long long)i * wk.width(s, T), T, (m | 1) >= n_m, m & 1);
                int tiles = 0;
                for (int k = 0; k < ps.n; ++k) {
                    const int slot = ps.slot(wk, k);
                    if (slot < 0) continue;
                    if (!written.count(slot) || written[slot].first != wk.item(s, i)) return 7;
                    tiles += written[slot].second; ++read;
                }
                if (tiles != T) return 8;
            }
        }
        first += (long long)Hkv * pairs * wk.width(s, T);
    }
    if (first != wk.total) return 9;
    return read == written.size() ? 0 : 10;
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("shared_work")
    src, so = d / "walk.cu", d / "walk.so"
    src.write_text(SOURCE)
    r = subprocess.run([build._nvcc(), "-std=c++17", "-O1", "-shared", "-Xcompiler", "-fPIC", "-I", build.INCLUDE, "-I", build.CSRC, str(src), "-o", str(so)],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    return ctypes.CDLL(str(so))


def _walk(lib, S, B, Hkv, shared_len, shared_m, own_m, G, ctxs, nodes=None, kv_rows=2 ** 31 - 1):
    ctx = np.asarray(ctxs, np.int32)
    nn = None if nodes is None else np.asarray(nodes, np.int32)
    longest = ctypes.c_longlong(0)
    p = lambda a: None if a is None else a.ctypes.data_as(ctypes.c_void_p)  # noqa: E731
    rc = lib.walk(S, B, Hkv, (shared_len + 127) // 128, shared_m, own_m, G, kv_rows, p(ctx), p(nn), ctypes.byref(longest))
    assert rc == 0, (rc, S, B, Hkv, shared_len, shared_m, own_m, G, ctxs, nodes)
    return longest.value


def test_random_lists(lib):
    rng = np.random.default_rng(0)
    for _ in range(3000):
        S, B, g = int(rng.integers(1, 40)), int(rng.integers(1, 129)), int(rng.integers(1, 17))
        shared_nb, own_nb = min(128 // g, S * B), min(B, 128 // g)
        shared_m, own_m = -(-S * B // shared_nb), -(-B // own_nb)
        top = int(2 ** rng.uniform(0, 15))
        _walk(lib, S, B, int(rng.integers(1, 9)), int(rng.choice([0, 1, 128, 129, int(2 ** rng.uniform(0, 17))])), shared_m, own_m,
              int(rng.choice([148, 132, 7, 1])), rng.integers(0, top, S), rng.integers(-1, B + 2, S) if rng.random() < .5 else None)


def test_shares_are_even(lib):
    """No CTA has more than an equal share of the places, up to one tile."""
    tiles = 8 * 16 * 64 + 16 * 8 * 17                       # 16 pairs a head over 8192 rows; 16 sequences of 2048 + 64 rows, a pair a head
    assert _walk(lib, 16, 64, 8, 8192, 32, 2, 148, [2048] * 16) <= (5 * tiles + 16 * (8 * 16 + 16 * 8)) // 148 + 5


def test_lengths_that_no_kernel_should_meet(lib):
    big = 2 ** 31 - 1
    for ctxs in ([big] * 30, [-1] * 30, [-2 ** 31] * 15 + [big] * 15):
        for kv_rows in (big, 1000):
            _walk(lib, 30, 64, 4, min(kv_rows, 10 ** 8), 15, 1, 148, ctxs, kv_rows=kv_rows)
    _walk(lib, 3, 64, 4, 0, 2, 1, 148, [5, 5, 5], [0, 0, 0])      # nothing at all
