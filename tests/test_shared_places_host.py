"""Where the partial results of the shared-prefix attention lie, compiled for the host from the kernels' own header: every slot has the rows
that its kind of M tile can have, every word of every row a place of its own, and the workspace is what goose.h says."""
import ctypes
import subprocess

import numpy as np
import pytest

from paper_2604_02047_b200 import build

SOURCE = r"""
#include <algorithm>
using std::max; using std::min;
#include "shared_work.cuh"
using namespace goose;
extern "C" long long lay(int S, int Hkv, int shared_tiles, int shared_m, int own_m, int G, int of_batch, int of_sequence, uint32_t* places, int n) {
    SharedWork wk{};
    wk.S = S; wk.Hkv = Hkv; wk.shared_tiles = shared_tiles; wk.shared_m = shared_m; wk.own_m = own_m; wk.G = G;
    const long long blocks = wk.lay(of_batch, of_sequence);
    if (n != wk.slots()) return -1;
    for (int i = 0; i < n; ++i) places[i] = wk.place(i);
    return blocks;
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("shared_places")
    src, so = d / "lay.cu", d / "lay.so"
    src.write_text(SOURCE)
    r = subprocess.run([build._nvcc(), "-std=c++17", "-O1", "-shared", "-Xcompiler", "-fPIC", "-I", build.INCLUDE, "-I", build.CSRC, str(src), "-o", str(so)],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    out = ctypes.CDLL(str(so))
    out.lay.restype = ctypes.c_longlong
    return out


def test_places(lib):
    rng = np.random.default_rng(0)
    for _ in range(300):
        S, Hkv, B, g = int(2 ** rng.uniform(0, 6)), int(rng.integers(1, 21)), int(rng.choice([1, 2, 60, 128, int(rng.integers(1, 129))])), int(rng.integers(1, 17))
        G, tiles, t = int(rng.choice([148, 132, 1])), int(rng.choice([0, 1, 77])), 128 // g
        pairs, up4 = (lambda n: -(-(-(-n // t)) // 2)), (lambda r: -(-r // 4) * 4)
        n_shared, n_own = (2 * Hkv * pairs(S * B) if tiles else 0), 2 * S * Hkv * pairs(B)
        n = n_shared + n_own + 4 * G
        place = np.zeros(n, np.uint32)
        blocks = lib.lay(S, Hkv, tiles, -(-S * B // min(t, S * B)), -(-B // min(t, B)), G, min(t, S * B) * g, min(t, B) * g,
                         place.ctypes.data_as(ctypes.c_void_p), n)
        rows = np.full(n, min(t, S * B if tiles else B) * g)     # what the M tiles of a slot can have
        rows[n_shared:n_shared + n_own] = min(t, B) * g
        # words of row r of a slot: place + r + 128 j, j < 25; the rows stay inside a block of 25 x 128 words, on sectors of 32 bytes
        block, first = (place // 3200).astype(int), (place % 3200).astype(int)
        assert (first + rows <= 128).all() and (first % 2 == 0).all()
        order = np.lexsort((first, block))
        b, f, r = block[order], first[order], rows[order]
        assert ((b[1:] > b[:-1]) | (f[:-1] + r[:-1] <= f[1:])).all()
        # goose.h's formula
        k = lambda m: max(2 ** e for e in range(6) if 2 ** e * min(m, t) * g <= 128)  # noqa: E731
        up = lambda m, d: -(-m // d)  # noqa: E731
        assert blocks == up(n_shared, k(S * B)) + up(n_own, k(B)) + up(4 * G, k(S * B) if tiles else k(B)) and block.max() < blocks
