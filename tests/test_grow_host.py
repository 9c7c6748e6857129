"""How a context's workspaces grow (grow() of csrc/goose_internal.cuh, compiled for the host with an allocator of the test's): twice the old size where
the device has it, what the call needs where it has that much, an error and nothing changed where it has not."""
import ctypes
import subprocess

import pytest

from paper_2604_02047_b200 import build

SOURCE = r"""
#include <cuda_runtime.h>
static size_t room;                                      // bytes that the device still has
static int calls;
static cudaError_t failure;                              // of an allocation that does not fit
static cudaError_t take(void** p, size_t n) {
    ++calls;
    if (n > room) return failure;
    room -= n;
    *p = (void*)(0x1000 + room);
    return cudaSuccess;
}
#define cudaMalloc(p, n) take((void**)(p), n)
#define cudaGetLastError() ((void)0)
#include "goose_internal.cuh"
extern "C" int run(size_t has, size_t need1, size_t need2, int error, size_t* bytes, int* kept, int* asked, size_t* left) {
    goose_ctx c{};
    room = has; calls = 0; failure = (cudaError_t)error;
    int rc = goose::grow(&c, &c.shared_parts, &c.shared_bytes, need1);
    void* first = c.shared_parts;
    if (rc == 0 && need2) {
        calls = 0;
        rc = goose::grow(&c, &c.shared_parts, &c.shared_bytes, need2);
        if ((rc != 0) != (c.shared_parts == first) && need2 > need1) return -1;
        if (c.n_outgrown == 1 && c.outgrown[0] != first) return -2;
    }
    *bytes = c.shared_bytes; *kept = c.n_outgrown; *asked = calls; *left = room;
    return rc;
}
"""
OUT_OF_MEMORY, CAPTURING = 2, 900                        # cudaErrorMemoryAllocation, cudaErrorStreamCaptureUnsupported


@pytest.fixture(scope="module")
def grow(tmp_path_factory):
    d = tmp_path_factory.mktemp("grow")
    src, so = d / "grow.cu", d / "grow.so"
    src.write_text(SOURCE)
    r = subprocess.run([build._nvcc(), "-std=c++17", "-O1", "-shared", "-Xcompiler", "-fPIC", "-I", build.INCLUDE, "-I", build.CSRC, str(src), "-o", str(so)],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    lib = ctypes.CDLL(str(so))

    def run(has, need1, need2=0, error=OUT_OF_MEMORY):
        out = [ctypes.c_size_t(0), ctypes.c_int(0), ctypes.c_int(0), ctypes.c_size_t(0)]
        rc = lib.run(ctypes.c_size_t(has), ctypes.c_size_t(need1), ctypes.c_size_t(need2), error, *[ctypes.byref(x) for x in out])
        return (rc,) + tuple(x.value for x in out[:3])
    return run


def test_first_call_takes_what_it_needs(grow):
    assert grow(1000, 300) == (0, 300, 0, 1)
    assert grow(299, 300) == (OUT_OF_MEMORY, 0, 0, 1)


def test_twice_the_old_size_where_there_is_room(grow):
    assert grow(1000, 300, 301) == (0, 600, 1, 1)
    assert grow(10000, 300, 900) == (0, 900, 1, 1)
    assert grow(1000, 300, 300) == (0, 300, 0, 0)


def test_what_is_needed_where_twice_the_old_size_does_not_fit(grow):
    assert grow(700, 300, 301) == (0, 301, 1, 2)
    assert grow(700, 300, 400) == (0, 400, 1, 2)


def test_nothing_changes_where_it_does_not_fit(grow):
    assert grow(700, 300, 401) == (OUT_OF_MEMORY, 300, 0, 2)
    assert grow(700, 300, 700) == (OUT_OF_MEMORY, 300, 0, 1)   # (more than twice: nothing smaller to ask for)
    assert grow(700, 300, 301, error=CAPTURING) == (CAPTURING, 300, 0, 1)
