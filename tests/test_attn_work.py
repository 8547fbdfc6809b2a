"""Where divided row tiles of prompts keep their partial results
(csrc/attn_work.h), compiled for the host: no two row tiles share a place,
whatever order the sequences' rows come in, and those of sequences that share no
token fit the room reserved for them."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2606_02955_amd", "csrc")
SHIM = r"""
#include "attn_work.h"
using namespace fdllm;
extern "C" int rows(const int32_t* cu, int b, int T, int max_q) { int f; return packed_rows(cu, b, T, max_q, &f); }
extern "C" long long places(int B, int T, int R) { return pa_places(B, T, R); }
extern "C" int first_place(const int32_t* cu, int b, int T, int max_q, int R, int step) {
  int n = 0;
  for (int lane = 0; lane < step; ++lane) n += pa_tiles_before(cu, b, T, max_q, R, lane, step);
  return n;
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("attn_work")
    src, so = d / "shim.cpp", d / "shim.so"
    src.write_text(SHIM)
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-I", CSRC, str(src), "-o", str(so)], check=True)
    lib = ctypes.CDLL(str(so))
    lib.places.restype = ctypes.c_longlong
    return lib


def _places(lib, cu, T, max_q, R):
    """Every row tile's place, and the rows of the sequences that have some."""
    arr = (ctypes.c_int32 * len(cu))(*cu)
    out, taken = [], []
    for b in range(len(cu) - 1):
        n = lib.rows(arr, b, T, max_q)
        first = lib.first_place(arr, b, T, max_q, R, 64)
        out += [first + t for t in range(-(-n * R // 128))]
        taken += list(range(cu[b], cu[b] + n))
    return out, taken


CASES = [
    # counts, T, max_q, R
    ([0, 100], 100, 100, 4),
    ([64, 128, 0, 64], 128, 64, 4),                    # the second runs backwards, the third lies before the first
    ([64, 128, 0, 64], 128, 64, 1),
    ([96, 128, 64, 96, 32, 64, 0, 32], 128, 32, 5),
    ([0, 1, 2, 3, 4, 5], 5, 1, 1),                     # many within one tile's rows
    ([0, 200, 300, 301], 301, 150, 2),                 # the first is longer than max_q
    ([5, 5, 5, 70, 300, 71, 90], 128, 100, 3),         # a count past the tensor
]


@pytest.mark.parametrize("cu,T,max_q,R", CASES)
def test_places_differ(lib, cu, T, max_q, R):
    places, taken = _places(lib, cu, T, max_q, R)
    assert len(taken) == len(set(taken))
    assert len(places) == len(set(places))
    assert all(0 <= p < lib.places(len(cu) - 1, T, R) for p in places)


def test_places_differ_for_random_orders(lib):
    rng = np.random.default_rng(0)
    for _ in range(300):
        n = int(rng.integers(1, 40))
        T, R = int(rng.integers(1, 600)), int(rng.integers(1, 9))
        cu = rng.integers(-5, T + 6, n + 1).tolist()
        places, taken = _places(lib, cu, T, int(rng.integers(1, T + 1)), R)
        assert len(places) == len(set(places))
        if len(taken) == len(set(taken)):
            assert all(0 <= p < lib.places(n, T, R) for p in places)
