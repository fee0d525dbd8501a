"""csrc/packed_rules.hpp, compiled for the host: which rows and keys a call over packed rows or a paged cache works on."""
import ctypes as C
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2412_03409_amd", "csrc")
SHIM = """
#define __device__
#define __host__
#define __forceinline__ inline
#include "packed_rules.hpp"
extern "C" int new_rows(int first, int last, int T) { return pkv::new_rows(first, last, T); }
extern "C" int keys_seen(int rows, int n, int len) { return pkv::keys_seen(rows, n, len); }
"""


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    d = tmp_path_factory.mktemp("packed_rules")
    (d / "shim.cpp").write_text(SHIM)
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-I", CSRC, str(d / "shim.cpp"), "-o", str(d / "shim.so")])
    return C.CDLL(str(d / "shim.so"))


def test_rows_of_a_sequence(rules):
    T = 5
    for first in range(-3, 9):
        for last in range(-3, 9):
            n = rules.new_rows(first, last, T)
            if 0 <= first <= last <= T:
                assert n == last - first
            else:       # every row that is worked on lies in the call's
                assert n == 0
    assert rules.new_rows(-(1 << 31), (1 << 31) - 1, T) == 0


def test_keys_of_a_segment(rules):
    """The most keys that one of the rows sees: a sequence that waits sees none of its cache, and has no work."""
    for n in range(0, 8):
        for rows in range(0, n + 1):
            for length in range(0, 12):
                seen = [max(0, min(length, length - n + i + 1)) for i in range(rows)]
                assert rules.keys_seen(rows, n, length) == max(seen, default=0), (rows, n, length)
    assert rules.keys_seen(0, 0, 1 << 20) == 0
