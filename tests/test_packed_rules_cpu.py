"""csrc/packed_rules.hpp, compiled for the host: which rows and keys a call over packed rows or a paged cache works on; what the
ring of free pages gives and takes; how many workgroups a compaction has."""
import ctypes as C
import os
import subprocess

import pytest

import paper_2412_03409_amd as P
from paper_2412_03409_amd import binding as Bd

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2412_03409_amd", "csrc")
SHIM = """
#define __device__
#define __host__
#define __forceinline__ inline
#include "packed_rules.hpp"
extern "C" int new_rows(int first, int last, int T) { return pkv::new_rows(first, last, T); }
extern "C" int keys_seen(int rows, int n, int len) { return pkv::keys_seen(rows, n, len); }
extern "C" int ring_range(int head, int count, int given, int P) { return pkv::ring_range(head, count, given, P); }
extern "C" int ring_place(unsigned at, int P) { return pkv::ring_place(at, P); }
extern "C" int gather_chunks(int N) { return pkv::gather_chunks(N); }
extern "C" int gather_fits(int N, int Hkv, long long segments) { return pkv::gather_fits(N, Hkv, segments); }
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


def test_ring_of_free_pages(rules):
    """Every place that an accepted call touches is in the ring, and none is both read and written, whatever the ends are."""
    for P in range(1, 8):
        for head in range(-1, P + 2):
            for count in range(-1, P + 2):
                for given in range(0, P + 3):
                    wrong = rules.ring_range(head, count, given, P)
                    assert wrong == (not (0 <= head < P and 0 <= count <= P and count + given <= P)), (P, head, count, given)
                    for taken in range(0, 0 if wrong else count + 1):
                        places = [rules.ring_place(head + i, P) for i in range(taken)]
                        places += [rules.ring_place(head + count + i, P) for i in range(given)]
                        assert len(set(places)) == taken + given and all(0 <= x < P for x in places)
                        assert places == [(head + i) % P for i in range(taken)] + [(head + count + i) % P for i in range(given)]
    top = (1 << 31) - 1
    assert not rules.ring_range(top - 1, top, 0, top) and rules.ring_range(top - 1, top, 1, top)
    assert not rules.ring_range(0, 0, top, top) and rules.ring_range(0, 1, top, top) and rules.ring_place(2 * top - 1, top) == top - 1


def test_workgroups_of_a_compaction(rules):
    """What is checked is what is launched: an odd number of chunks, 17 at most, and fewer than 2^24 workgroups of 256 threads."""
    for N in range(1, 8193):
        n = min((N + 63) // 64, 16)
        assert rules.gather_chunks(N) == n + (n % 2 == 0)
    A, st = C.c_void_p(4096), Bd._Strides(0, 8192, 128, 64)
    for N in (1, 64, 65, 128, 129, 1024, 1025, 8192):
        chunks, L, Hkv = rules.gather_chunks(N), 64, 3
        most = ((1 << 24) - 1) // (chunks * L * Hkv)          # sequences
        assert rules.gather_fits(N, Hkv, C.c_longlong(most * L)) and not rules.gather_fits(N, Hkv, C.c_longlong((most + 1) * L))
        assert (most * L * Hkv * chunks) * 256 < 1 << 32 <= ((most + 1) * L * Hkv * chunks) * 256
        shape = C.byref(Bd._Shape(most + 1, L, Hkv, Hkv, N, 64, P.PKV_BF16))
        paging = C.byref(Bd._Paging(8, 16, 4, 64))
        assert P.load().prefixkv_compact_paged(shape, A, st, A, st, A, A, paging, 0, A, A, A, A, None) == 7, N
