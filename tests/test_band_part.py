"""The part of an interval of relative positions that lies in a band of diagonals (csrc/qgx_plan.h, band_part), built with the host
compiler: whatever 32-bit bounds the interval has, the places that the gradient kernel then reads lie inside its span."""
import ctypes as C
import itertools
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
WRAPPER = r"""
#include "qgx_plan.h"
extern "C" void band_part(int bound, int stop, int first, int span, int* out)
{
    const qgx::BandPart p = qgx::band_part(bound, stop, first, span);
    out[0] = p.at;
    out[1] = p.n;
}
"""
LOW, HIGH = -(1 << 31), (1 << 31) - 1


@pytest.fixture(scope="module")
def band_part(tmp_path_factory):
    d = tmp_path_factory.mktemp("band")
    (d / "w.cpp").write_text(WRAPPER)
    subprocess.check_call(["g++", "-std=c++17", "-O2", "-Wall", "-Werror", "-shared", "-fPIC", "-I",
                           os.path.join(ROOT, "paper_2308_09187_amd", "csrc"), "-o", str(d / "w.so"), str(d / "w.cpp")])
    f = C.CDLL(str(d / "w.so")).band_part
    out = (C.c_int * 2)()

    def call(bound, stop, first, span):
        f(bound, stop, first, span, out)
        return out[0], out[1]

    return call


@pytest.mark.parametrize("span", [64 + 4, 128 + 8, 256 + 4, 512 + 8])
def test_every_part_lies_in_the_band(band_part, span):
    reach = (1 << 30) + (1 << 29)                              # of a diagonal: keys, queries and the first query's position
    firsts = [-reach - 1024, -reach, -(1 << 30) - 16, -(1 << 30), -2007, -span, -1, 0, 1, 2, 1999, (1 << 30) - 8, 1 << 30, reach - 4]
    far = [LOW, LOW + 1, -3 << 29, -(1 << 30), -1, 0, 1, 1 << 30, 3 << 29, HIGH - 1, HIGH]
    for first in firsts:
        near = [x for x in (first - 1, first, first + 1, first + 17, first + span - 1, first + span, first + span + 1) if LOW <= x <= HIGH]
        points = sorted(set(far + near))
        for bound, stop in itertools.combinations(points, 2):
            at, n = band_part(bound, stop, first, span)
            want = range(max(bound, first) - first, max(min(stop, first + span), max(bound, first)) - first)     # (Python's integers)
            assert 0 <= at <= span and 0 <= n and at + n <= span, (bound, stop, first)
            assert n == len(want) and (n == 0 or at == want.start), (bound, stop, first)
