"""Which rows a workgroup of the elementwise passes takes (csrc/row_deal.h), compiled for the host: every row once, in launches that the hardware takes."""
import ctypes as C
import os
import subprocess

import numpy as np
import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2109_04312_amd", "csrc")
SOURCE = """
#include "row_deal.h"
using namespace mate;
extern "C" {
// grid [2], rows of a workgroup, units of a row, 2^32 / units
void deal(int rows, int E, long* out) {
  const RowDeal d = deal_rows(rows, E, 32);
  const dim3 g = groups_of(d);
  out[0] = g.x; out[1] = g.y; out[2] = d.each; out[3] = d.units; out[4] = d.by;
}
// first row and rows of n workgroups
void rows_of(int rows, int E, long n, const unsigned* x, const unsigned* y, long* first, long* count) {
  const RowDeal d = deal_rows(rows, E, 32);
  for (long i = 0; i < n; ++i) { first[i] = first_row(d, x[i], y[i]); count[i] = rows_from(d, first[i]); }
}
}
"""
MOST = 2 ** 31 - 1025   # tokens of a call


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("rows")
    (d / "rows.cpp").write_text(SOURCE)
    so = str(d / "rows.so")
    subprocess.run(["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-D__HIP_PLATFORM_AMD__=1", "-I/opt/rocm/include", f"-I{CSRC}",
                    str(d / "rows.cpp"), "-o", so], check=True)
    return C.CDLL(so)


def dealt(lib, rows, E):
    out = (C.c_long * 5)()
    lib.deal(rows, E, out)
    return list(out)


def rows_of(lib, rows, E, x, y):
    x, y = np.broadcast_arrays(np.asarray(x, np.uint32), np.asarray(y, np.uint32))
    x, y = np.ascontiguousarray(x), np.ascontiguousarray(y)
    first, count = np.empty(len(x), np.int64), np.empty(len(x), np.int64)
    p = lambda a: a.ctypes.data_as(C.c_void_p)
    lib.rows_of(rows, E, C.c_long(len(x)), p(x), p(y), p(first), p(count))
    return first, count


WIDTHS = [8, 24, 32, 40, 72, 768, 1032, 2056, 4096, 4104, 5560, 8192, 65528, 65536]


@pytest.mark.parametrize("E", WIDTHS)
@pytest.mark.parametrize("rows", [1, 2, 255, 4097, 262145, 2 ** 23, 2 ** 24 - 1, 2 ** 24, 2 ** 24 + 1, 50000000, MOST])
def test_launches_that_the_hardware_takes(lib, rows, E):
    gx, gy, each, units, by = dealt(lib, rows, E)
    assert gx * 256 < 2 ** 32 and gy < 65536 and each >= 1
    # the rows of a grid row follow those of the one before, and the last workgroup with any ends at the last row
    first, count = rows_of(lib, rows, E, [0, gx - 1] * gy, np.repeat(np.arange(gy), 2))
    assert first[0] == 0 and np.array_equal(first[2::2], first[1:-1:2] + each)
    assert (count <= each).all() and (gx - 1) * each < rows <= gx * gy * each
    i = (rows - 1) // each
    assert [int(v[0]) for v in rows_of(lib, rows, E, [i % 2 ** 23], [i >> 23])] == [i * each, rows - i * each]
    if gx * gy > i + 1:   # those behind it have none
        assert int(rows_of(lib, rows, E, [(i + 1) % 2 ** 23], [(i + 1) >> 23])[1][0]) <= 0
        assert int(rows_of(lib, rows, E, [gx - 1], [gy - 1])[1][0]) <= 0


@pytest.mark.parametrize("rows,E", [(1, 8), (700, 48), (4097, 136), (300001, 40), (70000, 4104)])
def test_every_row_once(lib, rows, E):
    gx, gy, each, _, _ = dealt(lib, rows, E)
    first, count = rows_of(lib, rows, E, np.tile(np.arange(gx), gy), np.repeat(np.arange(gy), gx))
    has = count > 0
    assert np.array_equal(np.concatenate([np.arange(f, f + c) for f, c in zip(first[has], count[has])]), np.arange(rows))


@pytest.mark.parametrize("E", WIDTHS)
def test_quotient_by_the_units_of_a_row(lib, E):
    _, _, each, units, by = dealt(lib, 300000, E)
    i = np.arange(each * units + 1, dtype=np.uint64)
    assert np.array_equal((i * np.uint64(by)) >> np.uint64(32), i // np.uint64(units))
