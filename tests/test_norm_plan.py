"""How the norms' launches divide their rows (csrc/norm_plan.h), walked through on the host over all widths up to the largest row counts that are accepted (no GPU needed)."""
import ctypes
import itertools
import shutil
import subprocess

import pytest

import paper_2502_02581_amd as moe
from paper_2502_02581_amd import build
from paper_2502_02581_amd.binding import _CNorm

SHIM = r"""
#include "norm_plan.h"
using namespace moe;
static long teams(const NormPlan& p) { return wide_team(p.team) ? 1 : p.waves * 64 / lanes_of(p.team); }
extern "C" int max_rows() { return kNormMaxRows; }
// over all widths: the last index that a team's next row takes
extern "C" long last_index(int rows, int dtype, int backward, int drop, int in_place) {
  long last = 0;
  for (int d = 1; d <= kNormMaxD; d++) {
    const moe_norm_t n = {rows, d, dtype, dtype, 0, 0.f};
    const NormPlan p = norm_plan(&n, backward, drop, in_place);
    const long next = rows - 1L + p.blocks * teams(p);
    if (next > last) last = next;
  }
  return last;
}
// widths whose plan has not one block of rows at least and 2048 at most, or more of them than a team each needs
extern "C" int unfit(int rows, int dtype, int backward, int drop, int in_place) {
  int bad = 0;
  for (int d = 1; d <= kNormMaxD; d++) {
    const moe_norm_t n = {rows, d, dtype, dtype, 0, 0.f};
    const NormPlan p = norm_plan(&n, backward, drop, in_place);
    bad += p.blocks < 1 || p.blocks > 2048 || (p.blocks - 1) * teams(p) >= rows;
  }
  return bad;
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no host compiler")
    d = tmp_path_factory.mktemp("plan")
    (d / "shim.cpp").write_text(SHIM)
    subprocess.run([cxx, "-std=c++17", "-O1", "-Wall", "-Werror", "-fwrapv", "-shared", "-fPIC", "-I", build.CSRC, "-o", str(d / "shim.so"), str(d / "shim.cpp")], check=True)
    lib = ctypes.CDLL(str(d / "shim.so"))
    lib.last_index.restype = ctypes.c_long
    return lib


def forms():
    """dtype, backward, drop, in_place"""
    return itertools.product((0, 1), (0, 1), (0, 1), (0, 1))


def test_next_rows_are_indices(plan):
    """The kernels' row numbers have 32 bits, and a team asks for its next row before it looks whether there is one."""
    most = plan.max_rows()
    for form in forms():
        for rows in (1, 1000, 1 << 20, most - 1, most):
            assert plan.last_index(rows, *form) < 1 << 31, (rows, form)


def test_the_line_of_row_counts(plan):
    """The library refuses what is beyond the line that the plans were looked at to, and accepts what is on it."""
    lib = moe.load_library()
    assert lib.moe_norm_bwd_workspace_bytes(ctypes.byref(_CNorm(plan.max_rows(), 8, 1, 1, 0, 1e-5))) > 0
    assert lib.moe_norm_bwd_workspace_bytes(ctypes.byref(_CNorm(plan.max_rows() + 1, 8, 1, 1, 0, 1e-5))) == 0


ROWS = (1, 7, 1000, 1 << 20, 1 << 30, 2143297000, 2143400000, 2 ** 31 - 2 ** 15 - 2, 2 ** 31 - 2 ** 15 - 1)   # (the last: the largest accepted)


@pytest.mark.parametrize("rows", ROWS)
def test_blocks(plan, rows):
    """Every plan has blocks, and none that no row is left for."""
    for form in forms():
        assert plan.unfit(rows, *form) == 0, form


@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("d", [1, 128, 200, 1000, 1100, 7168, 16384])
def test_workspace(rows, d):
    """Two rows of sums for each of 2048 blocks at most."""
    for dtype, kind in itertools.product((0, 1), (0, 1)):
        need = moe.load_library().moe_norm_bwd_workspace_bytes(ctypes.byref(_CNorm(rows, d, dtype, 0, kind, 1e-5)))
        assert 8 * d <= need <= 2048 * 8 * d + 256, (need, dtype)
