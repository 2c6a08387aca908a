"""The grids of the 8-bit row kernels, on the CPU: every row has its work-items,
and no launch has more of them than a launch takes (fewer than 2^32)."""
import ctypes
import os
import re
import subprocess

import pytest

from paper_1904_05347_amd import build

SHIM_SRC = os.path.join(os.path.dirname(os.path.abspath(__file__)), "rows_i8_shim.cpp")


@pytest.fixture(scope="module")
def shim(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("shim") / "librows_i8_shim.so")
    subprocess.run(["g++", "-O1", "-std=c++20", "-shared", "-fPIC", SHIM_SRC, "-o", out], check=True, capture_output=True)
    lib = ctypes.CDLL(out)
    lib.shim_most_rows.restype = lib.shim_rows_groups.restype = ctypes.c_int64
    lib.shim_rows_groups.argtypes = [ctypes.c_int64, ctypes.c_int]
    return lib


def _teams():
    """Work-items a row of every form that the launches name."""
    with open(os.path.join(build.CSRC, "pk_rows_i8.hip")) as fh:
        text = fh.read()
    teams = {int(t) for t in re.findall(r"PK_ROWS\((\d+), \d+\)", text)}
    teams |= {int(t) for t in re.findall(r"dequantize_i8_kernel<T, (\d+)>", text)}
    return teams


def test_the_largest_launch_is_within_the_limit(shim):
    teams = _teams()
    assert {64, 256, 1024} <= teams
    for team in teams:
        assert shim.shim_rows_groups(shim.shim_most_rows(), team) * shim.shim_rows_group(team) < 1 << 32, team


def test_every_row_has_its_team(shim):
    for team in _teams():
        a_group = shim.shim_rows_group(team) // team
        assert a_group * team == shim.shim_rows_group(team) <= 1024
        for rows in (1, 2, 3, 4, 5, 1001, shim.shim_most_rows()):
            groups = shim.shim_rows_groups(rows, team)
            assert (groups - 1) * a_group < rows <= groups * a_group, (team, rows)
