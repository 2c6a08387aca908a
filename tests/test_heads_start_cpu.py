"""Which token's angles and which row each team of a work-group begins with, on the CPU: what the
kernels of the heads read of a work-group's angles lies within them, whatever the team."""
import ctypes
import os
import subprocess

import pytest


@pytest.fixture(scope="module")
def shim(tmp_path_factory):
    here = os.path.dirname(os.path.abspath(__file__))
    out = str(tmp_path_factory.mktemp("heads") / "heads_start_shim.so")
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-shared", "-fPIC", "-o", out, os.path.join(here, "heads_start_shim.cpp")],
                   check=True)
    return ctypes.CDLL(out)


@pytest.mark.parametrize("E", [4, 8])
def test_every_team_reads_angles_that_are_there(shim, E):
    layout, start = (ctypes.c_int * 5)(), (ctypes.c_int * 2)()
    idle = 0
    for d in (1, 2, 7, 16, 50, 64, 80, 96, 128, 200, 255, 256):
        for pairs in {0, 1, d // 4, d // 2}:
            if 2 * pairs > d:
                continue
            for rows in (1, 2, 3, 4, 5, 6, 7, 11, 12, 13, 15, 16, 20, 31, 32, 33, 48, 100):
                shim.shim_layout(d, pairs, E, ctypes.c_int64(rows), layout)
                threads, teams, tokens, team, pair_chunks = layout
                assert teams * team == threads
                seen = set()
                for slot in range(teams):
                    shim.shim_start(slot, tokens, rows, start)
                    token, row = start
                    # the angles of `tokens` tokens, `pairs` each; a lane's first is its chunk's
                    for c in range(pair_chunks):
                        assert 0 <= token * pairs + c * E < tokens * pairs, (d, pairs, rows, slot)
                    if tokens > 1 and row < rows:
                        assert (token, row) not in seen
                        seen.add((token, row))
                    idle += tokens > 1 and row >= rows
                if tokens > 1:
                    assert len(seen) == tokens * rows
                else:
                    assert start[0] == 0
    assert idle > 100  # work-groups with teams that have no row are among these
