"""Grids of the tiles' kernels: as many workgroups as there may be tiles, and fewer than 2^32 threads along an axis, which is what a launch takes.  No GPU needed."""
import os

import pytest

import tile_rules

pytestmark = pytest.mark.skipif(not os.path.exists(tile_rules.HIPCC), reason="no hipcc")


def test_grids_are_what_a_launch_takes():
    wanted = [1, 8, (1 << 20) - 8, 1 << 20, (1 << 20) + 8, (1 << 24) - 8, 1 << 24, 2050 * 8192, 0x7ff00010]
    got = tile_rules.values(("mw_few.h",), tuple("grid_of(%du).%s" % (n, axis) for n in wanted for axis in "xyz") + ("kTileThreads", "kAcross"))
    threads, across = got[-2:]
    for n, x, y, z in zip(wanted, got[0:-2:3], got[1:-2:3], got[2:-2:3]):
        assert x * threads < 1 << 32 and y < 65536 and z == 1 and x * y >= n and (x == n if y == 1 else x == across)
        assert (y - 1) * across < n                                    # (no row of the grid without a workgroup that is wanted)
    assert across % 8 == 0                                             # workgroups are dealt out to the eight XCDs in turn, row behind row
