"""The sizes at which the GPU tests try offsets that are none run the tiles that are split and joined; and
where the tiles of such offsets lie, counted on the CPU as the kernels count them: inside the
buffers."""
import pytest

import test_gpu_grouped_offsets as G
from group_launches import group_launches

UNITS, LEAST = 256, 64 * 8            # compute units; the least of a reduction that a part has


def test_they_run_the_split_tiles():
    got = group_launches([(what, G.P, 1 if what == "w" else len(G.SKEW), n, k) for what, n, k in G.SIZES])
    assert got == [[f"turns_kernel<{i}>", f"join_kernel<{i}>"] for i in range(3)]


def _rows(offsets, e):
    lo = min(max(offsets[e], 0), G.P)
    return lo, max(lo, min(offsets[e + 1], G.P))


def _shares(tiles, reduction):
    """(tiles worked on whole, the others, parts of each)."""
    rest = tiles % UNITS
    parts = min(UNITS // rest, reduction // LEAST) if rest else 1
    return (tiles - rest, rest, parts) if parts > 1 else (tiles, 0, 1)


@pytest.mark.parametrize("bad", G.BAD)
@pytest.mark.parametrize("what,n,k", G.SIZES[:2])
def test_tiles_lie_inside_the_buffers(bad, what, n, k):
    columns, reduction = (-(-n // 256), k) if what == "linear" else (-(-k // 256), n)
    placed = []
    for e in range(len(bad) - 1):
        lo, hi = _rows(bad, e)
        placed += [(lo + 256 * i, min(256, hi - lo - 256 * i)) for i in range(-(-(hi - lo) // 256))]
    assert all(0 <= first and live > 0 and first + live <= G.P for first, live in placed)
    whole, rest, parts = _shares(len(placed) * columns, reduction)
    # the parts of the others lie in the workspace, which has a tile for each unit
    assert rest * parts <= UNITS and whole + (rest if parts > 1 else 0) == len(placed) * columns
