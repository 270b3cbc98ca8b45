"""How far below its area the walk of an item (walk_item in mas_kernels.hip) can read in
LDS, whatever the step masks or descent bytes it walks from are: the steps of one group
of four chunks, every extreme choice of each, against the room the kernel leaves."""
from __future__ import annotations

import os
import re

import pytest

SOURCE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2409_07704_amd", "csrc", "mas_kernels.hip")
ROWS, CHUNK, ESCAPE = 63, 32, 64  # rows of a wave, columns of a chunk, first escape byte


def lowest(masks):
    """Lowest LDS address read, from the area's start on, by a group that begins in a row
    above 0, in the lowest chunk of an item of one wave (whose rows lie lowest)."""
    size = 4 if masks else 1
    least = 0

    def read(entry):
        nonlocal least
        least = min(least, entry * size)

    def body(e, g, n):
        if n == 0:
            return
        rr = e - ROWS * g
        # (mask population or byte, its highest position)
        choices = [(0, -1), (1, 0), (32, 31), (31, 30)] if masks else [(0, -1), (63, -1)] + [(b, b - ESCAPE) for b in (64, 94, 95, 255)]
        for value, pos in choices:
            if not (value > rr if masks else value >= ESCAPE):
                step(e - value, g, n)
                continue
            if pos < CHUNK - 1:
                read(CHUNK * (g - 1) + pos + 1)
            for mid in ((0,) if pos >= CHUNK - 1 else (0, 32) if masks else (0, 255)):
                step(e - (rr + 1 + mid), g - 1, n)

    def step(e, g, n):
        read(CHUNK + e - 63)  # the 64 lanes' rows, e down to e - 63
        body(e, g, n - 1)

    for e in range(1, 3 * ROWS):
        for g in range(e // ROWS, 4):  # unstaged bytes lower the row without its wave
            step(e, g, 5)
    return least


@pytest.mark.parametrize("masks", [True, False])
def test_reads_below_the_area(masks):
    below = int(re.search(r"kBelowArea = (\d+);", open(SOURCE).read()).group(1))
    assert -below <= lowest(masks) < 0


def test_the_room_is_what_the_worst_walk_takes():
    below = int(re.search(r"kBelowArea = (\d+);", open(SOURCE).read()).group(1))
    assert min(lowest(True), lowest(False)) == -below
