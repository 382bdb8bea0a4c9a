"""What the chunk's attention hands from warp to warp through shared memory, run on the host: the warps take steps in any
order that the waits of csrc/chunk.cu allow, and nothing that is still to be read is written over.  How many places there
are, and how they are chosen, is read from the sources."""
import os
import re

import numpy as np
import pytest

from .plans import CSRC

TEXT = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, "chunk.cu")).read())


def number(pattern):
    found = re.findall(pattern, TEXT)
    assert found and len(set(found)) == 1, (pattern, found)
    return int(found[0])


def ring_tiles():
    """Tiles of keys and values that a CTA's ring holds, for head_dim 64 and above."""
    a, b = re.search(r"kStages = D == 64 \? (\d+) : (\d+)", TEXT).groups()
    return int(a) // 2, int(b) // 2


def flags(tiles, places, segments, rng, owners_late):
    """Segments of one tile.  The copying warps note segment s's infinities in place s mod `places` once the ring has room for
    its tile; products end segment s; the owners of rows then read the place, and segment s + 1's products wait for them."""
    flag = [None] * places
    copied = ended = read = 0
    while read < segments:
        moves = []
        if copied < segments and copied < ended + tiles:
            moves.append("copy")
        if ended < copied and ended <= read:      # behind the owners' queries, which they bring behind their reading
            moves.append("end")
        if read < ended and rng.random() > owners_late:
            moves.append("read")
        if not moves:
            continue
        move = moves[rng.integers(len(moves))]
        if move == "copy":
            flag[copied % places] = copied
            copied += 1
        elif move == "end":
            ended += 1
        else:
            assert flag[read % places] == read, "the segment's flag is gone"
            read += 1


@pytest.mark.parametrize("which", [0, 1])
def test_flags_of_infinities_outlive_their_reading(which):
    places = number(r"volatile int unclean\[(\d+)\]")
    assert number(r"sh\.unclean\[seg & (\d+)\]") == places - 1 and places & (places - 1) == 0
    rng = np.random.default_rng(which)
    for late in (0.0, 0.5, 0.95):
        for _ in range(60):
            flags(ring_tiles()[which], places, 60, rng, late)


def test_as_many_places_as_tiles_would_not_do():
    with pytest.raises(AssertionError):
        for seed in range(200):
            flags(4, 4, 60, np.random.default_rng(seed), 0.95)
