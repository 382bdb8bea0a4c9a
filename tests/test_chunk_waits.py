"""What the chunk's attention hands from warp to warp through shared memory, run on the host: the warps take steps in any
order that the waits of csrc/chunk.cu allow, and nothing that is still to be read is written over.  How many places there
are, and how they are chosen, is read from the sources."""
import os
import re

import numpy as np
import pytest

from .plans import CSRC

TEXT = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, "chunk.cu")).read())
WEIGHTS = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, "weights.cu")).read())


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


def body(head, text=TEXT):
    """The text of the function whose declaration starts so."""
    start = text.index("{", text.index(head))
    depth = 0
    for i in range(start, len(text)):
        depth += (text[i] == "{") - (text[i] == "}")
        if depth == 0:
            return text[start:i + 1]


def landings(ring, warps, tiles, together, rng):
    """Tensor copies of values that are to be looked through: the first copying warp arms one barrier for each, all wait on it by
    one bit of its phases, look through what came and hand it on.  The ring has room once all have handed on the tile that stood
    there.  together: the warps meet behind the wait."""
    armed = landed = 0
    at = [0] * warps                  # tiles that a warp has handed on
    passed = [0] * warps              # waits that a warp is behind
    phase = lambda w, n: landed % 2 != n % 2          # the wait for phase n ends while another parity is current  # noqa: E731
    while min(at) < tiles:
        moves = []
        for w in range(warps):
            n = at[w]
            if n >= tiles:
                continue
            if w == 0 and armed == n and min(at) > n - ring:
                moves.append(("arm", w))
            if passed[w] == n and (w or armed > n) and min(at) > n - ring and phase(w, n):
                assert landed > n, "read before it is there"
                moves.append(("pass", w))
            if passed[w] > n and (not together or min(passed) > n):
                moves.append(("hand on", w))
        if landed < armed:
            moves.append(("land", 0))
        assert moves, "everybody waits"
        move, w = moves[rng.integers(len(moves))]
        if move == "arm":
            armed += 1
        elif move == "land":
            landed += 1
        elif move == "pass":
            passed[w] += 1
        else:
            at[w] += 1


def warps_meet():
    """Whether all copying warps meet between the wait for a tile's values and the looking through."""
    text = body("void tensor_tile(")
    wait = text.index("wait(bar,")
    return "named_sync(1, kCopyThreads)" in text[wait:text.index("clean(", wait)]


@pytest.mark.parametrize("which", [0, 1])
def test_no_copying_warp_is_left_a_phase_behind(which):
    rng = np.random.default_rng(which)
    for _ in range(200):
        landings(ring_tiles()[which], 3, 30, warps_meet(), rng)


def test_one_bit_would_not_do_without_meeting():
    with pytest.raises(AssertionError):
        for seed in range(200):
            landings(4, 3, 30, False, np.random.default_rng(seed))


def offsets(by_lanes, by_tile, warps, rng):
    """Tiles that are copied by lanes (else by tensor copies, at which these warps need not meet): each warp writes its part of the
    tile's table of offsets, all meet, each reads all of it.  by_tile: a tile's table goes by its number, else by how many were
    copied by lanes before it."""
    tables = [[None] * warps, [None] * warps]
    mine = [j for j, lanes in enumerate(by_lanes) if lanes]
    of = lambda i: tables[(mine[i] if by_tile else i) & 1]    # noqa: E731
    wrote, read = [0] * warps, [0] * warps
    while min(read) < len(mine):
        w = int(rng.integers(warps))
        if read[w] == len(mine):
            continue
        if wrote[w] == read[w]:
            of(wrote[w])[w] = mine[wrote[w]]
            wrote[w] += 1
        elif min(wrote) > read[w]:
            assert all(x == mine[read[w]] for x in of(read[w])), "another tile's offsets"
            read[w] += 1


def test_offsets_outlive_their_reading():
    text = body("void lane_tile(")
    by_tile = "sh.offset[j & 1]" in text
    assert by_tile or "sh.offset[(*tables)++ & 1]" in text
    rng = np.random.default_rng(0)
    for _ in range(300):
        offsets(rng.random(12) < rng.random(), by_tile, 3, rng)


def test_tables_by_the_tile_would_not_do():
    with pytest.raises(AssertionError):
        for seed in range(200):
            offsets([True, False, True], True, 3, np.random.default_rng(seed))


@pytest.mark.parametrize("file,head,step", [("chunk", "bool next(", "step("), ("weights", "bool move_on(", "next<false>()")])
def test_a_walk_in_shared_memory_is_read_behind_a_warp_barrier(file, head, step):
    """One lane moves the walk on and the others read it: a shuffle alone does not order memory."""
    inside = body(head, {"chunk": TEXT, "weights": WEIGHTS}[file])
    assert "__syncwarp()" in inside[:inside.index(step)] and "__syncwarp()" in inside[inside.index(step):]


def test_what_a_walk_in_shared_memory_refers_to_is_every_threads():
    """One lane's addresses of the batch and the plan serve the whole warp, so neither may be a thread's own copy."""
    walk = body("struct WeightWalk", WEIGHTS)
    kept = set(re.findall(r"const (\w+)& \w+;", walk))
    assert kept == {"Batch", "WeightPlan"}
    kernel = WEIGHTS[WEIGHTS.index("weights_kernel(AttnState"):]
    parameters = kernel[:kernel.index("{")]
    for kind in kept:
        assert re.search(rf"const __grid_constant__ {kind} \w+", parameters), kind
