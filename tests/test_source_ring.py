"""The ring of K and V tiles of the shared-prefix attention: barriers tell two phases apart, not three, so whoever waits for a tile must know that the one
before it in the same slot has landed; else the wait returns a phase early, on the old tile.  No run shows a breach; the order of the waits does."""
import os
import re

import pytest

from paper_2609_36938_b200 import build


def code():
    with open(os.path.join(build.CSRC, "attn_shared_tc.cu")) as f:
        return re.sub(r"//[^\n]*", "", f.read())


def rests_before_clearing():
    """Whether a group waits for its P . V of the tile before ahead of the V tile that it clears rows of."""
    loop = code().split("for (int t = first; t < tiles; t += step)")[1].split("// ---- what this fragment leaves")[0]
    clear = loop.index("wait_warp(&sh->full[slot]")
    rest = loop.find("wait_warp(&sh->pv_done[w]")
    return 0 <= rest < clear


def events(slots, fragments, partial, rest_first):
    """(predecessors of every event, waits for a tile with what they must know) of fragments one behind the other, (heavy, tiles) each; in tile `partial` some key does
    not count.  Heavy: both groups work on every tile; else they take the tiles in turn, across fragments too."""
    before, needs = {}, []

    def follow(event, *after):
        before.setdefault(event, set()).update(a for a in after if a is not None)
        return event

    steps, tile, light = [], 0, 0                   # (tile, group, heavy) by fragment
    for heavy, tiles in fragments:
        steps.append([(tile + t, w, heavy) for t in range(tiles) for w in ((0, 1) if heavy else ((light + t) & 1,))])
        tile += tiles
        light += 0 if heavy else tiles
    flat = [s for f in steps for s in f]
    user = {s[0]: s for s in flat}                  # the last step that a tile is used in
    last = None
    for u in range(2 * tile):                       # unit 2 t: K of tile t, 2 t + 1: V
        old = u - slots
        freed = None if old < 0 else ("qk" if old % 2 == 0 else "pv", user[old // 2])
        last = follow(("issue", u), last, freed)
        follow(("land", u), last)

    def wait_tile(name, u, *after):
        start = follow((name, u), *after)
        if u >= slots:
            needs.append((start, ("land", u - slots)))
        return follow((name, u, "done"), start, ("land", u))

    last, previous = None, None
    for s in flat:                                  # the warp of Q . K
        if s[1] == 0 or not s[2]:
            last = wait_tile("qk waits", 2 * s[0], last)
        last = follow(("qk", s), last, None if previous is None else ("in registers", previous))
        previous = s
    last = None
    for s in flat:                                  # the warp of P . V
        if s[1] == 0 or not s[2]:
            last = wait_tile("pv waits", 2 * s[0] + 1, last)
        last = follow(("pv", s), last, ("p", s))
    for w in (0, 1):                                # the groups
        last = None
        for fragment in steps:
            at_rest = None
            for s in [s for s in fragment if s[1] == w]:
                last = follow(("starts", s), last, ("qk", s))
                if s[0] == partial:
                    if rest_first:
                        last = follow(("rests", s), last, at_rest)
                    last = wait_tile(("clears", w), 2 * s[0] + 1, last)
                last = follow(("in registers", s), last)
                last = follow(("p", s), last, at_rest)
                at_rest = ("pv", s)
            if at_rest is not None:
                last = follow(("leaves", fragment[0], w), last, at_rest)
    return before, needs


def early(slots, fragments, partial, rest_first):
    """Waits that may return on the tile before."""
    before, needs = events(slots, fragments, partial, rest_first)
    out = []
    for start, must in needs:
        seen, todo = set(), [start]
        while todo:
            e = todo.pop()
            if e not in seen:
                seen.add(e)
                todo += before.get(e, ())
        if must not in seen:
            out.append((start, must))
    return out


@pytest.mark.parametrize("heavy", [False, True])
def test_a_group_that_clears_rows_waits_for_the_tile_itself(heavy):
    for slots in (4, 8):
        for partial in range(9):
            bad = [e for e in early(slots, [(heavy, 9)], partial, rests_before_clearing()) if e[0][0][0] == "clears"]
            assert not bad, (slots, partial, bad)


def test_tiles_of_k_and_v_keep_their_slots():
    """With a number of slots divisible by four K follows K and V follows V of the same group, whatever room there is."""
    expression = re.search(r"static constexpr int SLOTS = ([^;]*);", code()).group(1)
    most = int(re.search(r"ST_MAX_SLOTS = (\d+)", code()).group(1))
    picked = re.fullmatch(r"\(?ROOM < ST_MAX_SLOTS \? ROOM : ST_MAX_SLOTS\)?(?: / 4 \* 4)?", expression)
    assert picked, expression
    for room in range(4, 16):
        slots = min(room, most) // 4 * 4 if "/ 4 * 4" in expression else min(room, most)
        for heavy in (False, True):
            for partial in range(9):
                bad = early(slots, [(heavy, 9)], partial, rests_before_clearing())
                assert not bad, (room, slots, partial, bad)


@pytest.mark.parametrize("heavy", [(), (1,), (3, 1), (1, 1, 2)])
@pytest.mark.parametrize("light", [(1,), (3,), (1, 2, 1, 3), (5, 1, 1, 1, 4), (1, 1, 1, 1, 1, 1, 1, 1)])
def test_fragments_one_behind_the_other(heavy, light):
    """A CTA's stretch: segments of more than 128 rows come first, the groups' turns run on across the others."""
    fragments = [(True, n) for n in heavy] + [(False, n) for n in light]
    for slots in (4, 8):
        for partial in range(sum(heavy) + sum(light)):
            bad = early(slots, fragments, partial, rests_before_clearing())
            assert not bad, (slots, partial, bad)
