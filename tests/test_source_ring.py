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


def events(slots, tiles, heavy, partial, rest_first):
    """(predecessors of every event, waits for a tile with what they must know) of one fragment of `tiles` tiles, of which `partial` has keys that do not
    count.  Heavy: both groups work on every tile; else they take the tiles in turn."""
    before, needs = {}, []

    def follow(event, *after):
        before.setdefault(event, set()).update(a for a in after if a is not None)
        return event

    steps = [(t, w) for t in range(tiles) for w in ((0, 1) if heavy else (t & 1,))]
    last = None
    for u in range(2 * tiles):                      # unit 2 t: K of tile t, 2 t + 1: V
        old = u - slots
        freed = None if old < 0 else ("qk" if old % 2 == 0 else "pv", [s for s in steps if s[0] == old // 2][-1])
        last = follow(("issue", u), last, freed)
        follow(("land", u), last)

    def wait_tile(name, u, *after):
        start = follow((name, u), *after)
        if u >= slots:
            needs.append((start, ("land", u - slots)))
        return follow((name, u, "done"), start, ("land", u))

    last, previous = None, None
    for s in steps:                                 # the warp of Q . K
        if s[1] == 0 or not heavy:
            last = wait_tile("qk waits", 2 * s[0], last)
        last = follow(("qk", s), last, None if previous is None else ("in registers", previous))
        previous = s
    last = None
    for s in steps:                                 # the warp of P . V
        if s[1] == 0 or not heavy:
            last = wait_tile("pv waits", 2 * s[0] + 1, last)
        last = follow(("pv", s), last, ("p", s))
    for w in (0, 1):                                # the groups
        last, previous = None, None
        for s in [s for s in steps if s[1] == w]:
            at_rest = None if previous is None else ("pv", previous)
            last = follow(("starts", s), last, ("qk", s))
            if s[0] == partial:
                if rest_first:
                    last = follow(("rests", s), last, at_rest)
                last = wait_tile(("clears", w), 2 * s[0] + 1, last)
            last = follow(("in registers", s), last)
            last = follow(("p", s), last, at_rest)
            previous = s
    return before, needs


def early(slots, tiles, heavy, partial, rest_first):
    """Waits that may return on the tile before."""
    before, needs = events(slots, tiles, heavy, partial, rest_first)
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
            bad = [e for e in early(slots, 9, heavy, partial, rests_before_clearing()) if e[0][0][0] == "clears"]
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
                bad = early(slots, 9, heavy, partial, rests_before_clearing())
                assert not bad, (room, slots, partial, bad)
