"""The rings through which codes are widened (csrc/window.cu), as a model in which everything that can happen is tried.

An mbarrier's wait is by parity: it passes while the phase of the other parity is the current one.  So it tells two successive phases apart and no
more, and who does not see every phase of a barrier has to know otherwise that the one before last is over.  Two warps widen the tiles of a ring in
turn; copies land in any order.  Ring sizes and the order of the two waits come from the source."""
import re
from pathlib import Path

import pytest

SOURCE = (Path(__file__).resolve().parent.parent / "paper_2401_15077_b200" / "csrc" / "window.cu").read_text()
WARPS, STEPS = 2, 8


def _constant(name):
    return int(re.search(rf"\b{name} = (?:CODES \? )?(\d+)", SOURCE).group(1))


def _order(codes, slot):
    """The barriers that a widening warp waits for, in order."""
    line = next(x for x in SOURCE.splitlines() if f"mbar_wait_warp(B.{codes}(" in x and f"mbar_wait_warp(B.{slot}(" in x)
    return ["codes" if b == codes else "slot" for b in re.findall(r"mbar_wait_warp\(B\.(\w+)\(", line)]


def _first_wrong(stages, slots, order):
    """Every interleaving of the producer, copies that land when they like, two widening warps and an issuer whose MMAs end in order; what goes wrong
    first, or None.  All barriers count one arrival: their phases are numbers here."""
    passes = lambda phase, parity: (phase & 1) != parity  # noqa: E731
    # asked: copies issued; landed: of those, which have arrived; full / empty (stages), ready / used (slots): phases completed;
    # at: (step, waits passed) of the warps; read: steps widened; done: MMAs finished
    start = (0, frozenset(), (0,) * stages, (0,) * stages, (0,) * slots, (0,) * slots, tuple((w, 0) for w in range(WARPS)), 0)
    seen, todo = {start}, [start]
    bump = lambda t, i: t[:i] + (t[i] + 1,) + t[i + 1:]  # noqa: E731
    while todo:
        asked, landed, full, empty, ready, used, at, done = todo.pop()
        after = []
        if asked < STEPS and passes(empty[asked % stages], (asked // stages & 1) ^ 1):
            after.append((asked + 1, landed, full, empty, ready, used, at, done))
        for g in range(asked):
            if g not in landed:
                after.append((asked, landed | {g}, bump(full, g % stages), empty, ready, used, at, done))
        for w, (g, waits) in enumerate(at):
            if g >= STEPS:
                continue
            if waits < len(order):
                ok = passes(full[g % stages], g // stages & 1) if order[waits] == "codes" else passes(used[g % slots], (g // slots & 1) ^ 1)
                if ok:
                    after.append((asked, landed, full, empty, ready, used, at[:w] + ((g, waits + 1),) + at[w + 1:], done))
                continue
            if g not in landed:
                return f"step {g} is widened before its codes have landed"
            if done < g - slots + 1:
                return f"step {g} is widened into a tile that is still read"
            after.append((asked, landed, full, bump(empty, g % stages), bump(ready, g % slots), used, at[:w] + ((g + WARPS, 0),) + at[w + 1:], done))
        if done < STEPS and passes(ready[done % slots], done // slots & 1):
            after.append((asked, landed, full, empty, ready, bump(used, done % slots), at, done + 1))
        if not after and done < STEPS:
            return "everyone waits"
        for s in after:
            if s not in seen:
                seen.add(s)
                todo.append(s)
    return None


@pytest.mark.parametrize("ring", ["k", "v"])
def test_a_tile_is_widened_from_its_own_codes(ring):
    stages, slots = (_constant(f"k{ring.upper()}{what}") for what in ("Stages", "Slots"))
    order = _order(f"{ring}c_full", f"{ring}_empty")
    assert sorted(order) == ["codes", "slot"]
    assert _first_wrong(stages, slots, order) is None


def test_what_the_model_finds():
    """A stage with two owners that look at its codes first takes an earlier use's phase for their own; one owner, or the tile's turn first, and it is right."""
    assert "landed" in _first_wrong(3, 3, ["codes", "slot"])
    assert _first_wrong(4, 3, ["codes", "slot"]) is None
    assert _first_wrong(3, 3, ["slot", "codes"]) is None
    assert "landed" in _first_wrong(3, 4, ["slot", "codes"])      # (four tiles, of which the fourth's turn says nothing of the first's codes)
