"""CPU-only model of the 4-bit product's rings (mm4_kernel): loads that land in any order, products in order whose arrivals on
barriers come in any order, and sets of warps that make weights of every so many-th stage and wait by a phase's parity alone.
Every interleaving is walked through: no set may pass a wait before what it waits for, and none may wait for ever."""
import os
import re

import pytest

from paper_2504_06323_b200 import build

SOURCE = os.path.join(os.path.dirname(build.__file__), "csrc", "weight4.cu")
WIDTHS = (16, 32, 64, 128)


def constant(name, bn):
    """A constant of the kernel for a tile width: a number, or a chain of BN == width ? number : ..."""
    with open(SOURCE) as f:
        expression = re.search(rf"constexpr int {name} = ([^;]*);", f.read()).group(1)
    for case in expression.split(":"):
        condition, _, value = case.rpartition("?")
        if not condition or int(condition.split("==")[1]) == bn:
            return int(value)


def rings(bn):
    """(slots, made, sets, whether a set waits for room before it waits for codes) of the kernel."""
    slots, made, sets = constant("kC4Slots", bn), constant("kC4Made", bn), constant("kC4Sets", bn)
    with open(SOURCE) as f:
        text = f.read()
    order = [text.find(line) for line in ("if (kC4RoomFirst<BN> && !room()) break;", "if (!mbar_wait(&full[slot], (uint32_t)(s / kSlots) & 1u, err)",
                                          "if (!kC4RoomFirst<BN> && !room()) break;")]
    by_rule = "constexpr bool kC4RoomFirst = kC4Made % kC4Sets<BN> == 0;" in text and -1 < order[0] < order[1] < order[2]
    return slots, made, sets, by_rule and made % sets == 0


def walk(slots, made, sets, room_first, stages):
    """The first fault of any interleaving, or None.  A state: loads issued, the outstanding ones that landed, products done,
    arrivals on `used` and `empty` that came, and for every set its stage, the waits it passed and whether it made it."""
    start = (0, frozenset(), 0, frozenset(), frozenset(), tuple((s, 0) for s in range(sets)))
    seen, todo = {start}, [start]

    def phases(events, ring, slot):
        """Completed phases of a ring's barrier: its events come one after another."""
        return sum(1 for e in events if e % ring == slot)

    def passes(completed, phase):
        return completed & 1 != phase & 1          # what a wait for a parity sees

    while todo:
        issued, landed, done, used, empty, makers = state = todo.pop()
        after = []
        if issued < stages and (issued < slots or issued - slots in empty):
            after.append((issued + 1, landed, done, used, empty, makers))
        for s in range(issued):
            if s not in landed:
                after.append((issued, landed | {s}, done, used, empty, makers))
        for s in range(done):
            if s not in used:
                after.append((issued, landed, done, used | {s}, empty, makers))
            if s not in empty:
                after.append((issued, landed, done, used, empty | {s}, makers))
        if done < stages and done in landed and makers[done % sets][0] > done:   # the issuing warp sees every phase of both rings
            after.append((issued, landed, done + 1, used, empty, makers))
        for k, (s, passed) in enumerate(makers):
            if s >= stages:
                continue
            room = (passed == 0) == room_first
            if room:
                may, right = passes(phases(used, made, s % made), s // made - 1), s < made or s - made in used
            else:
                may, right = passes(phases(landed, slots, s % slots), s // slots), s in landed
            if not may:
                continue
            if not right:
                return f"stage {s} passes its wait for {'room' if room else 'codes'} too early"
            after.append((issued, landed, done, used, empty, makers[:k] + ((s, 1) if passed == 0 else (s + sets, 0),) + makers[k + 1:]))
        if not after and done < stages:
            return f"nobody goes on after {done} products"
        for state in after:
            if state not in seen:
                seen.add(state)
                todo.append(state)
    return None


@pytest.mark.parametrize("bn", WIDTHS)
def test_a_set_never_passes_a_wait_too_early(bn):
    slots, made, sets, room_first = rings(bn)
    assert walk(slots, made, sets, room_first, max(slots + 3, 12)) is None


@pytest.mark.parametrize("bn,room_first,what", [(64, False, "codes"), (128, True, "room")])
def test_the_other_order_would_pass_too_early(bn, room_first, what):
    """The model sees the mistake where the ring that is not a set's own is waited for first."""
    slots, made, sets, right = rings(bn)
    assert right != room_first and what in walk(slots, made, sets, room_first, 9)


def test_the_model_sees_more_sets_than_slots():
    assert "codes" in walk(2, 3, 3, False, 9) and walk(4, 3, 3, True, 9) is None
