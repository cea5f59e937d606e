"""The ring of the mma.sync attention kernel, every interleaving of its barriers on the CPU.

A barrier is waited for by the parity of a phase: the wait passes while the barrier's current phase has the other parity.  That is
sound only where the barrier is in the phase waited for or the one after it; a barrier that has run two phases on reads as open.
The producer fills stages (after the stage's release before) and, at a unit's end, hands one over for the join of the warps' sums.
"""

import os

import pytest

SOURCE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2604_13634_b200", "csrc", "csd_attention.cuh")


def explore(n_stages, units, consumers, join_waits):
    """Unit lengths in tiles -> the first bad state found: a step that passed a wait in a wrong phase, or nobody able to go on."""
    items, k = [], 0
    for tiles in units:
        for what in ["tile"] * tiles + ["join"]:
            items.append((what, k % n_stages, k // n_stages))
            k += 1
    producer = [step for what, s, rnd in items for step in (("wait", "empty", s, rnd - 1), ("arrive", "full", s, 1))]
    consumer = []
    for what, s, rnd in items:
        if what == "tile" or join_waits:
            consumer.append(("wait", "full", s, rnd))
        if what == "join":
            consumer.append(("meet",))                            # the barrier of the consumers among themselves
        consumer.append(("arrive", "empty", s, consumers))
    programs = [producer] + [consumer] * consumers
    start = ((0,) * len(programs), (((0, 0),) * n_stages,) * 2)      # (steps taken), (phase, arrivals) of full and empty
    todo, known = [start], {start}
    while todo:
        at, bars = todo.pop()
        follows = []
        for i, prog in enumerate(programs):
            if at[i] == len(prog):
                continue
            step = prog[at[i]]
            moved = list(at)
            moved[i] += 1
            if step[0] == "wait":
                phase = bars[step[1] == "empty"][step[2]][0]
                if phase % 2 == step[3] % 2:
                    continue                                      # by parity: not yet
                if phase != step[3] + 1:
                    return "early", at
                follows.append((tuple(moved), bars))
            elif step[0] == "meet":
                if any(at[j] < at[i] for j in range(1, len(programs))):
                    continue                                      # all of them come here before any goes on
                follows.append((tuple(moved), bars))
            else:
                kind = int(step[1] == "empty")
                row = list(bars[kind])
                phase, count = row[step[2]]
                row[step[2]] = (phase + 1, 0) if count + 1 == step[3] else (phase, count + 1)
                new = list(bars)
                new[kind] = tuple(row)
                follows.append((tuple(moved), tuple(new)))
        if not follows and any(at[i] < len(prog) for i, prog in enumerate(programs)):
            return "stuck", at
        for state in follows:
            if state not in known:
                known.add(state)
                todo.append(state)
    return None


RINGS = [(3, [1, 1, 1, 1, 1, 1], 2), (3, [2, 4, 1, 3], 2), (2, [1, 3, 2, 1], 3), (4, [5, 1, 2], 2), (7, [3, 9, 1], 2)]


@pytest.mark.parametrize("n_stages,units,consumers", RINGS)
def test_every_wait_is_in_its_phase_and_every_order_ends(n_stages, units, consumers):
    with open(SOURCE) as f:
        after_tiles = f.read().split("the warps' sums meet in the next stage", 1)[1]
    waits = "mbar_wait(full_k(at_ring.slot), at_ring.round, give_up);" in after_tiles.split("float *sums", 1)[0]
    assert explore(n_stages, units, consumers, join_waits=waits) is None


def test_a_join_stage_taken_without_a_wait_can_stop_the_producer():
    assert explore(3, [1, 1, 1, 1, 1, 1], 2, join_waits=False) is not None
