"""The barriers between k_linear_tc's two expanding teams and the warp that issues its MMAs.

Every interleaving of the three is gone through for a few tiles, with phases and parities
as the hardware counts them: an MMA may only read codes that its stage's teams have
written.  A part of an odd number of 128-column blocks ends in half a stage, for which the
second team writes nothing and only arrives; whether it waits for the slot before that is
read from the source.
"""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_06291_gb300", "csrc")
ND = 4     # barriers of "the stage's MMAs are done"


def _half_stage_waits():
    """Whether the team that has nothing to write waits for the slot before it arrives."""
    with open(os.path.join(CSRC, "linear_tc.cu")) as f:
        source = re.sub(r"//[^\n]*", "", f.read())
    at = source.index("if (S::X8 && kb + team >= kb1)")
    arrive = source.index("mbar_arrive(&aF[sa])", at)
    return re.search(r"ia >= S::NA && !wait_stage\(ia - S::NA\)", source[at:arrive]) is not None


def _explore(stages, slots, waits):
    """Goes through every order of events.  stages: True where the second team has its half.
    Returns the first fault found, or None; stuck states are faults too."""
    total = len(stages)
    # a team: (stage, written and not yet arrived); aF: (arrivals of the phase, phases over) a slot;
    # issued and complete stages; the teams' writes are done in order, so `reach` tells them
    start = ((0, False), (0, False), tuple((0, 0) for _ in range(slots)), 0, 0)
    seen, todo = {start}, [start]
    while todo:
        *teams, aF, issued, complete = todo.pop()

        def stage_done(j):      # wait_stage(j): parity (j / ND) & 1 on barrier j % ND
            over = (complete - 1 - j % ND) // ND + 1 if complete > j % ND else 0
            return over & 1 != (j // ND) & 1

        after = []
        for t in (0, 1):
            stage, written = teams[t]
            if stage == total:
                continue
            mine = t == 0 or stages[stage]
            if not written:
                if (mine or waits) and stage >= slots and not stage_done(stage - slots):
                    continue
                move, bars = (stage, True), aF
            else:
                count, over = aF[stage % slots]
                count += 1
                bars = list(aF)
                bars[stage % slots] = (0, over + 1) if count == 2 else (count, over)
                move, bars = (stage + 1, False), tuple(bars)
            two = list(teams)
            two[t] = move
            after.append((two[0], two[1], bars, issued, complete))
        if issued < total and aF[issued % slots][1] & 1 != (issued // slots) & 1:
            for t in (0, 1):
                stage, written = teams[t]
                if (t == 0 or stages[issued]) and not (stage > issued or (stage == issued and written)):
                    return f"stage {issued} is multiplied before team {t} has written it"
            after.append((*teams, aF, issued + 1, complete))
        if complete < issued:
            after.append((*teams, aF, issued, complete + 1))
        if not after and complete < total:
            return f"stuck with {complete} of {total} stages complete"
        for s in after:
            if s not in seen:
                seen.add(s)
                todo.append(s)
    return None


TILES = [[False] * 12, [True, False] * 5, [True, True, False] * 4, [True] * 5 + [False] + [True] * 5 + [False],
         [True] * 12]


@pytest.mark.parametrize("slots", [2, 4])
@pytest.mark.parametrize("stages", TILES)
def test_no_codes_are_multiplied_before_they_are_written(slots, stages):
    assert _explore(stages, slots, _half_stage_waits()) is None


@pytest.mark.parametrize("slots", [2, 4])
@pytest.mark.parametrize("stages", TILES[:-1])
def test_the_model_sees_an_arrival_without_the_wait(slots, stages):
    assert _explore(stages, slots, False) is not None
