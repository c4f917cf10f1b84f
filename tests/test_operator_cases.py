"""The drawn performance cases of the 4-bit cache stay inside their caches: sizes only, on the CPU."""
import random

import pytest

import perf.operators as M


@pytest.mark.parametrize("seed", range(10))
def test_appended_rows_have_slots(seed):
    """The plain form writes every appended row where it is told to."""
    rng, seen = random.Random(seed), 0
    cases = M.listed() + [M.draw(rng) for _ in range(300)]
    cases.append(M._case("", "step", 3, 2, 2, 64, 128, 116, pad=True, weight=True))
    for i, c in enumerate(cases):
        if c["kind"] in ("append", "step"):
            lengths, counts = M._host_lengths(c, seed + i)
            start = lengths - counts
            assert int(start.min()) >= 0 and int(start.max()) + c["Lq"] <= M._slots(c), c
            assert int(lengths.max()) <= M._slots(c), c
            seen += 1
    assert seen > 50
