"""The number of row tiles that a ragged attention launches (csrc/ragged_plan.h, compiled): the tiles of every request lie
below it, wherever its rows begin, for every kernel that the plan can choose."""
import random

from ragged_plans import plan


def test_the_tiles_that_are_launched_hold_every_row():
    rng = random.Random(18)
    seen = {16: 0, 32: 0, 128: 0}
    for _ in range(6000):
        Hkv, G, R = rng.choice([1, 2, 5]), rng.choice([1, 2, 3, 8, 40]), rng.randint(1, 40)
        T = rng.randint(1, rng.choice([2 * R, 20 * R, 700]))
        p = plan(R, T, Hkv * G, Hkv, rng.choice([64, 128]), rng.choice([0, 100, 5000]))
        rows, tiles = p["rows"], p["tiles"]
        seen[rows] += 1
        cuts = sorted(rng.randint(0, T) for _ in range(R + 1))
        if rng.random() < 0.5:
            cuts[0], cuts[-1] = 0, T
        if rng.random() < 0.3:  # all of the rows in the last request, the worst place
            cuts = [rng.choice([0, cuts[0]])] * R + [T]
        first = [c * G // rows + r for r, c in enumerate(cuts[:-1])]
        last = [f + -(-(b - a) * G // rows) - 1 for f, a, b in zip(first, cuts, cuts[1:])]
        assert all(x < y for x, y in zip(last, first[1:]))
        assert max(last) < tiles, (R, T, G, rows, cuts)
        assert tiles <= -(-T * G // rows) + R  # and none in excess of what odd starts need
    assert min(seen.values()) > 300, seen
