"""Pins of the plain eviction where slots have no page, and of its form for long units."""
import numpy as np

from oracle import paged
from paged_harness import evict_sources


def test_eviction_by_hand_where_slots_have_no_page():
    #      slot:  0    1    2    3    4    5    6    7
    weight = [1.0, 9.0, 2.0, 3.0, 4.0, 5.0, 0.5, 8.0]
    pos = [0, 1, 2, 3, 4, 5, 6, 7]

    def moves(gone, budget, sink=0, recent=0):
        return paged.evict_moves(pos, weight, 8, budget, sink, recent, [j not in gone for j in range(8)])
    # slot 1 cannot take a row: three places for the best three of the others, 7 (8.0), 5 and 4
    assert moves({1}, 4) == (4, [(0, 4), (2, 5), (3, 7)])
    # the heaviest above n' is not there
    assert moves({7}, 4) == (4, [(0, 4), (2, 5)])
    # a missing slot is protected by nothing, whatever its position: the sink is slot 1's 0 .. 1, without slot 0
    assert moves({0}, 3, sink=2) == (3, [(2, 7)])
    assert moves({0, 1, 2}, 3) == (3, []) and moves(set(range(8)), 5) == (5, []) and moves({6, 7}, 6) == (6, [])
    assert moves(set(), 4) == (4, [(0, 4), (2, 5), (3, 7)])


def test_the_form_for_long_units_is_the_same():
    rng = np.random.default_rng(5)
    for i in range(300):
        n = int(rng.integers(1, 60))
        pos = rng.permutation(n + 5)[:n] if i % 2 else rng.integers(0, 6, n)
        weight = rng.choice(np.array([np.nan, np.inf, -np.inf, 0.0, -0.0, 1.0, 2.0, 2.5], np.float32), n)
        there = rng.random(n) < (1.0, 0.8, 0.2, 0.0)[i % 4]
        budget, sink, recent = int(rng.integers(-1, n + 3)), int(rng.integers(0, 4)), int(rng.integers(0, 9))
        stay, moves = paged.evict_moves(pos, weight, n + 3, budget, sink, recent, there)
        want = np.arange(stay)
        for to, at in moves:
            want[to] = at
        np.testing.assert_array_equal(evict_sources(pos, weight, n + 3, budget, sink, recent, there), want)
        if there.all():
            assert paged.evict_moves(pos, weight, n + 3, budget, sink, recent) == (stay, moves)
