"""Pins of the page-table oracle (not gpu): no page is lost or held twice, whatever
the lengths, and what is short goes to nobody behind it."""
import numpy as np

from oracle import pages as G


def test_pages_are_conserved():
    rng = np.random.default_rng(1)
    B, P, most, n_pages = 7, 4, 9, 30
    held, table, stack = [0] * B, [[-1] * most for _ in range(B)], list(range(n_pages))
    for _ in range(200):
        length = [int(x) for x in rng.integers(0, P * most + 1, B)]
        old = [row[:h] for row, h in zip(table, held)]
        granted = G.resize(length, held, table, stack, P)
        mine = [p for row, h in zip(table, held) for p in row[:h]]
        assert sorted(mine + stack) == list(range(n_pages))
        for b in range(B):
            need = -(-length[b] // P)
            assert held[b] == need if granted[b] else held[b] == len(old[b]) < need
            k = min(held[b], len(old[b]))
            assert table[b][:k] == old[b][:k] and all(x == -1 for x in table[b][held[b]:])


def test_a_short_pool_serves_in_order():
    held, table, stack = [0, 1, 0, 1], [[-1] * 4 for _ in range(4)], [5, 6, 7]
    table[1][0], table[3][0] = 8, 9
    granted = G.resize([2, 10, 2, 1], held, table, stack, 2)
    # one page for the first, then four for the second are not there: nothing for it, nor for the third
    assert granted == [1, 0, 0, 1] and held == [1, 1, 0, 1] and table[0][0] == 7 and stack == [5, 6]


def test_slots_packed_and_padded():
    table = [[3, 1], [0, 2]]
    s, p, q, start = G.slot_map([3, 0], [2, 1], 5, 4, table)
    assert s == [15, 4, 0, -1, -1] and p == [3, 4, 0, 0, 0] and q == [0, 0, 1, -1, -1] and start == [0, 2, 3]
    s, p, q, _ = G.slot_map([3, 0], [2, 1], 6, 8, None, 3)
    assert s == [3, 4, -1, 8, -1, -1] and q == [0, 0, -1, 1, -1, -1]
