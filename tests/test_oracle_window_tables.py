"""Pins of the block-table oracle where sequences that end (with -2) have entries that hold no block."""
import numpy as np

from oracle import tables


def test_entries_below_0_hold_no_block():
    tb = np.array([[-1, 5, -1, 9], [-1, -7, -1, -1], [3, 1, -1, -1], [-1, 8, 2, -1]])
    ring = np.array([-5, -5, 4, 7, -5, -5, -5, -5, -5, -5])
    o = tables.step([60, 33, 20, 33], [4, 3, 2, 3], [-2, -9, 13, -2], ring, 2, 2, tb, 14)
    assert o["ring"].tolist() == [-5, -5, 4, 7, 5, 9, 8, 2, -5, -5]
    assert o["state"].tolist() == [3, 5] and o["tables"][2].tolist() == [3, 1, 4, -1]
    assert o["owned"].tolist() == [0, 0, 3, 0] and o["granted"].tolist() == [1, 1, 1, 1]
    assert o["slots"].tolist() == [16 + 4 + i for i in range(12)] + [64, -1]


def test_blocks_are_conserved_when_they_leave_windows():
    """Random steps with a window of 40 tokens behind 5 that stay: no block owned twice, none lost."""
    rng = np.random.default_rng(0)
    B, mb, nb, window, n_sink = 6, 60, 40, 40, 5
    ctx, owned, tb = np.zeros(B, int), np.zeros(B, int), np.full((B, mb), -1)
    ring, head, count = rng.permutation(nb), 3, nb
    over = 0
    for _ in range(300):
        new = np.where(rng.random(B) < 0.05, -2, rng.integers(0, 25, B))
        over += int(((new < 0) & (ctx > 200)).sum())
        o = tables.step(ctx, owned, new, ring, head, count, tb, 200)
        ctx, owned, ring, tb = o["ctx"], o["owned"], o["ring"], o["tables"]
        head, count = o["state"].tolist()
        tb[new < 0] = -1
        for s in range(B):
            for j in range(mb):
                if tb[s, j] >= 0 and 16 * j >= n_sink and 16 * j + 16 <= ctx[s] + 1 - window:
                    ring[(head + count) % nb] = tb[s, j]
                    count += 1
                    tb[s, j] = -1
        held = [tb[s, j] for s in range(B) for j in range(owned[s]) if tb[s, j] >= 0]
        free = [ring[(head + i) % nb] for i in range(count)]
        assert sorted(held + free) == list(range(nb))
    assert over > 20
