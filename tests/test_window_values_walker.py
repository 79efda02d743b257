"""CPU check of what V a wave of the windowed prefill kernel multiplies (no GPU).

A token that a column does not see has probability 0 there, and 0 times a value
that is not finite is not.  This restates which V tile a wave takes for each of
its steps, the last one's read behind the loop included (vtile), and what is
zeroed in the tiles for all waves (clip_v), and checks that a token's value
meets only columns within 62 positions of a row that sees it.

A kernel change to any of these must be mirrored here.
"""
import numpy as np
import pytest

KT = 32


def v_of(t0, lo_first, n_sink):
    """The tokens of the tile at t0 whose values a wave takes: its window's first token is lo_first."""
    if t0 + KT <= lo_first and t0 >= n_sink:      # hidden: a block of zeros
        return t0, t0
    return t0, t0 + KT


def furthest(T, n, G, window, n_sink, waves, nc, s):
    """The largest distance of a column from the rows that see a token whose value it meets."""
    cols, wave_cols, st = 16 * nc * waves // s, 16 * nc, KT * s
    ncols, worst = n * G, 0
    for c0 in range(0, ncols, cols):
        tok_last = (min(c0 + cols, ncols) - 1) // G
        n_kv = T - n + tok_last + 1
        lo = max(T - n + c0 // G - window + 1, 0)
        head = min(-(-n_sink // st), lo // st)
        gap = lo // st - head
        real = lambda j: j + gap if j >= head else j  # noqa: B023, E731
        frm = lambda r: r if r <= head else max(r - gap, head)  # noqa: B023, E731
        assert -(-n_kv // st) - gap > 0
        for w in range(waves):
            ks, cg = w % s, w // s
            if c0 + cg * wave_cols >= ncols:
                continue
            pmin = T - n + min(c0 + cg * wave_cols, ncols - 1) // G
            p_end = T - n + (min(c0 + (cg + 1) * wave_cols, ncols) - 1) // G
            nt_w = 0 if p_end < KT * ks else frm((p_end - KT * ks) // st + 1)
            for j in range(nt_w):
                first, end = v_of(st * real(j) + KT * ks, pmin - window + 1, n_sink)
                for x in range(first, min(end, T)):
                    if n_sink <= x < lo:
                        continue                  # zero in the tile
                    sees = (max(x, T - n), T - 1 if x < n_sink else min(x + window - 1, T - 1))
                    assert sees[0] <= sees[1]
                    worst = max(worst, sees[0] - pmin, p_end - sees[1])
    return worst


ITEMS = [(8, 2, 1), (4, 2, 1), (8, 1, 2), (8, 2, 2), (4, 1, 1)]


@pytest.mark.parametrize("waves,nc,s", ITEMS)
def test_values_stay_near(waves, nc, s):
    rng = np.random.default_rng(waves + nc + s)
    trials = [(384 + 300, 300, 1, 1, 192), (384 + 300, 300, 1, 2, 192), (900, 600, 1, 100, 0), (700, 700, 1, 33, 32)]
    for _ in range(40):
        T = int(rng.integers(1, 900))
        trials.append((T, int(rng.integers(1, T + 1)), int(rng.choice([1, 2, 8])), int(rng.integers(1, 300)),
                       int(rng.choice([0, 32, 64, 96, 192]))))
    worst = max(furthest(T, n, G, min(window, T), min(n_sink, T // KT * KT), waves, nc, s)
                for T, n, G, window, n_sink in trials)
    assert 0 < worst <= 62
