"""CPU check of what V a wave of the windowed prefill kernel multiplies (no GPU).

A token that a column does not see has probability 0 there, and 0 times a value
that is not finite is not.  This restates which V tile a wave takes for each of
its steps, the last one's read behind the loop included (vtile), and what is
zeroed in the tiles for all waves (clip_v), and checks that a token's value
meets only columns within 62 positions of a row that sees it, and that the
copy of the tile with the last sink is made in every item where a wave reads it,
and that the steps that choose another V tile take the branch that does so.

A kernel change to any of these must be mirrored here.
"""
import numpy as np
import pytest

KT = 32


def v_of(t0, lo_first, n_sink, copied):
    """The tokens of the tile at t0 whose values a wave takes: its window's first token is lo_first."""
    if t0 + KT > lo_first or t0 + KT <= n_sink or t0 < n_sink and not copied:
        return t0, t0 + KT
    return t0, max(t0, n_sink)                    # a block of zeros, or the copy of the last sink's tile


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
        nt = -(-n_kv // st) - gap
        sink_t0 = n_sink // KT * KT
        last = T - n + tok_last - window + 1
        j_sink = n_sink // st if sink_t0 != n_sink and lo < sink_t0 + KT <= last else -1
        assert j_sink < 0 or j_sink < nt and real(j_sink) == n_sink // st
        for w in range(waves):
            ks, cg = w % s, w // s
            if c0 + cg * wave_cols >= ncols:
                continue
            pmin = T - n + min(c0 + cg * wave_cols, ncols - 1) // G
            p_end = T - n + (min(c0 + (cg + 1) * wave_cols, ncols) - 1) // G
            nt_w = 0 if p_end < KT * ks else frm((p_end - KT * ks) // st + 1)
            lo_last = p_end - window + 1
            j_left = frm(lo_last // st + s) if lo_last > 0 else 0
            # (the steps of tokens that some column's window has passed, which the masks ask for)
            assert j_left >= frm((max(lo_last, 0) + st - 1) // st)
            for j in range(nt_w):
                first, end = v_of(st * real(j) + KT * ks, pmin - window + 1, n_sink, j_sink >= 0)
                if end < first + KT:              # chosen in the branch for the steps before j_left, or behind the loop
                    assert j == nt_w - 1 or j + 1 < j_left
                if first < end < first + KT:
                    assert first == sink_t0 and j == j_sink
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
                       int(rng.choice([0, 1, 4, 31, 32, 40, 64, 77, 96, 192]))))
    trials += [(600, 600, 1, 100, k) for k in (1, 8, 33, 48, 63)]
    worst = max(furthest(T, n, G, min(window, T), min(n_sink, T), waves, nc, s)
                for T, n, G, window, n_sink in trials)
    assert 0 < worst <= 62
