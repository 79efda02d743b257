"""CPU check of the window arithmetic of the decode kernel (no GPU).

The kernel streams the units (32 tokens of a bf16 cache, 64 of an e4m3 one)
that hold a token the query sees: the sinks' first, then, past a gap, the
window's.  This restates live_span, real_unit, live_block and the masks of
attend_unit, and checks against the definition that

  * the units listed are those with a visible token, once each, in order;
  * every block-table entry read is one of a live block of the unit;
  * a token passes the masks exactly if the query sees it, and a unit without
    a hidden token is not masked at all;
  * the host's bound on a sequence's units is never exceeded, nor met by more
    than two.

A kernel change to any of these must be mirrored here.
"""
import numpy as np
import pytest

BLOCK = 16


def span(ctx, window, n_sink, ut):
    lo = max(ctx - window, 0)
    first = lo // ut
    head = min(-(-n_sink // ut), first)
    return lo, head, first - head, -(-ctx // ut) - (first - head)


def live_block(lo, n_sink, j, b, nb, ub):
    first, wb = j * ub, lo // BLOCK
    blk = first + b
    seen = lambda x: x >= wb or x * BLOCK < n_sink  # noqa: E731
    return blk if blk < nb and seen(blk) else (first if seen(first) else wb)


def host_bound(max_ctx, window, n_sink, unit):
    return min(-(-max_ctx // unit), -(-n_sink // unit) + (window + unit - 2) // unit + 1)


@pytest.mark.parametrize("ut", [32, 64])
def test_units_blocks_and_masks(ut):
    rng = np.random.default_rng(ut)
    ub, nz = ut // BLOCK, ut // 4
    trials = [(1, 1, 0), (ut, ut, 0), (ut + 1, ut, 0), (ut + 1, 1, ut), (3 * ut, ut, ut + 1), (40 * ut, 1, 0)]
    trials += [(int(rng.integers(0, 900)), int(rng.integers(1, 400)), int(rng.choice([0, 1, 4, 15, 16, 17, 60, 300])))
               for _ in range(400)]
    for ctx, window, n_sink in trials:
        # (the host cuts both at the longest context)
        window, n_sink = min(window, max(ctx, 1)), min(n_sink, ctx)
        t = np.arange(ctx)
        see = (t >= ctx - window) | (t < n_sink)
        lo, head, gap, nus = span(ctx, window, n_sink, ut)
        units = [j + gap if j >= head else j for j in range(nus)]
        assert units == [u for u in range(-(-ctx // ut)) if see[u * ut:(u + 1) * ut].any()]
        assert nus <= host_bound(ctx, window, n_sink, ut)
        nb = -(-ctx // BLOCK)
        for u in units:
            for b in range(ub):
                blk = live_block(lo, n_sink, u, b, nb, ub)
                assert u * ub <= blk < min(nb, (u + 1) * ub) and see[blk * BLOCK:(blk + 1) * BLOCK].any()
                mine = see[(u * ub + b) * BLOCK:(u * ub + b + 1) * BLOCK]
                assert not mine.any() or blk == u * ub + b
            ragged = u * ut + ut > ctx or (u * ut < lo and u * ut + ut > n_sink)
            for lane in range(4):
                tok0 = u * ut + nz * lane
                first = lambda n: (1 << min(max(n - tok0, 0), nz)) - 1  # noqa: B023, E731
                live = first(ctx) & (~first(lo) | first(n_sink)) if ragged else (1 << nz) - 1
                want = sum(1 << e for e in range(nz) if tok0 + e < ctx and see[tok0 + e])
                assert live & ((1 << nz) - 1) == want


def test_host_bound_is_tight():
    worst = 0
    for window in range(1, 200):
        for ctx in range(window, window + 70):
            worst = max(worst, host_bound(ctx, window, 0, 32) - span(ctx, window, 0, 32)[3])
    assert worst <= 2
