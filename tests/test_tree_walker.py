"""CPU check of the tree attention's index arithmetic (tree_walk.py): who computes and writes what, on random batches."""
import numpy as np
import pytest

import tree_walk


def owners(q_start, ctx, total_q, hq, hkv, max_ctx, words, fp8):
    """Every tile of every item is taken once and joined from where it was left; {(row, KV head): its sequence}"""
    cols, wgs = tree_walk.walk(q_start, ctx, total_q, hq, hkv, max_ctx, words, fp8, cus=16)
    group = hq // hkv
    seqs = tree_walk.rows(q_start, ctx, total_q, max_ctx, words)
    tiles, records, starts, who = {}, set(), {}, {}
    for pieces in wgs:
        for p in pieces:
            assert 0 <= p.r0 and p.r0 + p.n <= total_q and 0 < p.n <= min(p.T, 64 * words) and 0 <= p.g < hkv
            assert p.c0 < p.n * group and 0 <= p.j0 < p.j1 <= p.nt == -(-p.T // (64 if fp8 else 32))
            for j in range(p.j0, p.j1):
                assert tiles.setdefault((p.s, p.g, p.c0, j), p.wg) == p.wg
            if not p.whole:
                slot = 2 * p.wg + (p.j0 == 0)
                assert slot not in records and slot < 2 * len(wgs)
                records.add(slot)
                if p.j0 == 0:
                    starts[p.wg] = p
            for c in range(p.c0, min(p.c0 + cols, p.n * group), group):
                who.setdefault((p.r0 + c // group, p.g), set()).add(p.s)
    n_items = sum(-(-n * group // cols) * hkv for _, n, _ in seqs)
    assert len({k[:3] for k in tiles}) == n_items
    assert len(tiles) == sum(-(-n * group // cols) * hkv * -(-T // (64 if fp8 else 32)) for _, n, T in seqs)
    for wg, p in starts.items():   # the join reads the start's record and those of all workgroups up to the last
        assert wg < p.last < len(wgs)
        for k in range(wg + 1, p.last + 1):
            assert 2 * k in records and any((x.s, x.g, x.c0) == (p.s, p.g, p.c0) for x in wgs[k][:1])
    assert len(records) == len(starts) + sum(p.last - wg for wg, p in starts.items())
    return who


@pytest.mark.parametrize("seed", range(30))
def test_every_tile_is_taken_once(seed):
    rng = np.random.default_rng(seed)
    hkv, group, words = int(rng.integers(1, 5)), int(rng.choice([1, 2, 5, 8, 16])), int(rng.integers(1, 3))
    ctx = np.exp(rng.uniform(0, np.log(3000), int(rng.integers(1, 30)))).astype(int)
    new = np.minimum(rng.integers(0, 40 * words, len(ctx)), ctx)
    q_start = np.concatenate([[0], np.cumsum(new)]).tolist()
    who = owners(q_start, ctx.tolist(), q_start[-1] + 3, hkv * group, hkv, 4096, words, bool(seed % 2))
    assert len(who) == q_start[-1] * hkv and all(len(s) == 1 for s in who.values())


@pytest.mark.parametrize("q_start,ctx,total", [
    ([0, 5, -3, 10 ** 9], [40, 30, 70], 17), ([7, 3, 9, 2, 12], [20, 20, 20, 20], 12),
    ([-2 ** 31, 2 ** 31 - 1, 0, 5, 4], [9, 9, 9, 9], 6), ([4, 0, 8], [30, 30], 8)])
def test_rows_have_one_owner_whatever_the_offsets(q_start, ctx, total):
    """Offsets out of order or range: no two sequences write the same rows."""
    who = owners(q_start, ctx, total, 8, 2, 80, 1, False)
    assert all(len(s) == 1 for s in who.values())
    assert all(0 <= r < total for r, _ in who)
