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
    than two;
  * where a segment is one workgroup's, its eight waves take every unit once, at
    most three each;
  * where segments are laid apart, every slice is part of one segment, the
    slices of a segment belong to one workgroup (to two, where they are eight),
    those in use have a unit each, and together they take every unit once;
  * the prefill kernel's items: their steps hold every token that one of their
    rows sees, block ids are staged for those alone and from entries of blocks
    that a row sees, a wave calls a tile hidden exactly if none of its columns
    sees it, the masking branch runs wherever a token is hidden from a column,
    and V is zeroed exactly where no row of the item sees it.

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


def lay_apart(nus, hkv, groups, waves, min_chunk, most):
    """(units of a slice, log2 of the slices of a segment, slices in use), zeros for equal slices."""
    live = [n for n in nus if n > 0]
    segs, c = hkv * len(live), max(-(-hkv * sum(nus) // (groups * waves)), min_chunk)
    if not live or segs > groups * waves:
        return 0, 0, 0
    lg = min((groups * waves // segs).bit_length() - 1, 3)
    slice_ = (max(live) + (1 << lg) - 1) >> lg
    last = (max(live) - 1) // slice_
    if min(live) > slice_ * last and slice_ >= min_chunk and slice_ <= min(c + 1 + (c >> 4), most):
        return slice_, lg, last + 1
    return 0, 0, 0


def test_segments_apart():
    rng = np.random.default_rng(3)
    waves, most, seen = 4, 256, [0, 0, 0, 0]
    for _ in range(3000):
        hkv, groups = int(rng.integers(1, 9)), int(rng.choice([1, 3, 16, 64, 256]))
        base, spread = int(rng.integers(1, 80)), int(rng.integers(0, 8))
        nus = [int(x) for x in rng.integers(max(base - spread, 1), base + 1, int(rng.integers(1, 80)))]
        nus = [0 if rng.random() < 0.1 else n for n in nus]
        c, lg, used = lay_apart(nus, hkv, groups, waves, int(rng.choice([1, 1, 2, 8])), most)
        if c == 0:
            continue
        seen[lg] += 1
        pre = np.concatenate([[0], np.cumsum([c << lg if n else 0 for n in nus])])
        total = hkv * int(pre[-1])
        assert c <= most and total <= groups * waves * c
        took = {}
        for gw in range(groups * waves):
            u0, u1 = gw * c, min(gw * c + c, total)
            if u0 >= u1 or gw % (1 << lg) >= used:
                continue
            s = max(i for i in range(len(nus)) if hkv * pre[i] <= u0)
            vnus = int(pre[s + 1] - pre[s])
            g, j = divmod(u0 - hkv * int(pre[s]), vnus)
            n = min(u1 - u0, nus[s] - j)
            assert n >= 1 and u1 - u0 == c and g < hkv
            took.setdefault((s, g), []).append((gw, range(j, j + n)))
        assert sorted(took) == [(s, g) for s in range(len(nus)) for g in range(hkv) if nus[s]]
        for (s, g), parts in took.items():
            assert [j for _, r in parts for j in r] == list(range(nus[s]))
            a0 = hkv * int(pre[s]) + g * (c << lg)
            k0, kend = a0 // c, (a0 + used * c - 1) // c
            assert [gw for gw, _ in parts] == list(range(k0, kend + 1)) and a0 == k0 * c
            assert kend // waves - k0 // waves <= (1 if lg == 3 else 0)
    assert min(seen) > 20, seen


def test_whole_segments():
    for nus in range(0, 25):
        mine = []
        for w in range(8):
            n = (nus - w - 1) // 8 + 1 if w < nus else 0
            assert n <= 3
            mine += [w + 8 * k for k in range(n)]
        assert sorted(mine) == list(range(nus))


@pytest.mark.parametrize("waves,nc,s", [(8, 2, 1), (4, 2, 1), (8, 1, 2), (8, 2, 2), (4, 1, 1)])
def test_prefill_items(waves, nc, s):
    rng = np.random.default_rng(waves + nc + s)
    wave_cols = 16 * nc
    cols, kt = wave_cols * waves // s, 32
    st = kt * s
    trunc = lambda a, b: int(a / b)  # noqa: E731  (C++ division)
    trials = [(1, 1, 1, 1, 0), (33, 33, 8, 32, 1), (700, 300, 1, 64, 70), (700, 300, 16, 1, 0), (130, 2, 5, 9, 64)]
    for _ in range(60):
        T = int(rng.integers(1, 900))
        trials.append((T, int(rng.integers(1, T + 1)), int(rng.choice([1, 2, 5, 8, 16])), int(rng.integers(1, 500)),
                       int(rng.choice([0, 1, 4, 20, 64, 200]))))
    for T, n, G, window, n_sink in trials:
        window, n_sink = min(window, T), min(n_sink, T)
        t = np.arange(-(-T // st) * st + st)
        ncols, nb = n * G, -(-T // 16)
        for qt in range(-(-ncols // cols)):
            c0 = qt * cols
            tok_last = (min(c0 + cols, ncols) - 1) // G
            n_kv = T - n + tok_last + 1
            lo = max(T - n + c0 // G - window + 1, 0)
            head = min(-(-n_sink // st), lo // st)
            gap = lo // st - head
            real = lambda j: j + gap if j >= head else j  # noqa: B023, E731
            frm = lambda r: r if r <= head else max(r - gap, head)  # noqa: B023, E731
            nt = -(-n_kv // st) - gap
            rows = np.arange(T - n + c0 // G, T - n + tok_last + 1)[:, None]
            see = (t <= rows) & ((t > rows - window) | (t < n_sink))
            steps = [real(j) for j in range(nt)]
            assert steps == [r for r in range(len(t) // st) if see[:, r * st:(r + 1) * st].any()]
            n_ids = min(2 * s * nt, nb - 2 * s * gap)
            assert n_ids >= 1
            rows_all = np.arange(T - n, T)[:, None]
            some = ((t <= rows_all) & ((t > rows_all - window) | (t < n_sink))).any(0)
            for i in range(n_ids):
                b = i + 2 * s * gap if i >= 2 * s * head else i
                e = lo // 16 if b * 16 >= n_sink and b * 16 + 16 <= lo else b
                assert b // (2 * s) == real(i // (2 * s)) and 0 <= e < nb and some[e * 16:e * 16 + 16].any()
            for j in range(nt):   # what is zeroed in V: hidden from every row of the item, but for causality
                x = t[real(j) * st:(real(j) + 1) * st]
                cut = ((x >= n_sink) & (x < lo)) | (x >= T)
                if real(j) * st < lo and real(j) * st + st > n_sink or real(j) * st + st > T:
                    assert not see[:, x[cut]].any()
                else:
                    assert not cut.any()
            for w in range(waves):
                ks, cg = w % s, w // s
                if c0 + cg * wave_cols >= ncols:
                    continue
                pmin = T - n + min(c0 + cg * wave_cols, ncols - 1) // G
                p_end = T - n + (min(c0 + (cg + 1) * wave_cols, ncols) - 1) // G
                nt_w = 0 if p_end < kt * ks else frm((p_end - kt * ks) // st + 1)
                lo_first, lo_last = pmin - window + 1, p_end - window + 1
                j_rare = frm(min(trunc(pmin + 1 - kt * ks, st), T // st))
                j_left = frm((max(lo_last, 0) + st - 1) // st)
                p = np.arange(pmin, p_end + 1)[:, None]
                for j in range(nt):
                    t0 = st * real(j) + kt * ks
                    x = t[t0:t0 + kt]
                    mine = (x <= p) & ((x > p - window) | (x < n_sink))
                    past = t0 > p_end
                    assert not mine.any() or j < nt_w
                    if j >= nt_w:
                        continue
                    hidden = t0 + kt <= lo_first and t0 >= n_sink
                    assert past or hidden == (not mine.any())
                    if not mine.all():
                        assert j >= j_rare or j < j_left
                        assert t0 + kt - 1 > pmin or (t0 < lo_last and t0 + kt > n_sink)
                    if st * real(j) < lo and st * real(j) + st > n_sink or st * real(j) + st > T:
                        assert j >= j_rare or j < j_left       # (the wave's part of V is zeroed there)


def test_host_bound_is_tight():
    worst = 0
    for window in range(1, 200):
        for ctx in range(window, window + 70):
            worst = max(worst, host_bound(ctx, window, 0, 32) - span(ctx, window, 0, 32)[3])
    assert worst <= 2


def test_few_rows_workgroups():
    """The workgroups of few rows: every (token, head) column once, none past the host's bound."""
    rng = np.random.default_rng(3)
    for _ in range(300):
        batch, G, hkv = int(rng.integers(1, 65)), int(rng.choice([1, 2, 5, 8, 16, 40])), 3
        T = rng.integers(0, 50, batch)
        asked = rng.integers(0, 6, batch)
        total_q = int(asked.sum())
        n = np.minimum(asked, T)                       # (rows past the tokens have no columns)
        groups = (total_q * G + 15 * batch) // 16 * hkv
        cnt = -(-(n * G) // 16)
        incl = np.cumsum(cnt)
        seen = set()
        for b in range(groups):
            item, g = b // hkv, b % hkv
            past = np.flatnonzero(incl > item)
            if len(past) == 0:
                continue
            s = int(past[0])
            col0 = 16 * (item - int(incl[s] - cnt[s]))
            cols = min(int(n[s]) * G - col0, 16)
            assert cols >= 1
            last = (col0 + cols - 1) // G
            ctx, rows = int(T[s]) - int(n[s]) + last + 1, last - col0 // G + 1
            for c in range(16):
                cc = col0 + min(c, cols - 1)
                tok = cc // G - col0 // G
                assert 0 <= tok < rows and ctx - rows + 1 + tok == int(T[s]) - int(n[s]) + cc // G + 1
                if c < cols:
                    key = (s, cc // G, g * G + cc % G)
                    assert key not in seen
                    seen.add(key)
        assert len(seen) == int(n.sum()) * G * hkv
