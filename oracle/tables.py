"""Block tables, slots and tree masks of one step, one request after the other.

Test infrastructure only (see the package header).

What is computed.  Blocks are handed out on demand (Sec. 3, effect 1) from a
ring of free ids; this restates the library's rule as a scheduler on the host
would run it: sequences in batch order; one that is over gives its blocks back
behind the free ids; one that grows takes the blocks it lacks from the ring's
head, unless they do not fit its table, its rows do not fit the batch, its
tree is too large for the masks, or the ring cannot cover the needs so far
(its own included; from then on only sequences that need nothing are served).
The paper has no formula for this; the rule is the library's.

Parity: pinned by hand-worked steps, by the host allocator of the library
(the same ids in the same order for a pool's first batch), and by invariants
(no block owned twice, blocks conserved) over a run of many random steps.
"""
from __future__ import annotations

import numpy as np

BS = 16


def step(ctx, owned, new, ring, head, count, tables, total_rows, parents=None, words=0):
    """Returns a dict of the outputs; the inputs are not changed.

    ctx, owned, new : int [B];  ring : int [num_blocks];  tables : int [B, max_blocks]
    parents : int [total_rows] or None;  words : 64-bit words of a mask row
    """
    ring, tables = np.array(ring, copy=True), np.array(tables, copy=True)
    nb, cap = len(ring), tables.shape[1] * BS
    B = len(ctx)
    out = dict(ctx=[], owned=[], granted=[], q_start=[0],
               slots=np.full(total_rows, -1, np.int64), positions=np.full(total_rows, -1, np.int32),
               mask=np.zeros((total_rows, max(words, 1)), np.uint64))
    want_so_far = took = gave = rows = 0
    for s in range(B):
        c, x = int(ctx[s]), int(new[s])
        b = max(int(owned[s]), -(-c // BS))
        if x < 0:
            for j in range(b):
                ring[(head + count + gave) % nb] = tables[s, j]
                gave += 1
            out["ctx"].append(0)
            out["owned"].append(0)
            out["granted"].append(1)
            out["q_start"].append(min(rows, total_rows))
            continue
        ok = c + x <= cap and rows + x <= total_rows and not (parents is not None and x > 64 * words)
        need = max(0, -(-(c + x) // BS) - b) if ok and x > 0 else 0
        want_so_far += need
        if need > 0 and want_so_far > count:
            ok = False
        if ok:
            for j in range(need):
                tables[s, b + j] = ring[(head + took) % nb]
                took += 1
        for i in range(min(x, max(total_rows - rows, 0))):
            t, r = c + i, rows + i
            out["positions"][r] = t
            if ok and tables[s, t // BS] >= 0:     # (an entry below 0 is no block)
                out["slots"][r] = int(tables[s, t // BS]) * BS + t % BS
            if parents is not None and min(rows + x, total_rows) - rows <= 64 * words:
                depth, at = 0, i
                while True:
                    out["mask"][r, at // 64] |= np.uint64(1 << (at % 64))
                    p = int(parents[rows + at])
                    if p < 0 or p >= at:
                        break
                    at, depth = p, depth + 1
                out["positions"][r] = c + depth
        rows += x
        out["q_start"].append(min(rows, total_rows))
        out["granted"].append(int(ok))
        out["ctx"].append(c + x if ok else c)
        out["owned"].append(b + need if ok else b)
    for k in ("ctx", "owned", "granted", "q_start"):
        out[k] = np.array(out[k], np.int32)
    return dict(out, ring=ring, tables=tables, state=np.array([(head + took) % nb, count - took + gave], np.int32))
