"""The index arithmetic of the tree attention, restated step for step as its launcher and kernel do it (CPU only).

plan() is the launcher's choice of columns and workgroups, rows() how a
sequence's rows follow from q_start, walk() the pieces that every workgroup
takes, run() which of their tiles are handed over or loaded anew.  A change of
the kernel to any of these must be mirrored here.
"""
from __future__ import annotations

from dataclasses import dataclass

ITEM_COST, MIN_SLICE, CHUNK = 4, 4, 56


@dataclass
class Piece:
    wg: int
    s: int
    g: int
    c0: int
    j0: int
    j1: int
    nt: int
    r0: int
    n: int
    T: int
    last: int        # the workgroup with the item's last piece

    @property
    def whole(self):
        return self.j0 == 0 and self.j1 == self.nt


def plan(batch, total_q, group, cus=256):
    """(columns of an item, workgroups)"""
    per_seq = (total_q * group + max(batch, 1) - 1) // max(batch, 1)
    if per_seq <= 64:
        return 64, 2 * cus
    return (128, 2 * cus) if per_seq <= 128 else (256, cus)


def rows(q_start, context_lens, total_q, max_ctx, words):
    """(first row, rows, cached tokens) of every sequence; offsets out of order count as the largest so far."""
    out = []
    r1 = min(max(q_start[0], 0), total_q)
    for s in range(len(context_lens)):
        r0 = r1
        r1 = min(max(q_start[s + 1], r0), total_q)
        T = min(max(context_lens[s], 0), max_ctx)
        out.append((r0, min(r1 - r0, T, 64 * words), T))
    return out


def walk(q_start, context_lens, total_q, hq, hkv, max_ctx, words, fp8, cus=256):
    """(columns, [pieces of workgroup 0, of workgroup 1, ...])"""
    group, kt = hq // hkv, 64 if fp8 else 32
    cols, nwg = plan(len(context_lens), total_q, group, cus)
    seqs = rows(q_start, context_lens, total_q, max_ctx, words)
    units = [-(-T // kt) + ITEM_COST for _, _, T in seqs]
    items = [-(-n * group // cols) * hkv for _, n, _ in seqs]
    total = sum(a * b for a, b in zip(units, items))
    size = max(-(-total // nwg), MIN_SLICE)
    out = []
    for wg in range(nwg):
        mine = []
        u = min(wg * size, total)
        u_hi = min(u + size, total)
        at = s = 0
        while u < u_hi:
            end = at + units[s] * items[s]
            if u >= end:
                at, s = end, s + 1
                continue
            r0, n, T = seqs[s]
            it = (u - at) // units[s]
            it0 = at + it * units[s]
            stop = min(u_hi, it0 + units[s])
            j0, j1 = max(u - it0 - ITEM_COST, 0), max(stop - it0 - ITEM_COST, 0)
            u = stop
            if j0 >= j1:
                continue
            nct = -(-n * group // cols)
            mine.append(Piece(wg, s, it // nct, it % nct * cols, j0, j1, units[s] - ITEM_COST, r0, n, T,
                              (it0 + units[s] - 1) // size))
        out.append(mine)
    return cols, out


def run(pieces):
    """[(piece, its tiles were handed over by the piece before, times that its list of 64 blocks was renewed)]"""
    out, linked = [], False
    for p in pieces:
        end = p.j0 + (p.j1 - p.j0 + 1) // 2 * 2
        out.append((p, linked, (end - p.j0 - 1) // CHUNK))
        linked = end - p.j0 >= 4
    return out
