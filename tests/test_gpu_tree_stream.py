"""Tree attention where workgroups stream: many pieces of many tiles each, handed from one to the next.

A workgroup whose slice is long keeps three tiles on their way across the
ends of its pieces and renews its list of block ids every 56 tiles.  Batches
for that need far more tiles than there are workgroups; a small pool, whose
blocks the tables name many times over, keeps them cheap.  tree_walk.py says
beforehand that the batch holds what a test is for; results are compared with
the oracle for a sample of sequences and KV heads.
"""
import numpy as np
import pytest
import torch

import tree_walk
import workloads
from oracle import tree
from test_gpu_tree import tree_masks

pytestmark = pytest.mark.gpu

FMT = ["bf16", "fp8_e4m3"]
# columns of an item -> rows of a tree (16 query heads to a KV head)
WIDTHS = {64: (1, 4), 128: (5, 8), 256: (12, 16)}
G, HKV, BLOCKS = 16, 2, 96


def note(msg):
    print(f"[gpu-test] {msg}", flush=True)


class Batch:
    def __init__(self, fmt, cols, seed, long_tail=True):
        rng = np.random.default_rng(seed)
        self.fmt, self.cols = fmt, cols
        kt = 64 if fmt != "bf16" else 32
        cus = torch.cuda.get_device_properties(0).multi_processor_count
        wgs = cus if cols == 256 else 2 * cus
        lo, hi = WIDTHS[cols]
        # tiles of the sequences: some of few, most of hundreds, as many as slices of 150 tiles take
        ctx, n, total = [], [], 0
        while total < 150 * wgs:
            tiles = int(rng.choice([rng.integers(1, 7), rng.integers(20, 90), rng.integers(100, 400 if long_tail else 130)]))
            t = kt * tiles - int(rng.integers(0, kt))
            m = min(int(rng.integers(lo, hi + 1)), t)
            ctx.append(t)
            n.append(m)
            total += HKV * (tiles + tree_walk.ITEM_COST)
        self.ctx, self.n = np.array(ctx), np.array(n)
        self.q_start = np.concatenate([[0], np.cumsum(n)])
        self.total_q, self.B = int(self.q_start[-1]), len(ctx)
        self.mb = -(-int(self.ctx.max()) // 16)
        self.max_ctx = 16 * self.mb
        got, wg = tree_walk.walk(self.q_start.tolist(), ctx, self.total_q, G * HKV, HKV, self.max_ctx, 1,
                                 fmt != "bf16", cus)
        assert got == cols and len(wg) == wgs
        self.runs = [r for p in wg for r in tree_walk.run(p)]
        self.kt = kt
        self.tables = rng.integers(0, BLOCKS, (self.B, self.mb)).astype(np.int32)
        t = np.uint16 if fmt == "bf16" else np.uint8
        x, y = rng.standard_normal((2, BLOCKS, HKV, 16, 128)).astype(np.float32)
        self.ks = self.vs = None
        if fmt == "bf16":
            self.K, self.V = workloads.to_bf16_codes(x), workloads.to_bf16_codes(y.swapaxes(2, 3))
        else:
            self.ks, self.vs = ((4.5 + rng.random(HKV)).astype(np.float32) / 448 for _ in range(2))
            self.K, self.V = workloads.to_e4m3_codes(x * 93), workloads.to_e4m3_codes(y.swapaxes(2, 3) * 93)
        assert self.K.dtype == t
        self.q = workloads.to_bf16_codes(rng.standard_normal((self.total_q, G * HKV, 128)).astype(np.float32))
        self.mask = tree_masks(rng, n, 1, "tree")
        self.scale = 128 ** -0.5

    def device(self, lib):
        dev = lambda a: torch.from_numpy(a.view(np.int16) if a.dtype == np.uint16 else a).cuda()  # noqa: E731
        dec = lib.TreeDecoder(self.B, G * HKV, HKV, self.mb, self.max_ctx, len(self.K), self.total_q, 1,
                              self.fmt != "bf16")
        dec.workspace.fill_(255)
        sc = [None if x is None else dev(x) for x in (self.ks, self.vs)]
        args = (dev(self.q), dev(np.ascontiguousarray(self.K)), dev(np.ascontiguousarray(self.V)), dev(self.tables),
                dev(self.ctx.astype(np.int32)), dev(self.q_start.astype(np.int32)), dev(self.mask.view(np.int64)))
        outs = []
        for _ in range(2):
            out = torch.full((self.total_q, G * HKV, 128), float("nan"), dtype=torch.bfloat16, device="cuda")
            dec(*args, self.scale, out, *sc)
            outs.append(out)
        torch.cuda.synchronize()
        assert torch.equal(outs[0].view(torch.int16), outs[1].view(torch.int16))
        return outs[0].float().cpu().numpy()

    def oracle(self, s, g, heads):
        """(out, bound) of one sequence and some heads of one KV head"""
        r = slice(self.q_start[s], self.q_start[s + 1])
        sc = [None if x is None else x[g:g + 1] for x in (self.ks, self.vs)]
        return tree.tree_attention(self.q[r][:, heads], self.K[:, g:g + 1], self.V[:, g:g + 1], self.tables[s:s + 1],
                                   self.ctx[s:s + 1], [0, self.n[s]], self.mask[r], self.scale, self.fmt, *sc)


@pytest.mark.parametrize("fmt", FMT)
@pytest.mark.parametrize("cols", WIDTHS)
def test_streams_against_the_oracle(gpu_lib, cols, fmt):
    """Handed-over pieces of even and odd tiles, of either KV head, and pieces of more than 56 and 112 tiles."""
    b = Batch(fmt, cols, cols)
    note(f"tree streams {fmt}, {cols} columns, {b.B} sequences of up to {b.ctx.max()} tokens, {len(b.runs)} pieces")
    linked = [p for p, link, _ in b.runs if link]
    assert len(linked) > 100 and max(k for _, _, k in b.runs) >= 2 and sum(k >= 1 for _, _, k in b.runs) > 50
    assert any(link and k >= 1 for _, link, k in b.runs)
    before = [a for (a, _, _), (_, link, _) in zip(b.runs, b.runs[1:]) if link]
    assert {(p.j1 - p.j0) % 2 for p in before} == {0, 1} and {p.g for p in linked} == {0, 1}
    assert min(p.j1 - p.j0 for p in linked) <= 2
    got = b.device(gpu_lib)
    assert np.isfinite(got).all()
    # of every kind a few: handed over, renewed once, renewed twice, short
    rng = np.random.default_rng(1)
    kinds = [[p for p, link, _ in b.runs if link and p.whole], [p for p, link, k in b.runs if link and k >= 1],
             [p for p, _, k in b.runs if k >= 2], [p for p in linked if p.nt <= 3], [p for p in linked if not p.whole]]
    picked = {(p.s, p.g) for ps in kinds for p in (ps[i] for i in rng.integers(0, len(ps), 3))}
    worst = 0.0
    for s, g in sorted(picked):
        heads = g * G + rng.choice(G, 3, replace=False)
        ref, bound = b.oracle(s, g, heads)
        mine = got[b.q_start[s]:b.q_start[s + 1]][:, heads]
        worst = max(worst, (np.abs(mine - ref) / bound).max())
    note(f"  {len(picked)} sequences and heads, largest error {worst:.2f} of its bound")
    assert worst <= 1.0


@pytest.mark.parametrize("fmt", FMT)
@pytest.mark.parametrize("cols", WIDTHS)
def test_values_that_are_not_finite_at_a_handover(gpu_lib, cols, fmt):
    """V of drafts that is not finite in the first tile of a piece that was handed over: rows that do not see it
    keep their bits, and so do all other sequences."""
    b = Batch(fmt, cols, 500 + cols)
    kt = b.kt
    # handed-over pieces whose first tile holds the last draft
    first = [p for p, link, _ in b.runs if link and p.j0 == (p.T - 1) // kt]
    later = [p for p, link, _ in b.runs if link and p.j0 < (p.T - p.n) // kt < p.j1]
    note(f"tree streams with NaN {fmt}, {cols} columns: {len(first)} handed-over pieces start with drafts")
    assert len(first) >= 4 and len(later) >= 4
    hits = sorted({(p.s, p.g) for p in first[:6] + later[:6]})
    # each hit sequence's last block of drafts becomes a block of its own
    own = {s: i for i, s in enumerate(sorted({s for s, _ in hits}))}
    K, V = [np.concatenate([x, np.zeros((len(own),) + x.shape[1:], x.dtype)]) for x in (b.K, b.V)]
    for s, i in own.items():
        last = (b.ctx[s] - 1) // 16
        K[BLOCKS + i], V[BLOCKS + i] = b.K[b.tables[s, last]], b.V[b.tables[s, last]]
        b.tables[s, last] = BLOCKS + i
    b.K, b.V = K, V.copy()
    clean = b.device(gpu_lib)
    assert np.isfinite(clean).all()
    nan = 0x7FC0 if fmt == "bf16" else 0x7F
    for s, g in hits:
        t = b.ctx[s] - 1                       # the last draft
        b.V[BLOCKS + own[s], g, 40:44, t % 16] = nan
    got = b.device(gpu_lib)
    want = clean.copy()
    for s, g in hits:
        r = np.arange(b.q_start[s], b.q_start[s + 1])
        see = tree.bits(b.mask[r], b.n[s])[:, -1]
        assert see.any()
        for h in range(g * G, (g + 1) * G):
            want[r[see], h, 40:44] = np.nan
    assert np.array_equal(got, want, equal_nan=True)
