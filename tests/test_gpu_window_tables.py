"""kv_tables_step on tables of sequences whose blocks have left a window: they end with -2, entries below 0 hold no block.

Whole numbers against the oracle, then a serving run in which blocks that left
the window go back to the ring, sequences end and others take their place.
"""
import numpy as np
import pytest
import torch

import window_cases as wc
import workloads
from oracle import rope, tables
from oracle import window as ow
from test_gpu_tables import run, same, state
from window_cases import dev

pytestmark = pytest.mark.gpu


def note(msg):
    print(f"[gpu-test] {msg}", flush=True)


@pytest.mark.parametrize("B,mb,free,over", [(1, 4, 3, 1.0), (3, 1, 0, 1.0), (64, 32, 40, 0.3), (65, 16, 10, 0.2),
                                            (256, 20, 300, 0.1), (300, 40, 9, 0.9), (1024, 6, 800, 0.5),
                                            (4096, 5, 2000, 0.05), (9, 600, 4000, 0.7), (2, 5000, 30, 1.0)])
@pytest.mark.parametrize("gone", [0.02, 0.5, 1.0])
def test_entries_that_hold_no_block(gpu_lib, B, mb, free, over, gone):
    note(f"tables with blocks gone B={B} blocks={mb} gone={gone}")
    rng = np.random.default_rng(B + mb)
    ctx, owned, tb, ring, head = state(rng, B, mb, free)
    tail = np.minimum(ctx // 16, mb - 1)                     # (the block that new tokens go into stays)
    lost = (rng.random((B, mb)) < gone) & (np.arange(mb) < tail[:, None]) & (tb >= 0)
    tb[lost] = rng.choice([-1, -2, -2 ** 31], int(lost.sum()))
    new = np.where(rng.random(B) < over, -2, rng.integers(0, 20, B))
    new[(new < 0) & ~lost.any(1) & (rng.random(B) < 0.5)] = -1   # (every entry holds a block)
    rows = int(np.maximum(new, 0).sum()) + 2
    want = tables.step(ctx, owned, new, ring, head, free, tb, rows)
    assert (want["ring"][(want["state"][0] + np.arange(want["state"][1])) % len(ring)] >= 0).all()
    same(run(gpu_lib, ctx, owned, new, ring, head, free, tb, rows, repeat=2), want)


def test_more_entries_than_the_pool_has_blocks(gpu_lib):
    """Contexts of many more blocks than the pool's, nearly all gone; one whole table of them."""
    note("tables, contexts longer than the pool")
    rng = np.random.default_rng(3)
    B, mb, nb, free = 5, 3000, 40, 6
    tb = np.full((B, mb), -1)
    ids = rng.permutation(nb)
    for s in range(4):
        tb[s, [0, 17, 1000 + s, 2990, 2999][:5 - s]] = ids[5 * s:5 * s + 5 - s]
    ctx, owned = np.full(B, 16 * mb - 3), np.array([mb, mb, mb - 5, 0, mb])
    ring = np.full(nb, -5)
    ring[(37 + np.arange(free)) % nb] = ids[30:30 + free]
    for new in ([-2, -2, -2, -2, -2], [-2, 2, -2, 0, -2], [3, -2, 1, -2, 1], [-2, -5, -2 ** 31, 1, -3]):
        want = tables.step(ctx, owned, np.array(new), ring, 37, free, tb, 8)
        same(run(gpu_lib, ctx, owned, np.array(new), ring, 37, free, tb, 8, repeat=2), want)


def test_a_serving_run_over_a_window(gpu_lib):
    """Tables and slots by kv_tables_step, the cache write, attention over a window; after each step blocks that no
    later row sees go back to the ring.  Sequences end and their ids are handed out again; none is lost or doubled.
    (The first step has more rows than a call takes: three sequences are refused.)"""
    note("window, block tables, sequences that end")
    lib, rng = gpu_lib, np.random.default_rng(4)
    B, hq, hkv, nb, mb, n_pos, window, n_sink, rows = 4, 4, 2, 24, 40, 640, 50, 3, 100
    table = dev(rope.table(n_pos, 128).astype(np.float32))
    tb = torch.full((B, mb), -1, dtype=torch.int32, device="cuda")
    ctx, owned = (torch.zeros(B, dtype=torch.int32, device="cuda") for _ in range(2))
    ring, st = torch.randperm(nb, device="cuda").int(), torch.tensor([5, nb], dtype=torch.int32, device="cuda")
    k, v = (torch.full((nb, hkv) + d, 0x7F, dtype=torch.uint8, device="cuda") for d in ((16, 128), (128, 16)))
    ks, vs = (torch.full((nb, hkv), 255, dtype=torch.uint8, device="cuda") for _ in range(2))
    sh, tsh = lib.qk_shape(rows, hq, hkv, nb, n_pos, block_scales=True), lib.tables_shape(B, mb, nb, rows)
    psh = lib.prefill_shape(B, hq, hkv, mb, 16 * mb, nb, rows, block_scales=True)
    plan = [[70, 33, 0, 1], [1, 1, 40, 1], [30, 20, 1, 1], [1, 1, 1, 60], [-2, 30, 1, 1], [90, 1, -2, 1],
            [1, -2, 30, 1], [1, 60, 1, -2], [40, 1, 1, 20], [-2, -2, -2, -2], [70, 5, 5, 5], [1, 1, 1, 1]]
    ended = 0
    for new in plan:
        x = torch.tensor(new, dtype=torch.int32, device="cuda")
        before = ctx.clone()
        out = [torch.zeros(n, dtype=t, device="cuda") for n, t in (
            (B, torch.int32), (B, torch.int32), (2, torch.int32), (B + 1, torch.int32), (rows, torch.int64),
            (rows, torch.int32), (B, torch.int32))]
        ctx2, owned2, st2, q_start, slots, pos, ok = out
        lib.kv_tables_step(ctx, owned, x, ring, st, tb, ctx2, owned2, st2, q_start, slots, pos, ok, tsh)
        first = np.concatenate([[0], np.cumsum(np.maximum(new, 0))])
        good = [s for s in range(B) if first[s + 1] <= rows]
        assert ok.tolist() == [int(s in good) for s in range(B)] and q_start.tolist() == np.minimum(first, rows).tolist()
        tb[x < 0] = -1
        ctx, owned, st = ctx2, owned2, st2
        qkv = dev(workloads.to_bf16_codes(rng.standard_normal((rows, hq + 2 * hkv, 128)).astype(np.float32)))
        q = torch.empty((rows, hq, 128), dtype=torch.int16, device="cuda")
        lib.qk_norm_rope_append_scaled(qkv[:, :hq].contiguous(), qkv[:, hq:hq + hkv].contiguous(),
                                       qkv[:, hq + hkv:].contiguous(), table, pos, slots, q, k, v, ks, vs, sh)
        o = torch.empty((rows, hq, 128), dtype=torch.bfloat16, device="cuda")
        lib.window_prefill_attention(q, k, v, tb, ctx, q_start, 0.088, window, n_sink, o, psh, ks, vs)
        torch.cuda.synchronize()
        live = np.concatenate([np.arange(first[i], first[i + 1]) for i in good]).astype(int)
        rest = np.setdiff1d(np.arange(rows), live)
        assert (slots[live] >= 0).all() and (slots[rest] == -1).all()
        if len(live):
            host = [t.cpu().numpy() for t in (q, k, v, tb, ctx, ks, vs)]
            hq_, hk, hv, htb, hctx, hks, hvs = host
            starts = np.concatenate([[0], np.cumsum(np.maximum(new, 0)[good])])
            ref, bound = ow.window_attention(hq_.view(np.uint16)[live], hk, hv, htb[good], hctx[good], starts, 0.088, window,
                                             n_sink, "e4m3_block", hks, hvs)
            wc.check(o[live], ref, bound)
        # blocks that no later row sees go to the end of the ring
        at = torch.arange(mb, device="cuda") * 16
        lost = (tb >= 0) & (at[None] >= n_sink) & (at[None] + 16 <= (ctx[:, None] + 1 - window))
        ids = tb[lost]
        st = st.clone()
        ring[(st[0] + st[1] + torch.arange(len(ids), device="cuda")) % nb] = ids
        st[1] += len(ids)
        tb[lost] = -1
        ended += sum(int(before[s]) > 0 for s in range(B) if new[s] < 0)
        held = tb[tb >= 0].tolist()
        free = ring[(st[0] + torch.arange(int(st[1]), device="cuda")) % nb].tolist()
        assert sorted(held + free) == list(range(nb))
    assert ended >= 6
