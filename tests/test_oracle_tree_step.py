"""Pins of the oracles of a step that verifies drafted tokens: block tables, rotation, tree attention, accepted paths."""
import numpy as np
import pytest

import workloads
from oracle import attention, numerics, prefill, rope, tables, tree


# ---------------------------------------------------------------- block tables

def test_tables_hand_worked_step():
    ring = np.array([70, 71, 72, 73, 74, 0, 0, 0])
    tb = np.full((4, 4), -1)
    tb[0, :2] = [10, 11]     # 17 tokens
    tb[1, :1] = [12]         # 16 tokens
    tb[3, :3] = [13, 14, 15]
    o = tables.step([17, 16, 0, 40], [2, 1, 0, 3], [1, 2, 40, -1], ring, 1, 4, tb, 50)
    assert o["granted"].tolist() == [1, 1, 1, 1]
    assert o["ctx"].tolist() == [18, 18, 40, 0] and o["owned"].tolist() == [2, 2, 3, 0]
    assert o["tables"][1, :2].tolist() == [12, 71] and o["tables"][2, :3].tolist() == [72, 73, 74]
    assert o["q_start"].tolist() == [0, 1, 3, 43, 43]
    assert o["slots"][:4].tolist() == [11 * 16 + 1, 71 * 16, 71 * 16 + 1, 72 * 16] and (o["slots"][43:] == -1).all()
    assert o["positions"][:5].tolist() == [17, 16, 17, 0, 1] and (o["positions"][43:] == -1).all()
    assert o["state"].tolist() == [5, 3]                       # four taken, three given back
    assert o["ring"][[5, 6, 7]].tolist() == [13, 14, 15]
    # one free id fewer: the third sequence is refused, the others are not
    o = tables.step([17, 16, 0, 40], [2, 1, 0, 3], [1, 2, 40, -1], ring, 1, 3, tb, 50)
    assert o["granted"].tolist() == [1, 1, 0, 1] and (o["slots"][3:] == -1).all() and o["ctx"][2] == 0


def test_tables_tree_masks():
    o = tables.step([5], [1], [5], np.arange(4), 0, 4, np.array([[9, -1]]), 6, parents=[-1, 0, 0, 2, 9, 0], words=1)
    assert o["mask"][:, 0].tolist() == [1, 0b11, 0b101, 0b1101, 0b10000, 0]   # (9 is no earlier token: a root)
    assert o["positions"].tolist() == [5, 6, 6, 7, 5, -1]
    assert o["slots"].tolist() == [9 * 16 + 5 + i for i in range(5)] + [-1]


def test_tables_first_batch_as_the_host_allocator(host_lib):
    pool = host_lib.KVPool(1, 1, 128, 2, 64, 20 * 2 * 128 * 2 * 64, 1.0, 0.0, seed=3)
    nb = pool.info().num_blocks
    ids = pool.alloc_seq(64)
    for _ in range(nb // 4 - 1):
        ids = np.concatenate([ids, pool.alloc_seq(64)])
    again = host_lib.KVPool(1, 1, 128, 2, 64, 20 * 2 * 128 * 2 * 64, 1.0, 0.0, seed=3)
    lens = [3, 40, 16, 64]
    o = tables.step([0] * 4, [0] * 4, lens, ids, 0, nb, np.full((4, 4), -1), sum(lens))
    for s, n in enumerate(lens):
        assert o["tables"][s, :-(-n // 16)].tolist() == again.alloc_seq(n).tolist()


def test_tables_blocks_are_conserved_over_random_steps():
    rng = np.random.default_rng(0)
    B, mb, nb = 6, 8, 30
    ctx, owned, tb = np.zeros(B, int), np.zeros(B, int), np.full((B, mb), -1)
    ring, head, count = rng.permutation(nb), 4, nb
    for _ in range(200):
        new = rng.integers(-1, 40, B)
        o = tables.step(ctx, owned, new, ring, head, count, tb, 200)
        ctx, owned, ring, tb = o["ctx"], o["owned"], o["ring"], o["tables"]
        head, count = o["state"].tolist()
        held = np.concatenate([tb[s, :owned[s]] for s in range(B)])
        free = ring[(head + np.arange(count)) % nb]
        assert sorted(np.concatenate([held, free]).tolist()) == list(range(nb))
        assert (owned * 16 >= ctx).all()


# ---------------------------------------------------------------- rotation

def test_rope_is_complex_multiplication_and_keeps_lengths():
    rng = np.random.default_rng(1)
    y = rng.standard_normal((5, 3, 128))
    t = rope.table(900, 64)[rng.integers(0, 900, 5)]
    cos, sin = t[:, :32], t[:, 32:]
    for inter in (False, True):
        out = rope.turn(y, cos, sin, inter)
        a, b = (y[..., 0:64:2], y[..., 1:64:2]) if inter else (y[..., :32], y[..., 32:64])
        z = (a + 1j * b) * (cos + 1j * sin)[:, None]
        u, v = (out[..., 0:64:2], out[..., 1:64:2]) if inter else (out[..., :32], out[..., 32:64])
        assert np.allclose(u, z.real, atol=1e-13) and np.allclose(v, z.imag, atol=1e-13)
        assert (out[..., 64:] == y[..., 64:]).all()
        assert np.allclose(np.linalg.norm(out, axis=-1), np.linalg.norm(y, axis=-1))
    assert (rope.turn(y, np.ones((5, 32)), np.zeros((5, 32))) == y).all()


def test_rope_products_depend_on_the_distance():
    rng = np.random.default_rng(2)
    x, y = rng.standard_normal((2, 1, 1, 128))
    t = rope.table(500, 128)

    def at(v, p):
        return rope.turn(v, t[p:p + 1, :64], t[p:p + 1, 64:])

    assert np.isclose((at(x, 400) * at(y, 390)).sum(), (at(x, 17) * at(y, 7)).sum())


def test_norm():
    x = np.array([[3.0] * 64 + [-3.0] * 64])
    w = np.linspace(0.5, 1.5, 128)
    assert np.allclose(rope.norm(x, w, 0.0), np.sign(x) * w)
    assert (rope.norm(np.zeros((1, 128)), w, 1e-6) == 0).all()


# ---------------------------------------------------------------- tree attention

@pytest.mark.parametrize("fmt", ["bf16", "fp8_e4m3"])
def test_tree_with_chain_masks_is_chunked_prefill(fmt):
    w = workloads.make_prefill([(5, 40), (1, 17), (3, 3)], 4, 2, c_max=64, kv_format=fmt, seed=3)
    qs = w.meta["q_start"]
    mask = np.array([[(2 << i) - 1] for s in range(3) for i in range(qs[s + 1] - qs[s])], np.uint64)
    args = (w.q_bits, w.k_store.dense(), w.v_store.dense(), w.block_tables, w.context_lens, qs)
    out, _ = tree.tree_attention(*args, mask, w.scale, fmt, w.k_scale, w.v_scale)
    ref = prefill.chunked_prefill_attention(*args, w.scale, kv_format=fmt, k_scale=w.k_scale, v_scale=w.v_scale)
    assert np.abs(out - ref).max() < 1e-12


def test_tree_of_one_draft_is_decode():
    w = workloads.make_workload(3, 4, 2, [1, 20, 33], c_max=64, seed=4)
    out, _ = tree.tree_attention(w.q_bits, w.k_store.dense(), w.v_store.dense(), w.block_tables, w.context_lens,
                                 np.arange(4), np.ones((3, 1), np.uint64), w.scale)
    ref = attention.paged_decode_attention(w.q_bits, w.k_store, w.v_store, w.block_tables, w.context_lens, w.scale)
    assert np.abs(out - ref).max() < 1e-12


def test_tree_sparse_masks_by_brute_force_and_nan_in_unseen_tokens():
    w = workloads.make_prefill([(4, 21)], 2, 1, c_max=32, seed=5)
    K, V = w.k_store.dense(), w.v_store.dense()
    see = np.array([[1, 0, 0, 0], [1, 1, 0, 0], [0, 0, 0, 0], [0, 1, 0, 1]], bool)
    mask = np.array([[sum(1 << j for j in range(4) if see[i, j])] for i in range(4)], np.uint64)
    blk, off = w.block_tables[0][19 // 16], 19 % 16     # draft 2, which no row sees
    K[blk, 0, off] = 0x7FC0
    V[blk, 0, :, off] = 0x7FC0
    out, bound = tree.tree_attention(w.q_bits, K, V, w.block_tables, w.context_lens, [0, 4], mask, w.scale)
    assert np.isfinite(out).all() and np.isfinite(bound).all()
    q = numerics.decode_bf16(w.q_bits)
    for i in range(4):
        for h in range(2):
            ts = [t for t in range(21) if t < 17 or see[i, t - 17]]
            k = [numerics.decode_bf16(K[w.block_tables[0][t // 16], 0, t % 16]) for t in ts]
            v = [numerics.decode_bf16(V[w.block_tables[0][t // 16], 0, :, t % 16]) for t in ts]
            e = [np.exp(w.scale * sum(a * b for a, b in zip(q[i, h], x))) for x in k]
            ref = sum(a * b for a, b in zip(e, v)) / sum(e)
            assert np.abs(out[i, h] - ref).max() < 1e-12


def test_tree_row_without_tokens_is_zero():
    w = workloads.make_prefill([(2, 2)], 2, 1, c_max=16, seed=6)
    out, _ = tree.tree_attention(w.q_bits, w.k_store.dense(), w.v_store.dense(), w.block_tables, w.context_lens,
                                 [0, 2], np.array([[0], [2]], np.uint64), w.scale)
    assert (out[0] == 0).all() and (out[1] != 0).any()


def test_bits():
    m = np.array([[1 << 63, 1], [5, 0]], np.uint64)
    b = tree.bits(m, 66)
    assert np.flatnonzero(b[0]).tolist() == [63, 64] and np.flatnonzero(b[1]).tolist() == [0, 2]


# ---------------------------------------------------------------- accepted drafts

def test_accept_by_scalar_moves():
    rng = np.random.default_rng(7)
    K = rng.integers(0, 60000, (6, 2, 16, 128)).astype(np.uint16)
    V = rng.integers(0, 60000, (6, 2, 128, 16)).astype(np.uint16)
    bt = np.array([[4, 0], [2, 5]])
    k, v, ctx = tree.accept(K, V, bt, [20, 18], [0, 9, 12], np.array([[0, 3, 4, 8], [1, 1, 2, -1]]), [4, 3])
    assert ctx.tolist() == [15, 16]                     # the second path's entry 1 repeats: one token is kept
    ek, ev = K.copy(), V.copy()
    for s, b, path in ((0, 11, [0, 3, 4, 8]), (1, 15, [1])):
        for j, i in enumerate(path):
            for d in range(128):
                for g in range(2):
                    src, dst = b + i, b + j
                    ek[bt[s][dst // 16], g, dst % 16, d] = K[bt[s][src // 16], g, src % 16, d]
                    ev[bt[s][dst // 16], g, d, dst % 16] = V[bt[s][src // 16], g, d, src % 16]
    assert (k == ek).all() and (v == ev).all()


# ---------------------------------------------------------------- counts that a context corrects

def test_tables_owned_counts_below_the_context():
    ring = np.array([70, 71, 72, 73, 0, 0, 0, 0])
    tb = np.array([[10, 11, 12], [13, 14, -1], [15, -1, -1]])
    o = tables.step([40, 20, 3], [1, 0, -1], [-1, 13, -1], ring, 0, 4, tb, 13)
    assert o["ring"].tolist() == [70, 71, 72, 73, 10, 11, 12, 15] and o["state"].tolist() == [1, 7]
    assert o["owned"].tolist() == [0, 3, 0] and o["tables"][1].tolist() == [13, 14, 70]
    assert o["slots"][-1] == 70 * 16
