"""A step that verifies drafted tokens with every operator's result held against its oracle, the caches among them.

The caches are copied between the layers' attention and the move of the
accepted path: what norm, rotation and append wrote is compared with the
formula (V's codes exactly, everything that no row owns unchanged), every
granted sequence's attention in every layer with the oracle over those
copies, and the caches after the move with tree.accept exactly.
"""
import numpy as np
import pytest
import torch

from oracle import append, numerics, rope, tables, tree
from test_gpu_tree_step import Engine, dev, draws

pytestmark = pytest.mark.gpu

# Norm and rotation in float32: 140 roundings of what a turned value sums, |a c| + |b s| <= 2 max |y|, and 2 max |y| more
# as in test_gpu_rope.py
E = 140 * 2.0 ** -24


def note(msg):
    print(f"[gpu-test] {msg}", flush=True)


class Recorder(Engine):
    """The engine's step, with what each layer's attention read and the caches before the move kept."""

    def step(self, new, parents, qkv, accepted, n_accepted):
        lib, hq, hkv = self.lib, self.hq, self.hkv
        lib.kv_tables_step(self.ctx, self.owned, new, self.ring, self.state, self.tb, self.ctx2, self.owned2,
                           self.state2, self.q_start, self.slots, self.pos, self.granted, self.tables, parents,
                           self.mask)
        self.qs = []
        for l in range(self.layers):
            x = qkv[l]
            lib.qk_norm_rope_append(x[:, :hq * 128], x[:, hq * 128:(hq + hkv) * 128], x[:, (hq + hkv) * 128:], self.cs,
                                    self.pos, self.slots, self.q, self.k[l], self.v[l], self.qk, self.qw, self.kw,
                                    1e-6, self.ks, self.vs)
            self.dec(self.q, self.k[l], self.v[l], self.tb, self.ctx2, self.q_start, self.mask, 128 ** -0.5,
                     self.outs[l], self.ks, self.vs)
            self.qs.append(self.q.clone())
        self.before = [[t.clone() for t in ts] for ts in (self.k, self.v)]
        lib.kv_cache_accept(self.cl, self.tb, self.ctx2, self.q_start, accepted, n_accepted, self.ctx3, self.dec.shape)
        self.ctx.copy_(self.ctx3)
        self.owned.copy_(self.owned2)
        self.state.copy_(self.state2)


def codes(t, fmt):
    return t.cpu().numpy().view(np.uint16 if fmt == "bf16" else np.uint8)


def branches(mask):
    """Whether some row of a tree (one mask word a row) does not see the row before it."""
    return any(not (int(mask[i, 0]) >> (i - 1)) & 1 for i in range(1, len(mask)))


@pytest.mark.parametrize("fmt", ["bf16", "fp8_e4m3"])
def test_every_operator_of_a_step(gpu_lib, fmt):
    note(f"verification steps with their caches, {fmt}")
    B, mb, nb, hq, hkv, rows = 6, 8, 16, 8, 2, 240
    e = Recorder(gpu_lib, B, mb, nb, hq, hkv, rows, fmt != "bf16")
    rng = np.random.default_rng(11)
    o = dict(ctx=np.zeros(B, int), owned=np.zeros(B, int), ring=e.ring.cpu().numpy(), state=[0, nb],
             tables=e.tb.cpu().numpy())
    K, V = ([codes(t, fmt) for t in ts] for ts in (e.k, e.v))
    ks, vs = (None if t is None else t.cpu().numpy() for t in (e.ks, e.vs))
    qw, kw = (numerics.decode_bf16(t.cpu().numpy().view(np.uint16)) for t in (e.qw, e.kw))
    table = e.cs.cpu().numpy().astype(np.float64)
    refused = moved = 0
    for i in range(8):
        new, par, qkv, acc, n_acc = draws(rng, B, rows, hq, hkv, e.layers, i == 0)
        o = tables.step(o["ctx"], o["owned"], new, o["ring"], *map(int, o["state"]), o["tables"], rows, par, 1)
        n = np.diff(o["q_start"])
        refused += int((o["granted"] == 0).sum())
        n_acc = np.where(o["granted"] == 1, n_acc, -1)
        e.step(dev(new, np.int32), dev(par, np.int32), [dev(x) for x in qkv], dev(acc, np.int32), dev(n_acc, np.int32))
        torch.cuda.synchronize()
        for name, t in (("slots", e.slots), ("positions", e.pos), ("tables", e.tb), ("granted", e.granted),
                        ("q_start", e.q_start), ("ctx", e.ctx2)):
            assert np.array_equal(t.cpu().numpy(), o[name]), (i, name)

        # norm, rotation and cache write: rows with a slot in the caches, rows with a position in q
        pos, slots = o["positions"], o["slots"]
        live, put = np.flatnonzero(pos >= 0), np.flatnonzero(slots >= 0)
        cos, sin = table[np.maximum(pos, 0), :64], table[np.maximum(pos, 0), 64:]
        blk, off = slots[put] // 16, slots[put] % 16
        for l in range(e.layers):
            x = qkv[l].reshape(rows, -1, 128)
            want = []
            for part, w in ((x[:, :hq], qw), (x[:, hq:hq + hkv], kw)):
                r = rope.turn(rope.norm(numerics.decode_bf16(part), w, 1e-6), cos, sin)
                want.append((r, 4 * E * np.abs(r).max(axis=-1, keepdims=True)))
            (rq, eq), (rk, ek) = want
            q = e.qs[l].view(torch.int16).cpu().numpy().view(np.uint16)
            err = np.abs(numerics.decode_bf16(q) - rq)
            assert (err[live] <= (eq + 2.0 ** -8 * np.abs(rq))[live]).all(), (i, l)
            k, v = codes(e.before[0][l], fmt), codes(e.before[1][l], fmt)
            own = np.zeros((nb, 16), bool)
            own[blk, off] = True
            assert own.sum() == len(put)
            same = np.broadcast_to(~own[:, None, :, None], k.shape)
            assert np.array_equal(k[same], K[l][same]), (i, l)
            got = numerics.decode(k[blk, :, off], fmt)
            if fmt == "bf16":
                assert (np.abs(got - rk[put]) <= (ek + 2.0 ** -8 * np.abs(rk))[put]).all(), (i, l)
            else:
                z = rk[put] / ks.astype(np.float64)[:, None]
                cut = np.clip(z, -448, 448)
                lim = np.maximum(2.0 ** -4 * np.abs(cut), 2.0 ** -10) + 2 * ek[put] / ks[:, None]
                assert (np.abs(got - cut) <= lim).all(), (i, l)
            wv = V[l].copy()
            for g in range(hkv):
                wv[blk, g, :, off] = append.encode(x[put, hq + hkv + g], fmt, None if vs is None else vs[g])
            assert np.array_equal(v, wv), (i, l)
            # attention over those caches, every granted sequence
            trees = 0
            for s in range(B):
                if n[s] == 0 or not o["granted"][s]:
                    continue
                r = slice(o["q_start"][s], o["q_start"][s + 1])
                ref, bound = tree.tree_attention(q[r], k, v, o["tables"][s:s + 1], o["ctx"][s:s + 1], [0, n[s]],
                                                 o["mask"][r], 128 ** -0.5, fmt, ks, vs)
                assert (np.abs(e.outs[l][r].float().cpu().numpy() - ref) <= bound).all(), (i, l, s)
                trees += branches(o["mask"][r])
            assert trees >= (i > 0), i
            # the accepted path's move
            K[l], V[l], ctx = tree.accept(k, v, o["tables"], o["ctx"], o["q_start"], acc, n_acc)
            assert np.array_equal(codes(e.k[l], fmt), K[l]) and np.array_equal(codes(e.v[l], fmt), V[l]), (i, l)
            moved += int((K[l] != k).any())
        assert np.array_equal(e.ctx.cpu().numpy(), ctx)
        o["ctx"] = ctx
    assert refused > 0 and moved >= 6 * e.layers
