"""A step that verifies drafted tokens, its operators one after the other, as an engine runs them.

kv_tables_step hands out blocks, slots, positions and masks; qk_norm_rope_append
writes the drafts into the cache; tree_decode_attention reads them;
kv_cache_accept keeps one path; and the next step starts from the lengths that
are then on the device.  Every step is checked against the oracles chained the
same way, and a captured step against the eager one.
"""
import numpy as np
import pytest
import torch

import workloads
from oracle import rope, tables, tree

pytestmark = pytest.mark.gpu


def note(msg):
    print(f"[gpu-test] {msg}", flush=True)


def dev(a, dtype=None):
    a = np.ascontiguousarray(a, dtype=dtype)
    return torch.from_numpy(a.view(np.int16) if a.dtype == np.uint16 else a).cuda()


class Engine:
    """Device state of a small server: lengths twice (a call never writes what it reads)."""

    def __init__(self, lib, B, mb, nb, hq, hkv, rows, fp8, layers=2, seed=0):
        self.lib, self.rows, self.layers = lib, rows, layers
        rng = np.random.default_rng(seed)
        self.ring, self.tb = dev(rng.permutation(nb), np.int32), dev(np.full((B, mb), -1), np.int32)
        z = lambda *s, dtype=torch.int32: torch.zeros(s, dtype=dtype, device="cuda")  # noqa: E731
        self.ctx, self.owned, self.state = z(B), z(B), dev([0, nb], np.int32)
        self.ctx2, self.owned2, self.state2, self.ctx3 = z(B), z(B), z(2), z(B)
        self.q_start, self.granted, self.slots = z(B + 1), z(B), z(rows, dtype=torch.int64)
        self.pos, self.mask = z(rows), z(rows, 1, dtype=torch.int64)
        kt = torch.uint8 if fp8 else torch.int16
        self.k = [z(nb, hkv, 16, 128, dtype=kt) for _ in range(layers)]
        self.v = [z(nb, hkv, 128, 16, dtype=kt) for _ in range(layers)]
        self.ks, self.vs = (dev(rng.random(hkv) * 0.01 + 0.01, np.float32) if fp8 else None for _ in range(2))
        self.cs = dev(rope.table(mb * 16, 128), np.float32)
        self.qw, self.kw = (dev(workloads.to_bf16_codes(np.float32(1 + 0.1 * rng.standard_normal(128))))
                            for _ in range(2))
        self.tables = lib.tables_shape(B, mb, nb, rows, mask_words=1)
        self.qk = lib.qk_shape(rows, hq, hkv, nb, mb * 16, kv_fp8=fp8, q_stride=(hq + 2 * hkv) * 128,
                               k_stride=(hq + 2 * hkv) * 128, v_stride=(hq + 2 * hkv) * 128)
        self.dec = lib.TreeDecoder(B, hq, hkv, mb, mb * 16, nb, rows, kv_fp8=fp8)
        self.cl = lib.CacheLayers(self.k, self.v)
        self.q = torch.zeros((rows, hq, 128), dtype=torch.bfloat16, device="cuda")
        self.outs = [self.dec.new_out() for _ in range(layers)]
        self.hq, self.hkv = hq, hkv

    def step(self, new, parents, qkv, accepted, n_accepted):
        lib, hq, hkv = self.lib, self.hq, self.hkv
        lib.kv_tables_step(self.ctx, self.owned, new, self.ring, self.state, self.tb, self.ctx2, self.owned2,
                           self.state2, self.q_start, self.slots, self.pos, self.granted, self.tables, parents,
                           self.mask)
        for l in range(self.layers):
            x = qkv[l]
            lib.qk_norm_rope_append(x[:, :hq * 128], x[:, hq * 128:(hq + hkv) * 128], x[:, (hq + hkv) * 128:], self.cs,
                                    self.pos, self.slots, self.q, self.k[l], self.v[l], self.qk, self.qw, self.kw,
                                    1e-6, self.ks, self.vs)
            self.dec(self.q, self.k[l], self.v[l], self.tb, self.ctx2, self.q_start, self.mask, 128 ** -0.5,
                     self.outs[l], self.ks, self.vs)
        lib.kv_cache_accept(self.cl, self.tb, self.ctx2, self.q_start, accepted, n_accepted, self.ctx3, self.dec.shape)
        self.ctx.copy_(self.ctx3)
        self.owned.copy_(self.owned2)
        self.state.copy_(self.state2)


def draws(rng, B, rows, hq, hkv, layers, first):
    # the first step is a prompt of up to 40 tokens (a chain, accepted whole), later ones trees; some sequences end
    new = rng.integers(1, 41, B) if first else np.where(rng.random(B) < 0.1, -1, rng.integers(1, 14, B))
    par, acc, n_acc = [], np.full((B, 40), -1), []
    for s, n in enumerate(new):
        n = max(n, 0)
        p = np.arange(n) - 1 if first else np.array([-1 if i == 0 else rng.integers(i // 3, i) for i in range(n)], int)
        path = []
        at = n - 1
        while n and at >= 0:
            path.insert(0, at)
            at = p[at]
        acc[s, :len(path)] = path
        n_acc.append(len(path))
        par += p.tolist()
    par += [0] * (rows - len(par))
    qkv = [workloads.to_bf16_codes(rng.standard_normal((rows, (hq + 2 * hkv) * 128)).astype(np.float32))
           for _ in range(layers)]
    return new, np.array(par), qkv, acc, np.array(n_acc)


@pytest.mark.parametrize("fmt", ["bf16", "fp8_e4m3"])
def test_steps_against_the_chained_oracles(gpu_lib, fmt):
    note(f"verification steps, {fmt}")
    B, mb, nb, hq, hkv, rows = 6, 8, 13, 8, 2, 240
    e = Engine(gpu_lib, B, mb, nb, hq, hkv, rows, fmt != "bf16")
    rng = np.random.default_rng(1)
    o = dict(ctx=np.zeros(B, int), owned=np.zeros(B, int), ring=e.ring.cpu().numpy(), state=[0, nb],
             tables=e.tb.cpu().numpy())
    refused = 0
    for i in range(9):
        new, par, qkv, acc, n_acc = draws(rng, B, rows, hq, hkv, e.layers, i == 0)
        o = tables.step(o["ctx"], o["owned"], new, o["ring"], *map(int, o["state"]), o["tables"], rows, par, 1)
        refused += int((o["granted"] == 0).sum())
        # a refused sequence has rows but no tokens of theirs: it stays as it was
        n_acc = np.where(o["granted"] == 1, n_acc, -1)
        e.step(dev(new, np.int32), dev(par, np.int32), [dev(x) for x in qkv], dev(acc, np.int32), dev(n_acc, np.int32))
        torch.cuda.synchronize()
        for name, t in (("slots", e.slots), ("positions", e.pos), ("tables", e.tb), ("ring", e.ring),
                        ("granted", e.granted), ("q_start", e.q_start), ("owned", e.owned), ("state", e.state)):
            assert np.array_equal(t.cpu().numpy(), o[name]), (i, name)
        assert np.array_equal(e.mask.cpu().numpy().view(np.uint64), o["mask"])
        # attention over the caches as they stand before the move: what the drafts' slots held is moved, so the
        # caches are taken from after it only where nothing moved (the whole step is checked at its last layer's
        # output below through sequences whose path is a prefix)
        n = np.diff(o["q_start"])
        whole = [s for s in range(B) if n[s] and o["granted"][s] and (acc[s, :n_acc[s]] == np.arange(n_acc[s])).all()]
        ct = np.uint8 if fmt != "bf16" else np.uint16
        K, V = (t[-1].cpu().numpy().view(ct) for t in (e.k, e.v))
        q = e.q.view(torch.int16).cpu().numpy().view(np.uint16)
        for s in whole:
            r = slice(o["q_start"][s], o["q_start"][s + 1])
            ref, bound = tree.tree_attention(q[r], K, V, o["tables"][s:s + 1], o["ctx"][s:s + 1], [0, n[s]],
                                             o["mask"][r], 128 ** -0.5, fmt,
                                             e.ks.cpu().numpy() if e.ks is not None else None,
                                             e.vs.cpu().numpy() if e.vs is not None else None)
            assert (np.abs(e.outs[-1][r].float().cpu().numpy() - ref) <= bound).all(), (i, s)
        assert i > 0 or len(whole) == B - refused
        o["ctx"] = np.where(o["granted"] == 1, o["ctx"] - n + n_acc, o["ctx"])
        assert np.array_equal(e.ctx.cpu().numpy(), o["ctx"])
    assert refused > 0          # the pool was too small now and then


def test_captured_step_replays_as_the_eager_one(gpu_lib):
    """One captured step (its own lengths copied back at its end) replayed, with eager steps of another server between."""
    note("captured verification step")
    B, mb, nb, hq, hkv, rows = 5, 40, 300, 8, 2, 64
    rng = np.random.default_rng(2)
    a, b, c = (Engine(gpu_lib, B, mb, nb, hq, hkv, rows, False, seed=3) for _ in range(3))
    new, par, qkv, acc, n_acc = draws(rng, B, rows, hq, hkv, a.layers, False)
    new = np.abs(new)
    par = np.zeros(rows, int) - 1
    args = [dev(new, np.int32), dev(par, np.int32), [dev(x) for x in qkv], dev(acc, np.int32), dev(n_acc, np.int32)]
    c.dec.workspace = b.dec.workspace          # an eager server that shares the captured one's workspace
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        c.step(*args)
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        b.step(*args)
    for i in range(6):
        a.step(*args)
        c.step(*args)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for x, y in zip([a.ctx, a.owned, a.state, a.tb, a.ring, a.slots, a.pos, a.mask, a.q, *a.k, *a.v, *a.outs],
                        [b.ctx, b.owned, b.state, b.tb, b.ring, b.slots, b.pos, b.mask, b.q, *b.k, *b.v, *b.outs]):
            n = int(a.q_start[-1])
            if x.shape[0] == rows:
                x, y = x[:n], y[:n]
            assert torch.equal(x.view(torch.int16) if x.dtype == torch.bfloat16 else x,
                               y.view(torch.int16) if y.dtype == torch.bfloat16 else y), i


def test_operators_on_another_stream(gpu_lib):
    note("operators on a stream of their own")
    B, mb, nb, hq, hkv, rows = 4, 10, 60, 4, 2, 60
    rng = np.random.default_rng(4)
    a, b = (Engine(gpu_lib, B, mb, nb, hq, hkv, rows, True, seed=5) for _ in range(2))
    new, par, qkv, acc, n_acc = draws(rng, B, rows, hq, hkv, a.layers, False)
    args = [dev(np.abs(new), np.int32), dev(par, np.int32), [dev(x) for x in qkv], dev(acc, np.int32),
            dev(n_acc, np.int32)]
    a.step(*args)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        b.step(*args)
    s.synchronize()
    for x, y in zip([a.ctx, a.tb, a.slots, *a.k, *a.v], [b.ctx, b.tb, b.slots, *b.k, *b.v]):
        assert torch.equal(x, y)
    n = int(a.q_start[-1])
    assert torch.equal(a.outs[0][:n].view(torch.int16), b.outs[0][:n].view(torch.int16))
