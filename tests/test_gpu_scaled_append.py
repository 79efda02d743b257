"""qk_norm_rope_append_scaled (through the C ABI) against the oracle in float64.

V enters as it is: its codes and scales must be equal to the oracle's.  K is
normed and turned in float32 first, off by at most E = 140 * 2^-24 of the
pair's magnitudes (as for qk_norm_rope_append); its scale's byte must be the
one of a largest magnitude within E of the true one, its codes off by half a
step of e4m3 (2^-4 of the value, 2^-10 of the scale below the normal range)
and E, and codes of earlier tokens must be the exact re-encoding between the
two bytes.  Queries: E and half a step of bf16.
"""
import numpy as np
import pytest
import torch

import window_cases as wc
import workloads
from oracle import numerics, rope
from oracle import window as ow
from window_cases import dev

pytestmark = pytest.mark.gpu


def note(msg):
    print(f"[gpu-test] {msg}", flush=True)


def runs_of(slots, nb):
    r, out = 0, []
    while r < len(slots):
        end = r + 1
        if 0 <= slots[r] < 16 * nb:
            while end < len(slots) and slots[end] >= 0 and slots[end] // 16 == slots[r] // 16 and end - r < 16:
                end += 1
            out.append((r, end))
        r = end
    return out


def check(lib, rng, slots, pos, hq=4, hkv=2, rotary=128, paired=False, weights=(True, True), fused=False, nb=40,
          n_pos=500, eps=1e-6, codes=None, byte_range=(118, 124), repeat=1, inplace=False):
    slots, pos = np.asarray(slots, np.int64), np.asarray(pos, np.int32)
    rows = len(slots)
    if codes is None:
        x = rng.standard_normal((rows, hq + 2 * hkv, 128)) * np.exp(rng.standard_normal((rows, hq + 2 * hkv, 1)))
        codes = workloads.to_bf16_codes(x.astype(np.float32))
    q, k, v = codes[:, :hq], codes[:, hq:hq + hkv], codes[:, hq + hkv:]
    table = rope.table(n_pos, rotary).astype(np.float32)
    w = [workloads.to_bf16_codes((rng.standard_normal(128) * 0.5).astype(np.float32)) if on else None for on in weights]
    kp, vp = (rng.integers(0, 256, (nb, hkv) + d).astype(np.uint8) for d in ((16, 128), (128, 16)))
    ks, vs = (rng.integers(*byte_range, (nb, hkv)).astype(np.uint8) for _ in range(2))
    if fused:
        big = dev(codes).view(rows, -1)
        dq, dk, dv = (t.view(rows, -1, 128) for t in big.split([hq * 128, hkv * 128, hkv * 128], dim=1))
    else:
        dq, dk, dv = (dev(t) for t in (q, k, v))
    out = None if hq == 0 else dq if inplace else torch.full((rows, hq, 128), 77, dtype=torch.int16, device="cuda")
    dkp, dvp, dks, dvs = (dev(t) for t in (kp, vp, ks, vs))
    sh = lib.qk_shape(rows, hq, hkv, nb, n_pos, rotary, paired, q_stride=dq.stride(0) if hq else 0, block_scales=True,
                      k_stride=dk.stride(0), v_stride=dv.stride(0))
    for _ in range(repeat):
        lib.qk_norm_rope_append_scaled(dq if hq else None, dk, dv, dev(table) if rotary else None, dev(pos), dev(slots),
                                       out, dkp, dvp, dks, dvs, sh, *[dev(x) if x is not None else None for x in w], eps)
    torch.cuda.synchronize()
    gk, gv, gks, gvs = (t.cpu().numpy() for t in (dkp, dvp, dks, dvs))

    live = (pos >= 0) & (pos < n_pos)
    t = table[np.where(live, pos, 0)].astype(np.float64)
    cos, sin = t[:, :rotary // 2], t[:, rotary // 2:]
    res = []
    with np.errstate(invalid="ignore", over="ignore"):
        for x, wt in ((q, w[0]), (k, w[1])):
            y = rope.norm(numerics.decode_bf16(x), numerics.decode_bf16(wt) if wt is not None else None, eps)
            r = rope.turn(y, cos, sin, paired)
            res.append((r, 140 * 2.0 ** -24 * 3 * np.abs(np.where(np.isfinite(y), y, 0)).max(axis=-1, keepdims=True)))
    (rq, eq), (rk, ek) = res
    if hq:
        gq = out.cpu().numpy().view(np.uint16).reshape(rows, hq, 128)
        err, fine = np.abs(numerics.decode_bf16(gq) - rq), np.isfinite(rq)
        assert (err <= eq + 2.0 ** -8 * np.abs(rq))[live & fine.all((1, 2))].all()
        before = q if inplace else np.full_like(gq, 77)
        assert np.array_equal(gq[~live], before[~live])
    where = np.where(live, slots, -1)
    _, wv, _, wvs = ow.append_scaled(rk, numerics.decode_bf16(v), kp, vp, ks, vs, where)
    assert np.array_equal(gvs, wvs)
    nan = (wv & 0x7F) == 0x7F
    assert np.array_equal(gv[~nan], wv[~nan]) and ((gv[nan] & 0x7F) == 0x7F).all()
    want, want_s = kp.copy(), ks.copy()
    for r0, r1 in runs_of(where, nb):
        blk, s0 = int(where[r0]) // 16, int(where[r0]) % 16
        for g in range(hkv):
            y, e = rk[r0:r1, g], ek[r0:r1, g]
            fine, old = np.isfinite(y), int(ks[blk, g]) if s0 else 0
            a = np.where(fine, np.abs(y), 0)
            byte = int(gks[blk, g])
            lo = max(max(ow.need_byte(x) for x in (a - e).max(axis=1)), old)
            hi = max(max(ow.need_byte(x) for x in (a + e).max(axis=1)), old)
            assert lo <= byte <= hi
            want_s[blk, g] = byte
            if s0 and byte != old:
                want[blk, g, :s0] = ow.encode_block(numerics.decode_e4m3(kp[blk, g, :s0]) * ow.pow2(old), byte)
            at = [int(s) % 16 for s in where[r0:r1]]
            got = numerics.decode_e4m3(gk[blk, g, at])
            cut = np.clip(np.where(fine, y, 0) * 2.0 ** (127 - byte), -448, 448)
            lim = np.maximum(2.0 ** -4 * np.abs(cut), 2.0 ** -10) + 2 * e * 2.0 ** (127 - byte)
            assert (np.abs(got - cut) <= lim)[fine].all() and np.isnan(got[~fine]).all()
            want[blk, g, at] = gk[blk, g, at]
    assert np.array_equal(gks, want_s)
    nan = (want & 0x7F) == 0x7F
    assert np.array_equal(gk[~nan], want[~nan]) and ((gk[nan] & 0x7F) == 0x7F).all()


def sequences(rng, specs, nb, n_pos):
    """Slots and positions of sequences (cached, new): blocks of a shuffled pool, in order."""
    perm, at, slots, pos = rng.permutation(nb), 0, [], []
    for c, n in specs:
        ids = perm[at:at + -(-(c + n) // 16)]
        at += len(ids)
        t = np.arange(c, c + n)
        slots.append(ids[t // 16] * 16 + t % 16)
        pos.append(t % n_pos)
    return np.concatenate(slots), np.concatenate(pos)


@pytest.mark.parametrize("rows,hq,hkv", [(1, 1, 1), (1, 64, 8), (3, 5, 5), (19, 8, 2), (33, 7, 1), (37, 16, 4)])
def test_single_tokens(gpu_lib, rows, hq, hkv):
    note(f"scaled append single tokens rows={rows} heads={hq}/{hkv}")
    rng = np.random.default_rng(rows + hq)
    slots = rng.permutation(40)[:rows] * 16 + rng.integers(0, 16, rows)
    check(gpu_lib, rng, slots, rng.integers(0, 500, rows), hq, hkv)


@pytest.mark.parametrize("specs", [
    [(0, 16)], [(0, 1)], [(15, 1)], [(15, 2)], [(3, 40)], [(16, 16), (0, 48), (5, 11), (5, 12)], [(7, 3)] * 9,
    [(0, 300)], [(i, 17) for i in range(17)]])
@pytest.mark.parametrize("paired", [False, True])
def test_runs(gpu_lib, specs, paired):
    note(f"scaled append runs {specs} paired={paired}")
    rng = np.random.default_rng(len(specs))
    check(gpu_lib, rng, *sequences(rng, specs, 60, 500), nb=60, paired=paired, fused=paired)


@pytest.mark.parametrize("rotary", [0, 16, 64, 112, 128])
@pytest.mark.parametrize("paired", [False, True])
@pytest.mark.parametrize("weights", [(True, True), (False, False), (True, False), (False, True)])
def test_rotations_and_norms(gpu_lib, rotary, paired, weights):
    note(f"scaled append rotary={rotary} paired={paired} norms={weights}")
    rng = np.random.default_rng(rotary)
    check(gpu_lib, rng, *sequences(rng, [(3, 20), (15, 1), (0, 9)], 40, 500), hq=6, rotary=rotary, paired=paired,
          weights=weights, fused=paired)


@pytest.mark.parametrize("batch,new", [(300, 1), (90, 7), (5, 900), (300, 16)])
def test_launch_sizes(gpu_lib, batch, new):
    """Rows up to 256, up to 4,095 and beyond take other work splits."""
    note(f"scaled append {batch} sequences of {new}")
    rng = np.random.default_rng(batch)
    specs = [(int(c), new) for c in rng.integers(0, 40, batch)]
    nb = sum(-(-(c + n) // 16) for c, n in specs) + 3
    check(gpu_lib, rng, *sequences(rng, specs, nb, 500), hq=3, hkv=1, nb=nb)


@pytest.mark.parametrize("hq,hkv,rows", [(0, 2, 20), (0, 1, 1)])
def test_keys_and_values_only(gpu_lib, hq, hkv, rows):
    note("scaled append without queries")
    rng = np.random.default_rng(3)
    check(gpu_lib, rng, *sequences(rng, [(5, rows)], 40, 500), hq=0, hkv=hkv, rotary=0, weights=(False, False))


def test_dead_rows(gpu_lib):
    """Positions outside the table leave a row alone; slots outside the pool leave the cache alone."""
    note("scaled append dead rows")
    rng = np.random.default_rng(4)
    slots, pos = sequences(rng, [(2, 5), (9, 20), (0, 3)], 40, 500)
    pos, slots = pos.copy(), slots.copy()
    pos[[5, 6]], slots[[25, 26, 27]] = [-1, 500], [-1, 40 * 16, -9]
    check(gpu_lib, rng, slots, pos)
    check(gpu_lib, rng, slots, pos, inplace=True)


def test_scales_rise_by_steps_and_limits(gpu_lib):
    """Old bytes far below, at and far above what the new tokens need; zeros; the least and the largest values."""
    note("scaled append rising scales")
    rng = np.random.default_rng(5)
    slots, pos = sequences(rng, [(i % 16, 1 + i % 5) for i in range(30)], 80, 500)
    for lo, hi in ((1, 3), (60, 61), (110, 121), (127, 135), (244, 247)):
        check(gpu_lib, rng, slots, pos, nb=80, byte_range=(lo, hi), weights=(False, False))
    shape = (len(slots), 8, 128)
    for mag in (0.0, 2.0 ** -130, 2.0 ** -120, 3.5, 448.0, 2.0 ** 100, 3e38):
        x = np.where(rng.random(shape) < 0.5, mag, -mag).astype(np.float32)
        check(gpu_lib, rng, slots, pos, nb=80, codes=workloads.to_bf16_codes(x), weights=(False, False), rotary=0)


def test_begun_blocks_of_the_largest_scales(gpu_lib):
    """2^126 and 2^127, whose inverses are the least normal value and below it."""
    note("scaled append largest scales")
    rng = np.random.default_rng(55)
    slots, pos = sequences(rng, [(1 + i % 15, 1 + i % 5) for i in range(30)], 80, 500)
    x = (rng.standard_normal((len(slots), 8, 128)) * 1e38).clip(-3e38, 3e38).astype(np.float32)
    for byte in (253, 254):
        check(gpu_lib, rng, slots, pos, nb=80, codes=workloads.to_bf16_codes(x), byte_range=(byte, byte + 1),
              weights=(False, False), rotary=0)


def test_values_that_are_not_finite(gpu_lib):
    note("scaled append NaN and infinities")
    rng = np.random.default_rng(6)
    slots, pos = sequences(rng, [(0, 5), (3, 20), (8, 1)], 40, 500)
    codes = workloads.to_bf16_codes(rng.standard_normal((len(slots), 8, 128)).astype(np.float32))
    for r, h, d, c in ((0, 4, 3, 0x7FC0), (7, 5, 100, 0x7F80), (7, 6, 1, 0xFF80), (8, 7, 2, 0x7F80), (25, 6, 0, 0xFFC1)):
        codes[r, h, d] = c
    check(gpu_lib, rng, slots, pos, codes=codes, weights=(False, False), rotary=0)
    codes[25, 4:] = 0x7F80                        # nothing finite at all
    check(gpu_lib, rng, slots, pos, codes=codes, weights=(False, False), rotary=0)


def test_repeated_calls_change_nothing(gpu_lib):
    note("scaled append repeated")
    rng = np.random.default_rng(7)
    x = rng.standard_normal((30, 8, 128)).astype(np.float32) * 0.01
    slots, pos = sequences(rng, [(0, 13), (16, 17)], 40, 500)
    # (a scale that the first call raised stays: earlier tokens are encoded anew once)
    check(gpu_lib, rng, slots, pos, codes=workloads.to_bf16_codes(x), repeat=3)


def test_tokens_one_by_one_or_at_once(gpu_lib):
    """A block filled token by token holds what a block written at once holds: the same scale, and codes that
    differ where an earlier rounding was below the final scale's normal range only."""
    note("scaled append one by one")
    rng = np.random.default_rng(8)
    lib, hkv, n = gpu_lib, 2, 16
    x = workloads.to_bf16_codes((rng.standard_normal((n, 2 * hkv, 128)) * np.exp(rng.standard_normal((n, 1, 1))))
                                .astype(np.float32))
    outs = []
    for step in (1, n):
        k, v = (torch.zeros((1, hkv) + d, dtype=torch.uint8, device="cuda") for d in ((16, 128), (128, 16)))
        ks, vs = (torch.full((1, hkv), 200, dtype=torch.uint8, device="cuda") for _ in range(2))
        for i in range(0, n, step):
            part = dev(x[i:i + step])
            sh = lib.qk_shape(step, 0, hkv, 1, 16, rotary_dim=0, block_scales=True)
            at = torch.arange(i, i + step, device="cuda")
            lib.qk_norm_rope_append_scaled(None, part[:, :hkv].contiguous(), part[:, hkv:].contiguous(), None, at.int(),
                                           at, None, k, v, ks, vs, sh)
        torch.cuda.synchronize()
        outs.append([t.cpu().numpy() for t in (k, v.transpose(2, 3).contiguous(), ks, vs)])
    (k1, v1, ks1, vs1), (k2, v2, ks2, vs2) = outs
    assert np.array_equal(ks1, ks2) and np.array_equal(vs1, vs2)
    for a, b in ((k1, k2), (v1, v2)):
        a, b = numerics.decode_e4m3(a), numerics.decode_e4m3(b)
        normal = np.abs(b) >= 2.0 ** -6
        assert np.array_equal(a[normal], b[normal])
        assert np.abs(a - b).max() <= 2.0 ** -9


def test_captured_and_replayed(gpu_lib):
    note("scaled append graph")
    rng = np.random.default_rng(9)
    lib, hq, hkv, nb = gpu_lib, 4, 2, 20
    slots, pos = sequences(rng, [(3, 5), (0, 20), (15, 1)], nb, 500)
    codes = dev(workloads.to_bf16_codes(rng.standard_normal((len(slots), 8, 128)).astype(np.float32)))
    q, k, v = codes[:, :hq].contiguous(), codes[:, hq:hq + hkv].contiguous(), codes[:, hq + hkv:].contiguous()
    table = dev(rope.table(500, 128).astype(np.float32))
    ds, dp = dev(slots), dev(pos.astype(np.int32))
    first = [torch.randint(0, 120, (nb, hkv) + d, dtype=torch.uint8, device="cuda") for d in ((16, 128), (128, 16), (), ())]
    state, out = [t.clone() for t in first], torch.zeros_like(q)
    sh = lib.qk_shape(len(slots), hq, hkv, nb, 500, block_scales=True)

    def call():
        lib.qk_norm_rope_append_scaled(q, k, v, table, dp, ds, out, *state, sh)
    call()
    torch.cuda.synchronize()
    want = [t.clone() for t in state + [out]]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for _ in range(4):
        for t, f in zip(state, first):
            t.copy_(f)
        out.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for t, x in zip(state + [out], want):
            assert torch.equal(t, x)


@pytest.mark.parametrize("window,n_sink", [(64, 4), (5000, 0)])
def test_a_serving_run(gpu_lib, window, n_sink):
    """Prompts are written and attended, then tokens, one and a few at a time, each call's cache the next one's."""
    note(f"scaled append, prefill and decode in turn, window={window}")
    rng = np.random.default_rng(10)
    lib, hq, hkv, nb, n_pos, mb = gpu_lib, 8, 2, 60, 700, 30
    table = rope.table(n_pos, 128).astype(np.float32)
    perm = rng.permutation(nb).astype(np.int32)
    tables = np.stack([perm[:mb], perm[mb:2 * mb]])
    k, v = (torch.full((nb, hkv) + d, 0x7F, dtype=torch.uint8, device="cuda") for d in ((16, 128), (128, 16)))
    ks, vs = (torch.full((nb, hkv), 255, dtype=torch.uint8, device="cuda") for _ in range(2))
    ctx = np.zeros(2, np.int64)
    dec = lib.WindowDecoder(2, hq, hkv, mb, mb * 16, nb, window, n_sink, block_scales=True)
    dt = dev(tables)
    for new in ([150, 33], [1, 1], [1, 1], [5, 3], [1, 1], [40, 1], [1, 1]):
        rows = sum(new)
        seq = np.repeat([0, 1], new)
        t = np.concatenate([ctx[s] + np.arange(n) for s, n in enumerate(new)])
        slots = tables[seq, t // 16].astype(np.int64) * 16 + t % 16
        codes = workloads.to_bf16_codes(rng.standard_normal((rows, hq + 2 * hkv, 128)).astype(np.float32))
        big = dev(codes).view(rows, -1)
        dq, dk, dv = (x.view(rows, -1, 128) for x in big.split([hq * 128, hkv * 128, hkv * 128], dim=1))
        q = torch.empty((rows, hq, 128), dtype=torch.int16, device="cuda")
        sh = lib.qk_shape(rows, hq, hkv, nb, n_pos, q_stride=dq.stride(0), k_stride=dk.stride(0), v_stride=dv.stride(0),
                          block_scales=True)
        lib.qk_norm_rope_append_scaled(dq, dk, dv, dev(table), dev(t.astype(np.int32)), dev(slots), q, k, v, ks, vs, sh)
        ctx += new
        dctx = dev(ctx.astype(np.int32))
        out = torch.empty((rows, hq, 128), dtype=torch.bfloat16, device="cuda")
        q_start = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        if rows == 2:
            dec(q, k, v, dt, dctx, 0.088, out, ks, vs)
        else:
            psh = lib.prefill_shape(2, hq, hkv, mb, mb * 16, nb, rows, block_scales=True)
            lib.window_prefill_attention(q, k, v, dt, dctx, dev(q_start), 0.088, window, n_sink, out, psh, ks, vs)
        torch.cuda.synchronize()
        ref, bound = ow.window_attention(q.cpu().numpy().view(np.uint16), k.cpu().numpy(), v.cpu().numpy(), tables, ctx,
                                         q_start, 0.088, window, n_sink, "e4m3_block", ks.cpu().numpy(), vs.cpu().numpy())
        wc.check(out, ref, bound)
        # what was written is what the projections hold, to the rounding of e4m3
        for r in range(rows):
            b, o = int(slots[r]) // 16, int(slots[r]) % 16
            for g in range(hkv):
                want = numerics.decode_bf16(codes[r, hq + hkv + g])
                step = 2.0 ** (int(vs[b, g]) - 127)
                got = numerics.decode_e4m3(v[b, g, :, o].cpu().numpy()) * step
                assert (np.abs(got - want) <= np.maximum(2.0 ** -4 * np.abs(want), 2.0 ** -10 * step)).all()
