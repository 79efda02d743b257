"""qk_norm_rope_append (through the C ABI) against the oracle in float64.

Tolerances, from the arithmetic alone: every intermediate is float32 (half a
step 2^-24 of the value).  The norm's sum has 128 terms (136 roundings with
the mean, the root and the two products), a turned value is two products and
a sum: E = 140 * 2^-24 * (|a c| + |b s|).  A bf16 result adds 2^-8 of itself,
an e4m3 code 2^-4 of the value it stands for (2^-10 below the normal range).
V is moved or encoded by the append's rule: its codes must be equal.
"""
import numpy as np
import pytest
import torch

import workloads
from oracle import append, numerics, rope

pytestmark = pytest.mark.gpu


def note(msg):
    print(f"[gpu-test] {msg}", flush=True)


def codes(rng, *shape, scale=1.0):
    return workloads.to_bf16_codes((rng.standard_normal(shape) * scale).astype(np.float32))


def dev(a):
    a = np.ascontiguousarray(a)
    return torch.from_numpy(a.view(np.int16) if a.dtype == np.uint16 else a).cuda()


def host(t, like):
    return t.cpu().numpy().view(like.dtype)


def check(lib, rng, rows, hq, hkv, slots, pos, fmt="bf16", rotary=128, paired=False, weights=(True, True), fused=False,
          nb=40, n_pos=500, inplace=False, eps=1e-6, scale=1.0):
    qkv = codes(rng, rows, hq + 2 * hkv, 128, scale=scale)
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    table = rope.table(n_pos, rotary).astype(np.float32)
    w = [codes(rng, 128, scale=0.5) if on else None for on in weights]
    kt = np.uint16 if fmt == "bf16" else np.uint8
    kp = rng.integers(0, 100, (nb, hkv, 16, 128)).astype(kt)
    vp = rng.integers(0, 100, (nb, hkv, 128, 16)).astype(kt)
    ks = vs = None
    if fmt != "bf16":
        ks, vs = ((rng.random(hkv) * 0.05 + 0.004).astype(np.float32) for _ in range(2))
    slots, pos = np.asarray(slots, np.int64), np.asarray(pos, np.int32)
    if fused:
        big = dev(qkv).view(rows, -1)
        dq, dk, dv = big[:, :hq * 128], big[:, hq * 128:(hq + hkv) * 128], big[:, (hq + hkv) * 128:]
    else:
        dq, dk, dv = (dev(t).view(rows, -1) for t in (q, k, v))
    out = dq if inplace else torch.full((rows, hq, 128), 77, dtype=torch.int16, device="cuda")
    dkp, dvp = dev(kp), dev(vp)
    sh = lib.qk_shape(rows, hq, hkv, nb, n_pos, rotary, paired, fmt != "bf16", dq.stride(0), dk.stride(0), dv.stride(0))
    lib.qk_norm_rope_append(dq, dk, dv, dev(table) if rotary else None, dev(pos), dev(slots), out, dkp, dvp, sh,
                            *[dev(x) if x is not None else None for x in w], eps,
                            dev(ks) if ks is not None else None, dev(vs) if vs is not None else None)
    torch.cuda.synchronize()
    got_q, got_k, got_v = host(out, q).reshape(rows, hq, 128), host(dkp, kp), host(dvp, vp)

    live = (pos >= 0) & (pos < n_pos)
    t = table[np.where(live, pos, 0)].astype(np.float64)
    cos, sin = t[:, :rotary // 2], t[:, rotary // 2:]
    res = []
    for x, wt in ((q, w[0]), (k, w[1])):
        y = rope.norm(numerics.decode_bf16(x), numerics.decode_bf16(wt) if wt is not None else None, eps)
        res.append((rope.turn(y, cos, sin, paired), 140 * 2.0 ** -24 * rope.turn(np.abs(y), np.abs(cos), -np.abs(sin), paired)))
    (rq, eq), (rk, ek) = res
    eq, ek = np.abs(eq), np.abs(ek)
    # the second member of a pair came out as |b c| - |a s| above: take the sum
    for (r, e), x in zip(((rq, eq), (rk, ek)), (0, 1)):
        e += 140 * 2.0 ** -24 * 2 * np.abs(r).max(axis=-1, keepdims=True)
    err = np.abs(numerics.decode_bf16(got_q) - rq)
    assert (err[live] <= (eq + 2.0 ** -8 * np.abs(rq))[live]).all()
    before = q if inplace else np.full_like(got_q, 77)
    assert np.array_equal(got_q[~live], before[~live])
    # caches: untouched but for the live rows' slots
    ok = live & (slots >= 0) & (slots < nb * 16)
    want_v, k_mine = np.array(vp, copy=True), np.zeros((nb, 16), bool)
    for r in np.flatnonzero(ok):
        b, o = int(slots[r]) // 16, int(slots[r]) % 16
        k_mine[b, o] = True
        for g in range(hkv):
            want_v[b, g, :, o] = append.encode(v[r, g], fmt, None if vs is None else vs[g])
            got = numerics.decode(got_k[b, g, o], fmt)
            if fmt == "bf16":
                assert (np.abs(got - rk[r, g]) <= ek[r, g] + 2.0 ** -8 * np.abs(rk[r, g])).all()
            else:
                z = rk[r, g] / float(ks[g])
                cut = np.clip(z, -448, 448)
                lim = np.maximum(2.0 ** -4 * np.abs(cut), 2.0 ** -10) + 2 * ek[r, g] / ks[g]
                assert (np.abs(got - cut) <= lim).all()
    assert np.array_equal(got_v, want_v)
    same = np.broadcast_to(~k_mine[:, None, :, None], kp.shape)
    assert np.array_equal(got_k[same], kp[same])


def scattered(rng, rows, nb, n_pos):
    return rng.permutation(nb * 16)[:rows], rng.integers(0, n_pos, rows)


@pytest.mark.parametrize("fmt", ["bf16", "fp8_e4m3"])
@pytest.mark.parametrize("rows,hq,hkv", [(1, 1, 1), (1, 64, 8), (3, 5, 5), (19, 8, 2), (40, 7, 1), (130, 16, 4)])
def test_scattered_rows(gpu_lib, rows, hq, hkv, fmt):
    note(f"rope rows={rows} heads={hq}/{hkv} {fmt}")
    rng = np.random.default_rng(rows + hq)
    check(gpu_lib, rng, rows, hq, hkv, *scattered(rng, rows, 40, 500), fmt=fmt)


@pytest.mark.parametrize("rotary", [0, 16, 64, 112, 128])
@pytest.mark.parametrize("paired", [False, True])
@pytest.mark.parametrize("weights", [(True, True), (False, False), (True, False), (False, True)])
def test_rotations_and_norms(gpu_lib, rotary, paired, weights):
    note(f"rope rotary={rotary} paired={paired} norms={weights}")
    rng = np.random.default_rng(rotary)
    check(gpu_lib, rng, 21, 6, 2, *scattered(rng, 21, 40, 500), rotary=rotary, paired=paired, weights=weights,
          fused=paired)


@pytest.mark.parametrize("fmt", ["bf16", "fp8_e4m3"])
@pytest.mark.parametrize("starts", [[(0, 100)], [(5, 60), (0, 33), (15, 2)], [(0, 16), (16, 16), (3, 13), (9, 40)],
                                    [(1, 1)] * 12, [(7, 300), (0, 250)]])
def test_runs_of_rows(gpu_lib, starts, fmt):
    """Prompts and drafts: rows of consecutive slots, from any offset, over blocks in any order."""
    note(f"rope runs {starts} {fmt}")
    rng = np.random.default_rng(len(starts))
    nb = 60
    ids = rng.permutation(nb).tolist()
    slots, pos = [], []
    for c, n in starts:
        blocks = [ids.pop() for _ in range(-(-(c + n) // 16))]
        slots += [blocks[t // 16] * 16 + t % 16 for t in range(c, c + n)]
        pos += range(c, c + n)
    check(gpu_lib, rng, len(slots), 4, 3, slots, pos, fmt=fmt, nb=nb, fused=True)
    # a hole within, rows in no slot, and a padded end
    slots[0] = -1
    pos[len(pos) // 2] = -1
    check(gpu_lib, rng, len(slots) + 9, 4, 3, slots + [-1] * 5 + [nb * 16] * 4, pos + [-1] * 5 + [3] * 4, fmt=fmt,
          nb=nb)
    # adjacent blocks whose slots follow each other
    check(gpu_lib, rng, 50, 2, 3, list(range(70, 120)), list(range(50)), fmt=fmt, nb=nb)


@pytest.mark.parametrize("rows", [700, 5000])
def test_many_rows(gpu_lib, rows):
    note(f"rope rows={rows}")
    rng = np.random.default_rng(rows)
    nb = rows // 16 + 30
    half = rows // 2
    slots = np.concatenate([np.arange(5, 5 + half), rng.permutation(np.arange(half + 20, nb * 16))[:rows - half]])
    check(gpu_lib, rng, rows, 3, 2, slots, rng.integers(0, 500, rows), nb=nb, fmt="fp8_e4m3" if rows > 1000 else "bf16")


def test_in_place_and_far_positions(gpu_lib):
    note("rope in place, far positions")
    rng = np.random.default_rng(9)
    pos = rng.integers(0, 131072, 33)
    pos[:4] = [0, 131071, 131072, -1]
    check(gpu_lib, rng, 33, 8, 2, rng.permutation(640)[:33], pos, inplace=True, n_pos=131072)


@pytest.mark.parametrize("scale", [0.0, 1e-4, 1e4])
def test_small_and_large_values(gpu_lib, scale):
    note(f"rope values {scale}")
    rng = np.random.default_rng(10)
    check(gpu_lib, rng, 12, 4, 2, *scattered(rng, 12, 40, 500), scale=scale)
    check(gpu_lib, rng, 12, 4, 2, *scattered(rng, 12, 40, 500), scale=scale, fmt="fp8_e4m3", weights=(False, False))


def test_infinities_stay_in_their_head(gpu_lib):
    note("rope, values that are not finite")
    rng = np.random.default_rng(11)
    rows, hq, hkv, nb = 9, 4, 2, 20
    q, k, v = codes(rng, rows, hq, 128), codes(rng, rows, hkv, 128), codes(rng, rows, hkv, 128)
    q[3, 1, 100], k[5, 0, 127], v[2, 1, 7] = 0x7F80, 0x7FC0, 0x7F80
    outs = []
    for bad in (True, False):
        if not bad:
            q[3, 1, 100], k[5, 0, 127], v[2, 1, 7] = 0, 0, 0
        out, kp, vp = dev(np.zeros_like(q)), dev(np.zeros((nb, hkv, 16, 128), np.uint16)), dev(
            np.zeros((nb, hkv, 128, 16), np.uint16))
        gpu_lib.qk_norm_rope_append(dev(q), dev(k), dev(v), dev(rope.table(99, 64).astype(np.float32)),
                                    dev(np.arange(rows, dtype=np.int32)), dev(np.arange(rows, dtype=np.int64) * 17),
                                    out, kp, vp, gpu_lib.qk_shape(rows, hq, hkv, nb, 99, 64))
        torch.cuda.synchronize()
        outs.append([t.cpu().numpy() for t in (out, kp, vp)])
    (a, ak, av), (b, bk, bv) = outs
    diff = np.argwhere(a != b)
    assert diff.tolist() == [[3, 1, 100]]            # without a norm, dimension 100 is not turned
    assert (np.argwhere(ak != bk)[:, :3] == [85 // 16, 0, 85 % 16]).all()
    assert np.argwhere(av != bv).tolist() == [[34 // 16, 1, 7, 34 % 16]]


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("rows", [1, 37, 300, 4200])
def test_nan_stays_nan_in_an_e4m3_cache(gpu_lib, rows, norm):
    """A NaN, given or made by the norm of an infinity, is stored as a NaN code; an infinity as the largest value."""
    note(f"rope, NaN into an e4m3 cache, rows={rows} norm={norm}")
    rng = np.random.default_rng(rows)
    hq, hkv, nb = 2, 3, rows // 16 + 3
    q, k, v = codes(rng, rows, hq, 128), codes(rng, rows, hkv, 128), codes(rng, rows, hkv, 128)
    hit = rng.choice(rows, min(rows, 40), replace=False)
    for i, r in enumerate(hit):
        k[r, i % hkv, int(rng.integers(0, 128))] = (0x7FC0, 0x7F80, 0xFF80)[i % 3]
        v[r, i % hkv, int(rng.integers(0, 128))] = (0xFFC0, 0x7F80, 0xFF80)[i % 3]
    w = codes(rng, 128) if norm else None
    ks, vs = ((rng.random(hkv) * 0.05 + 0.01).astype(np.float32) for _ in range(2))
    table = rope.table(rows, 64).astype(np.float32)
    pos, slots = np.arange(rows, dtype=np.int32), np.arange(3, rows + 3, dtype=np.int64)
    kp, vp = dev(np.zeros((nb, hkv, 16, 128), np.uint8)), dev(np.zeros((nb, hkv, 128, 16), np.uint8))
    out = dev(np.zeros_like(q))
    gpu_lib.qk_norm_rope_append(dev(q), dev(k), dev(v), dev(table), dev(pos), dev(slots), out, kp, vp,
                                gpu_lib.qk_shape(rows, hq, hkv, nb, rows, 64, kv_fp8=True), None,
                                dev(w) if norm else None, 1e-6, dev(ks), dev(vs))
    torch.cuda.synchronize()
    t = table.astype(np.float64)
    with np.errstate(invalid="ignore"):
        want_k = rope.turn(rope.norm(numerics.decode_bf16(k), numerics.decode_bf16(w) if norm else None, 1e-6),
                           t[:, :32], t[:, 32:]) / ks.astype(np.float64)[:, None]
        want_v = numerics.decode_bf16(v) / vs.astype(np.float64)[:, None]
    assert np.isnan(want_k).any() and np.isnan(want_v).any()
    s = slots
    got_k = kp.cpu().numpy()[s // 16, :, s % 16]
    got_v = vp.cpu().numpy()[s // 16, :, :, s % 16]
    for got, want in ((got_k, want_k), (got_v, want_v)):
        assert np.array_equal((got & 0x7F) == 0x7F, np.isnan(want))
        big = np.isinf(want)
        assert np.array_equal(got[big], np.where(want[big] < 0, 0xFE, 0x7E))
