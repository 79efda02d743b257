"""Attention over a sliding window with visible first tokens, and over a cache with block scales, in float64.

Test infrastructure only (see the package header).

What is computed.  Query row i of a sequence with T cached tokens and n query
rows sits at position p = T - n + i (decode: n = 1) and sees the tokens

    p - window < t <= p,  and  t < n_sink (t <= p):
    z_t = scale * q_i . K_t,  out_i = sum_t exp(z_t - max z) V_t / sum_t exp(z_t - max z)

A row that sees no token (T = 0), or whose scores are all -infinity, gives
zeros.  K, V, heads and block tables are as for the decode oracle.

Block scales.  In a cache of format "e4m3_block" every (block, KV head) tile
has an exponent byte e, and its values are code * 2^(e - 127) (OCP E8M0; 255
is NaN).  ``append_scaled`` restates how tokens enter such a cache: the rows of
one block form a run; with a the largest finite magnitude among them and s0
the block's first slot they write,

    need = smallest power of two with a <= 448 * need (bytes 1 .. 246)
    new  = max(old, need) if s0 > 0, else need
    slots before s0:  codes re-encoded, code * old / new rounded
    the run's slots:  value / new rounded to e4m3, NaN where it is not finite

Parity: a window as long as the context and no sinks is pinned by the decode
and chunked-prefill oracles, the mask by brute-force loops, hidden tokens by
tokens that hold NaN; the byte of a magnitude by a search over all bytes.
"""
from __future__ import annotations

import numpy as np

from . import numerics
from .append import e4m3_encode
from .attention import _gather_rows

BF16_HALF = 2.0 ** -8     # half a step of bf16, relative
F32_HALF = 2.0 ** -24
BYTE_LO, BYTE_HI = 1, 246


def pow2(byte):
    """The values of E8M0 bytes."""
    b = np.asarray(byte).astype(np.float64)
    return np.where(b == 255, np.nan, 2.0 ** (b - 127.0))


def sees(T, n, window, n_sink):
    """bool [n, T]: which cached tokens each of the last n sees."""
    t, p = np.arange(T)[None, :], (T - n + np.arange(n))[:, None]
    return (t <= p) & ((t > p - window) | (t < n_sink))


def window_attention(q_bits, k_pool, v_pool, block_tables, context_lens, q_start, scale, window, n_sink,
                     kv_format="bf16", k_scale=None, v_scale=None, block_size=16):
    """(out, bound): float64 [total_q, Hq, D]; rows of no sequence are NaN.  q_start None: one row a sequence.

    bound: how far a computation may be off that rounds the probabilities to
    bf16 against running references (numerator and denominator alike), keeps
    everything else in float32 and rounds the result to bf16:
      probabilities: each off by BF16_HALF of itself and by twice the error of
        its score; the sums' quotient moves by at most that times sum p |v - o|;
      scores: D + 8 float32 roundings of sum |q k| scale, and of the score;
      sums of m terms in float32, in some order: (m + 8) roundings of sum p |v|;
      the result: BF16_HALF of itself.
    Second-order terms and exp2 (an ulp or two) are covered by a factor 1.25.
    """
    q = numerics.decode_bf16(q_bits)
    total_q, Hq, D = q.shape
    Hkv = k_pool.shape[1]
    G = Hq // Hkv
    if q_start is None:
        rows = [(s, s + 1 if context_lens[s] > 0 else s) for s in range(len(context_lens))]
    else:
        rows = [(int(q_start[s]), int(q_start[s + 1])) for s in range(len(q_start) - 1)]
    out = np.full((total_q, Hq, D), np.nan)
    bound = np.zeros_like(out)
    fmt = "fp8_e4m3" if kv_format == "e4m3_block" else kv_format
    for s, (r0, r1) in enumerate(rows):
        n, T = r1 - r0, int(context_lens[s])
        if q_start is None and T == 0:
            out[r0] = 0.0
        if n == 0:
            continue
        if n > T:
            raise ValueError(f"sequence {s}: {n} rows of {T} tokens")
        see = sees(T, n, window, n_sink)
        bt = np.asarray(block_tables[s])
        some = see.any(0)
        ids = np.where(bt < 0, 0, bt)      # (entries of blocks that no row sees may hold anything)
        for g in range(Hkv):
            K = numerics.decode(_gather_rows(k_pool, ids, g, T, block_size, False), fmt)
            V = numerics.decode(_gather_rows(v_pool, ids, g, T, block_size, True), fmt)
            if kv_format == "e4m3_block":
                blk = ids[np.arange(T) // block_size]
                K, V = K * pow2(k_scale[blk, g])[:, None], V * pow2(v_scale[blk, g])[:, None]
            elif k_scale is not None:
                K, V = K * float(k_scale[g]), V * float(v_scale[g])
            hs = slice(g * G, (g + 1) * G)
            for i in range(n):
                t = np.flatnonzero(see[i] & some)
                with np.errstate(invalid="ignore", over="ignore"):
                    z = scale * (q[r0 + i, hs] @ K[t].T)                       # [G, m]
                    top = z.max(axis=1, keepdims=True)
                    p = np.exp(z - np.where(np.isneginf(top), 0.0, top))
                    tot = p.sum(axis=1, keepdims=True)
                    p = np.where(tot == 0, 0.0, p / np.where(tot == 0, 1.0, tot))
                    o = np.stack([np.where(w != 0, w, 0) @ V[t] if np.isfinite(V[t]).all() else
                                  (w[w != 0] @ V[t][w != 0]) for w in p])
                    dz = F32_HALF * ((D + 8) * abs(scale) * (np.abs(q[r0 + i, hs]) @ np.abs(K[t]).T) + 4 * np.abs(z))
                    dz = np.where(np.isneginf(z), 0.0, dz).max(axis=1)   # (what has no weight has no error)
                    far = np.einsum("gm,gmd->gd", p, np.abs(V[t][None] - o[:, None]))
                    out[r0 + i, hs] = o
                    bound[r0 + i, hs] = 1.25 * ((BF16_HALF + 2 * dz)[:, None] * far + BF16_HALF * np.abs(o)
                                                + F32_HALF * (len(t) + 8) * (p @ np.abs(V[t])))
    return out, bound + 1e-30


def need_byte(a):
    """The smallest byte in [BYTE_LO, BYTE_HI] with a <= 448 * 2^(byte - 127); BYTE_HI if none."""
    for b in range(BYTE_LO, BYTE_HI):
        if a <= 448.0 * 2.0 ** (b - 127):
            return b
    return BYTE_HI


def encode_block(x, byte):
    """e4m3 codes of float64 values over 2^(byte - 127): nearest, ties to even, NaN where not finite."""
    fine = np.isfinite(x)
    code = e4m3_encode(np.where(fine, x, 0.0) * 2.0 ** (127.0 - byte))
    return np.where(fine, code, 0x7F).astype(np.uint8)


def append_scaled(k_new, v_new, k_pool, v_pool, k_scale, v_scale, slots, block_size=16):
    """(k_pool, v_pool, k_scale, v_scale) after the rows are in; k_new, v_new float64 [rows, Hkv, D].

    slots[r] < 0: row r goes nowhere.  Rows of one block lie next to each
    other, their slots rising."""
    pools = [np.array(k_pool, copy=True), np.array(v_pool, copy=True)]
    scales = [np.array(k_scale, copy=True), np.array(v_scale, copy=True)]
    rows, hkv, _ = k_new.shape
    r = 0
    while r < rows:
        if slots[r] < 0 or slots[r] >= block_size * k_pool.shape[0]:
            r += 1
            continue
        blk, s0, end = int(slots[r]) // block_size, int(slots[r]) % block_size, r + 1
        while end < rows and end - r < block_size and slots[end] >= 0 and int(slots[end]) // block_size == blk:
            end += 1
        for x, pool, scale, token_major in ((k_new, pools[0], scales[0], True), (v_new, pools[1], scales[1], False)):
            for g in range(hkv):
                tile = pool[blk, g] if token_major else pool[blk, g].T      # [16, D], a view
                new = x[r:end, g]
                old = int(scale[blk, g]) if s0 > 0 else 0
                byte = max(old, need_byte(np.abs(new[np.isfinite(new)]).max(initial=0.0)))
                if s0 > 0 and byte != old:
                    keep = numerics.decode_e4m3(np.ascontiguousarray(tile[:s0])) * pow2(old)
                    tile[:s0] = encode_block(keep, byte)
                tile[[int(slots[i]) % block_size for i in range(r, end)]] = encode_block(new, byte)
                scale[blk, g] = byte
        r = end
    return pools[0], pools[1], scales[0], scales[1]
