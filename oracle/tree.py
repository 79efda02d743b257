"""Attention of drafted trees over the paged cache, and the move of accepted drafts, in float64.

Test infrastructure only (see the package header).

What is computed.  Speculative decoding checks n drafted tokens of a sequence
in one pass; their K and V sit in the last n of its T cached tokens, and row i
sees the T - n committed tokens and every draft j whose bit is set in its mask:

    z_t = scale * q_i . K_t,  out_i = sum_t exp(z_t - max z) V_t / sum_t exp(z_t - max z)

over the tokens it sees; a row that sees none gives zeros.  K, V, heads and
block tables are as for the decode oracle.  Afterwards the accepted drafts'
K and V move to tokens T - n, T - n + 1, ...

Parity: with chain masks pinned by the chunked-prefill oracle, with one draft
by the decode oracle, with sparse masks by brute-force loops over dense
gathers, and by masked tokens that hold NaN.
"""
from __future__ import annotations

import numpy as np

from . import numerics
from .attention import _gather_rows

BF16_HALF = 2.0 ** -8     # half a step of bf16, relative
F32_HALF = 2.0 ** -24


def bits(mask, n):
    """bool [rows, n] of uint64 mask words [rows, w]."""
    mask = np.asarray(mask).view(np.uint64)
    j = np.arange(n)
    return ((mask[:, j // 64] >> (j % 64).astype(np.uint64)) & np.uint64(1)).astype(bool)


def tree_attention(q_bits, k_pool, v_pool, block_tables, context_lens, q_start, mask, scale, kv_format="bf16",
                   k_scale=None, v_scale=None, block_size=16):
    """(out, bound): float64 [total_q, Hq, D]; rows of no sequence are NaN.

    bound: how far a computation may be off that rounds the probabilities to
    bf16 against a running reference (numerator and denominator alike), keeps
    everything else in float32 and rounds the result to bf16:
      probabilities: each off by BF16_HALF of itself and by twice the error of
        its score; the sums' quotient moves by at most that times sum p |v - o|;
      scores: D + 8 float32 roundings of sum |q k| scale, and of the score;
      sums of T terms in float32, in some order: (T + 8) roundings of sum p |v|;
      the result: BF16_HALF of itself.
    Second-order terms and exp2 (an ulp or two) are covered by a factor 1.25.
    """
    q = numerics.decode_bf16(q_bits)
    total_q, Hq, D = q.shape
    Hkv = k_pool.shape[1]
    G = Hq // Hkv
    out = np.full((total_q, Hq, D), np.nan)
    bound = np.zeros_like(out)
    for s in range(len(q_start) - 1):
        r0, r1 = int(q_start[s]), int(q_start[s + 1])
        n, T = r1 - r0, int(context_lens[s])
        if n == 0:
            continue
        if n > T or n > 64 * mask.shape[1]:
            raise ValueError(f"sequence {s}: {n} drafts of {T} tokens")
        see = np.ones((n, T), bool)
        see[:, T - n:] = bits(mask[r0:r1], n)
        bt = np.asarray(block_tables[s])
        for g in range(Hkv):
            K = numerics.decode(_gather_rows(k_pool, bt, g, T, block_size, False), kv_format)
            V = numerics.decode(_gather_rows(v_pool, bt, g, T, block_size, True), kv_format)
            if k_scale is not None:
                K, V = K * float(k_scale[g]), V * float(v_scale[g])
            for h in range(g * G, (g + 1) * G):
                for i in range(n):
                    t = np.flatnonzero(see[i])
                    if len(t) == 0:
                        out[r0 + i, h] = 0.0
                        continue
                    with np.errstate(invalid="ignore", over="ignore"):
                        z = scale * (K[t] @ q[r0 + i, h])
                        p = np.exp(z - z.max())
                        p /= p.sum()
                        o = p @ V[t]
                        dz = F32_HALF * ((D + 8) * scale * (np.abs(K[t]) @ np.abs(q[r0 + i, h])) + 4 * np.abs(z))
                        dz = dz.max()
                        spread = p @ np.abs(V[t] - o)
                        out[r0 + i, h] = o
                        bound[r0 + i, h] = 1.25 * ((BF16_HALF + 2 * dz) * spread + BF16_HALF * np.abs(o)
                                                   + F32_HALF * (len(t) + 8) * (p @ np.abs(V[t])))
    return out, bound + 1e-30


def accept(k_pool, v_pool, block_tables, context_lens, q_start, accepted, n_accepted, block_size=16):
    """(k, v, context_lens) after the accepted drafts have moved to the front; codes are moved as they are."""
    k, v = np.array(k_pool, copy=True), np.array(v_pool, copy=True)
    num_blocks = k.shape[0]
    ctx = []
    for s in range(len(q_start) - 1):
        n, T = int(q_start[s + 1] - q_start[s]), int(context_lens[s])
        a, last = 0, -1
        if int(n_accepted[s]) < 0:
            ctx.append(T)
            continue
        for j in range(min(int(n_accepted[s]), accepted.shape[1], n)):
            i = int(accepted[s][j])
            if i <= last or i >= n:
                break
            a, last = j + 1, i
        ctx.append(T - n + a)
        for j in range(a):
            ts, td = T - n + int(accepted[s][j]), T - n + j
            bs, bd = int(block_tables[s][ts // block_size]), int(block_tables[s][td // block_size])
            if not (0 <= bs < num_blocks and 0 <= bd < num_blocks):
                continue
            k[bd, :, td % block_size] = k_pool[bs, :, ts % block_size]
            v[bd, :, :, td % block_size] = v_pool[bs, :, :, ts % block_size]
    return k, v, np.array(ctx, np.int32)
