"""Per-head RMS norm and rotary position embedding, written out from their definitions in float64.

Test infrastructure only (see the package header).

What is computed.  The models of the paper's case studies (Llama-3-70B, Sec.
4.1; Qwen3-235B-A22B, Sec. 4.7) turn each query and key head by its token's
position before the attention, the second after an RMS norm of the head:

    y = x w / sqrt(mean(x^2) + eps)            (or y = x)
    for each pair (a, b) of the first R dimensions, with the angle's cosine c
    and sine s at the token's position:  a' = a c - b s,  b' = b c + a s

Pair d of R / 2 is dimensions (d, d + R / 2), or (2d, 2d + 1).

Parity: pinned by complex multiplication, by identities (angle 0 changes
nothing, lengths are kept, products depend on the distance only) and by
brute-force loops.
"""
from __future__ import annotations

import numpy as np


def norm(x, w, eps):
    """x [..., D] float64; w [D] or None."""
    if w is None:
        return x
    return x / np.sqrt((x * x).mean(axis=-1, keepdims=True) + eps) * w


def turn(y, cos, sin, interleaved=False):
    """y [rows, heads, D]; cos, sin [rows, R / 2]: the first R dimensions are turned."""
    half = cos.shape[1]
    out = np.array(y, copy=True)
    for d in range(half):
        i, j = (2 * d, 2 * d + 1) if interleaved else (d, d + half)
        c, s = cos[:, None, d], sin[:, None, d]
        out[..., i] = y[..., i] * c - y[..., j] * s
        out[..., j] = y[..., j] * c + y[..., i] * s
    return out


def table(n_positions, rotary_dim, theta=500000.0):
    """[n_positions, rotary_dim] float64: cosines, then sines, of p * theta^(-2 d / rotary_dim)."""
    half = rotary_dim // 2
    a = np.arange(n_positions)[:, None] * theta ** (-np.arange(half) / max(half, 1))
    return np.concatenate([np.cos(a), np.sin(a)], axis=1)
