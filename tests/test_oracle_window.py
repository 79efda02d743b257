"""The oracle of windows and block scales against the oracles of whole contexts, scalar loops and searches."""
import numpy as np
import pytest

from oracle import append, attention, numerics, prefill
from oracle import window as ow
from window_cases import FMTS, Case


def whole(c):
    """The case's cache as float64-exact e4m3 or bf16 pools of the old formats (block scales folded into none)."""
    return dict(kv_format="fp8_e4m3" if c.fmt == "fp8_e4m3" else "bf16", k_scale=c.ks, v_scale=c.vs)


@pytest.mark.parametrize("fmt", ["bf16", "fp8_e4m3"])
def test_wide_window_is_the_whole_context(fmt):
    rng = np.random.default_rng(1)
    c = Case(rng, [0, 1, 17, 50], None, 4, 2, fmt, 50, 0)
    ref = attention.paged_decode_attention(c.q, c.k, c.v, c.tables, c.ctx, c.scale, **whole(c))
    assert np.allclose(c.oracle()[0], ref, rtol=0, atol=1e-12)
    c = Case(rng, [5, 33, 40], [5, 20, 1], 4, 2, fmt, 40, 3)
    ref = prefill.chunked_prefill_attention(c.q, c.k, c.v, c.tables, c.ctx, c.q_start, c.scale, **whole(c))
    assert np.allclose(c.oracle()[0], ref, rtol=0, atol=1e-12)


@pytest.mark.parametrize("window,n_sink", [(1, 0), (1, 1), (7, 0), (7, 3), (16, 16), (20, 40), (100, 2)])
def test_masks_by_loops(window, n_sink):
    for T, n in ((1, 1), (5, 2), (40, 40), (64, 3)):
        see = ow.sees(T, n, window, n_sink)
        for i in range(n):
            p = T - n + i
            for t in range(T):
                assert see[i, t] == (t <= p and (p - t < window or t < n_sink))


def test_block_scales_by_scalar_values():
    rng = np.random.default_rng(2)
    c = Case(rng, [37], None, 1, 1, "e4m3_block", 9, 2)
    t = [0, 1] + list(range(28, 37))
    K = np.array([[numerics.e4m3_value(int(x)) * 2.0 ** (int(c.ks[c.tables[0, i // 16], 0]) - 127)
                   for x in c.k[c.tables[0, i // 16], 0, i % 16]] for i in t])
    V = np.array([[numerics.e4m3_value(int(x)) * 2.0 ** (int(c.vs[c.tables[0, i // 16], 0]) - 127)
                   for x in c.v[c.tables[0, i // 16], 0, :, i % 16]] for i in t])
    z = c.scale * K @ numerics.decode_bf16(c.q[0, 0])
    p = np.exp(z - z.max())
    assert np.allclose(c.oracle()[0][0, 0], p @ V / p.sum(), rtol=0, atol=1e-12)


def test_scores_of_minus_infinity_leave_zeros():
    rng = np.random.default_rng(3)
    c = Case(rng, [3], None, 1, 1, "bf16", 3, 0)
    c.q[0, 0] = 0x3F80                                    # ones
    blk = c.tables[0, 0]
    c.k[blk, 0, :3] = 0xBF80                              # a finite row of -1, then -infinity in one dimension
    c.k[blk, 0, :3, 0] = 0xFF80
    assert (c.oracle()[0] == 0).all()


@pytest.mark.parametrize("a", [0.0, 1e-45, 1e-38, 448 * 2.0 ** -126, 448 * 2.0 ** -126 * (1 + 2 ** -20), 1.75, 1.7500001,
                               3.5, 448.0, 449.0, 3e38, 3.38e38])
def test_need_byte_is_the_smallest(a):
    b = ow.need_byte(a)
    assert 1 <= b <= 246
    assert b == 246 or a <= 448 * 2.0 ** (b - 127)
    assert b == 1 or a > 448 * 2.0 ** (b - 128)


def test_append_scaled_by_hand():
    k = np.zeros((2, 1, 16, 128), np.uint8)
    v = np.zeros((2, 1, 128, 16), np.uint8)
    ks, vs = np.full((2, 1), 200, np.uint8), np.full((2, 1), 200, np.uint8)
    new = np.zeros((3, 1, 128))
    new[0, 0, 0], new[1, 0, 1], new[2, 0, 2] = 3.5, -448.0, np.inf
    # a new block: the stale scale does not count; rows 0 and 1 end block 1
    k1, v1, ks1, vs1 = ow.append_scaled(new[:1], new[:1], k, v, ks, vs, [16])
    assert ks1[1, 0] == 120 and k1[1, 0, 0, 0] == 0x7E and v1[1, 0, 0, 0] == 0x7E and ks1[0, 0] == 200
    # a louder token raises it, the older one keeps its value
    k2, v2, ks2, vs2 = ow.append_scaled(new[1:2], new[1:2], k1, v1, ks1, vs1, [17])
    assert ks2[1, 0] == 127
    assert numerics.e4m3_value(int(k2[1, 0, 0, 0])) == 3.5 and numerics.e4m3_value(int(v2[1, 0, 1, 1])) == -448.0
    # what is not finite is NaN and does not raise the scale
    k3, _, ks3, _ = ow.append_scaled(new[2:], new[2:], k2, v2, ks2, vs2, [18])
    assert ks3[1, 0] == 127 and k3[1, 0, 2, 2] == 0x7F and k3[1, 0, 2, 0] == 0


def test_encode_block_is_the_append_code_where_scales_agree():
    x = np.random.default_rng(4).standard_normal(500) * 100
    assert np.array_equal(ow.encode_block(x, 127), append.e4m3_encode(x))


@pytest.mark.parametrize("fmt", FMTS)
def test_hidden_tokens_never_count(fmt):
    rng = np.random.default_rng(5)
    for window, sinks in ((3, 0), (16, 1), (20, 18)):
        out, bound = Case(rng, [70, 16, 1, 33], [40, 2, 1, 33], 2, 1, fmt, window, sinks).oracle()
        assert np.isfinite(out).all() and np.isfinite(bound).all()
