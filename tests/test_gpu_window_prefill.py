"""window_prefill_attention (through the C ABI) against the oracle in float64, within the oracle's bound.

Every token that no row sees, every unused block and its scale is NaN, and
table entries of blocks without a visible token are -1.
"""
import numpy as np
import pytest
import torch

import window_cases as wc
from oracle import window as ow
from window_cases import FMTS, Case

pytestmark = pytest.mark.gpu


def note(msg):
    print(f"[gpu-test] {msg}", flush=True)


EDGES = [(1, 0), (1, 3), (15, 1), (32, 0), (33, 33), (64, 4), (100, 65), (3000, 0), (3000, 9)]
BATCHES = {"ragged": ([1, 16, 33, 200, 64, 300], [1, 16, 2, 150, 64, 7]),
           "chunks": ([700, 513, 90], [128, 257, 90]),
           "single": ([500, 17, 1], [1, 1, 1]),
           "gaps": ([400, 5, 40], [65, 0, 0])}


def crowded(ctx, rows):
    """The same sequences among enough others without rows that a batch is not one of few rows (64 sequences)."""
    return list(ctx) + [3] * 64, list(rows) + [0] * 64


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("window,n_sink", EDGES)
@pytest.mark.parametrize("batch", list(BATCHES))
def test_windows(gpu_lib, fmt, window, n_sink, batch):
    note(f"window prefill {fmt} window={window} sinks={n_sink} batch={batch}")
    rng = np.random.default_rng(window * 100 + n_sink)
    c = Case(rng, *BATCHES[batch], 8, 2, fmt, window, n_sink)
    ref, bound = c.oracle()
    wc.check(wc.prefill(gpu_lib, c), ref, bound)
    wc.check(wc.prefill(gpu_lib, c, max_ctx=4800 if c.max_blocks >= 300 else 16 * c.max_blocks, out_fp32=True), ref,
             bound)
    c = Case(rng, *crowded(*BATCHES[batch]), 8, 2, fmt, window, n_sink, max_blocks=300)
    ref, bound = c.oracle()
    wc.check(wc.prefill(gpu_lib, c), ref, bound)
    # contexts that may be long take other variants (pairs of waves) where the window is wide
    wc.check(wc.prefill(gpu_lib, c, max_ctx=4800, out_fp32=True), ref, bound)


# batches on each side of the launch rule's lines: 256 columns to eight waves, 128
# to four, 64 and 128 to pairs, 64 to four (a batch of more than 64), few rows
VARIANTS = {
    "256": ([1000] * 4, [512] * 4, 64, 32, 63, 800, 5), "128": ([600] * 3, [350] * 3, 64, 32, 40, 290, 0),
    "128 short": ([600] * 3, [350] * 3, 64, 32, 40, 70, 5), "pairs 64": ([2600, 90], [100, 90], 16, 2, 200, 2100, 3),
    "pairs 128": ([2600, 2300], [150, 150], 64, 2, 200, 2100, 0), "64": ([200] * 70, [3] * 70, 8, 4, 20, 70, 5),
    "few": ([600, 90], [100, 90], 16, 2, 40, 290, 5), "few, many heads": ([300, 90], [9, 7], 64, 1, 40, 64, 1)}


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("variant", list(VARIANTS))
def test_variants(gpu_lib, fmt, variant):
    ctx, rows, hq, hkv, max_blocks, window, n_sink = VARIANTS[variant]
    note(f"window prefill {fmt} variant {variant}")
    rng = np.random.default_rng(hq + window)
    c = Case(rng, ctx, rows, hq, hkv, fmt, window, n_sink, max_blocks=max_blocks)
    out = wc.prefill(gpu_lib, c, max_ctx=max_blocks * 16)
    if hkv == 32:  # a head of each launch is enough for the oracle
        out = out.view(c.total, hkv, hq // hkv, 128)[:, 5].contiguous()
        one = Case.__new__(Case)
        one.__dict__.update(c.__dict__)
        one.q, one.k, one.v = c.q.reshape(c.total, hkv, -1, 128)[:, 5], c.k[:, 5:6], c.v[:, 5:6]
        if fmt != "bf16":
            one.ks, one.vs = (x[:, 5:6] if fmt == "e4m3_block" else x[5:6] for x in (c.ks, c.vs))
        c = one
    wc.check(out, *c.oracle())


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("hq,hkv", [(1, 1), (5, 5), (12, 1), (14, 2), (40, 1)])
def test_heads(gpu_lib, fmt, hq, hkv):
    note(f"window prefill {fmt} heads {hq}/{hkv}")
    rng = np.random.default_rng(hq)
    c = Case(rng, [290, 40, 500], [290, 3, 66], hq, hkv, fmt, 120, 20)
    wc.check(wc.prefill(gpu_lib, c), *c.oracle())
    c = Case(rng, *crowded([290, 40, 500], [290, 3, 66]), hq, hkv, fmt, 120, 20)
    wc.check(wc.prefill(gpu_lib, c), *c.oracle())


@pytest.mark.parametrize("fmt", FMTS)
def test_decode_is_the_case_of_one_row(gpu_lib, fmt):
    note(f"window prefill {fmt} against decode")
    rng = np.random.default_rng(5)
    c = Case(rng, [290, 40, 1, 1000], [1, 1, 1, 1], 8, 2, fmt, 120, 20)
    ref, bound = c.oracle()
    wc.check(wc.prefill(gpu_lib, c), ref, bound)
    wc.check(wc.decode(gpu_lib, c), ref, bound)


@pytest.mark.parametrize("fmt", ["bf16", "fp8_e4m3"])
@pytest.mark.parametrize("max_blocks", [40, 300])
def test_whole_contexts_agree_with_chunked_prefill(gpu_lib, fmt, max_blocks):
    """A window that hides nothing, in a batch that is not one of few rows: the same arithmetic as the call without
    one, bit for bit."""
    note(f"window prefill {fmt} against chunked_prefill_attention")
    rng = np.random.default_rng(6)
    c = Case(rng, [600, 33, 1], [200, 33, 1], 32, 8, fmt, 10000, 0, max_blocks=max_blocks)
    d = c.device()
    a = wc.prefill(gpu_lib, c, d=d, max_ctx=16 * max_blocks)
    b = torch.empty_like(a)
    gpu_lib.chunked_prefill_attention(d["q"], d["k"], d["v"], d["tables"], d["ctx"], d["q_start"], c.scale, b,
                                      wc.prefill_shape(gpu_lib, c, max_ctx=16 * max_blocks), d["ks"], d["vs"])
    assert torch.equal(a, b)


@pytest.mark.parametrize("fmt", FMTS)
def test_context_past_the_staged_ids(gpu_lib, fmt):
    """A context of more than 65,536 tokens, of which the window leaves few."""
    note(f"window prefill {fmt} long context")
    rng = np.random.default_rng(7)
    for ctx, rows in (([200_003, 90], [70, 5]), crowded([200_003, 90], [70, 5])):
        c = Case(rng, ctx, rows, 2, 1, fmt, 333, 40)
        wc.check(wc.prefill(gpu_lib, c), *c.oracle())


def test_widest_window_past_the_staged_ids(gpu_lib):
    """The largest window + n_sink that contexts past 65,536 tokens may have, in items of 256 tokens."""
    note("window prefill widest window")
    rng = np.random.default_rng(8)
    c = Case(rng, [66_500], [256], 1, 1, "fp8_e4m3", 65_000, 24)
    out = wc.prefill(gpu_lib, c)
    rows = [0, 1, 100, 255]
    see = ow.sees(66_500, 256, 65_000, 24)[rows]
    from oracle import numerics
    K, V = (numerics.decode_e4m3(x[c.tables[0, :-(-66_500 // 16)], 0]) for x in (c.k, c.v))
    K = K.reshape(-1, 128)[:66_500] * float(c.ks[0])
    V = V.transpose(0, 2, 1).reshape(-1, 128)[:66_500] * float(c.vs[0])
    q = numerics.decode_bf16(c.q[rows, 0])
    for i, r in enumerate(rows):
        t = np.flatnonzero(see[i])
        z = c.scale * (K[t] @ q[i])
        p = np.exp(z - z.max())
        p /= p.sum()
        o = p @ V[t]
        lim = 1.25 * ((2.0 ** -8 + 2.0 ** -24 * 136 * np.abs(z).max() * 20) * (p @ np.abs(V[t] - o)) + 2.0 ** -8 * np.abs(o)
                      + 2.0 ** -24 * (len(t) + 8) * (p @ np.abs(V[t])))
        assert (np.abs(out[r, 0].double().cpu().numpy() - o) <= lim).all()


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("hq,hkv", [(8, 1), (1, 1)])
@pytest.mark.parametrize("many", [False, True])
def test_a_value_that_is_not_finite_stays_near(gpu_lib, fmt, hq, hkv, many):
    """NaN in the rows that see its token, in none farther than 62 positions from those."""
    note(f"window prefill {fmt} NaN value heads {hq}/{hkv}")
    rng = np.random.default_rng(9)
    T, n, window, sinks = 900, 600, 100, 8
    c = Case(rng, *(crowded([T], [n]) if many else ([T], [n])), hq, hkv, fmt, window, sinks)
    see = ow.sees(T, n, window, sinks)
    for t in (3, 250, 555, 899):
        d = c.device()
        d["v"][int(c.tables[0, t // 16]), :, 5, t % 16] = int(np.int16(wc.NAN_CODE[fmt])) if fmt == "bf16" else 0x7F
        got = wc.prefill(gpu_lib, c, d=d).float().isnan().any(-1).any(-1).cpu().numpy()
        sees = np.flatnonzero(see[:, t])
        assert got[sees].all()
        far = np.ones(n, bool)
        far[max(sees.min() - 62, 0):sees.max() + 63] = False
        assert not got[far].any()


@pytest.mark.parametrize("fmt", ["bf16", "fp8_e4m3"])
@pytest.mark.parametrize("max_blocks,many", [(20, False), (20, True), (300, True)])
@pytest.mark.parametrize("window", [70, 3000])
def test_scores_of_minus_infinity_and_odd_scales(gpu_lib, fmt, max_blocks, many, window):
    note(f"window prefill {fmt} infinite scores, odd scales")
    rng = np.random.default_rng(10)
    c = Case(rng, *(crowded([100, 300], [20, 30]) if many else ([100, 300], [20, 30])), 4, 2, fmt, window, 2,
             max_blocks=max_blocks)
    c.q[:, :, 0] = 0x3F80
    if fmt == "bf16":
        c.k[c.tables[0, :7], 0, :, 0] = 0xFF80
    else:
        c.ks[:] = [0.0, -0.01]
    ref, bound = c.oracle()
    if fmt == "bf16":
        assert (ref[:20, :2] == 0).all()
    wc.check(wc.prefill(gpu_lib, c, max_ctx=16 * max_blocks), ref, bound)
    if fmt != "bf16":
        c.ks[0] = np.nan
        got = wc.prefill(gpu_lib, c, max_ctx=16 * max_blocks).float().cpu().numpy()
        assert np.isnan(got[:, :2]).all() and np.isfinite(got[:, 2:]).all()


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("many", [False, True])
def test_rows_behind_the_batch_stay(gpu_lib, fmt, many):
    note(f"window prefill {fmt} padded batch")
    rng = np.random.default_rng(11)
    c = Case(rng, *(crowded([60, 30], [20, 30]) if many else ([60, 30], [20, 30])), 4, 2, fmt, 25, 2)
    ref, bound = c.oracle()
    d = c.device()
    pad = torch.zeros((13, 4, 128), dtype=d["q"].dtype, device="cuda")
    d["q"] = torch.cat([d["q"], pad])
    out = torch.full((c.total + 13, 4, 128), 5.0, dtype=torch.bfloat16, device="cuda")
    c.total += 13
    wc.prefill(gpu_lib, c, d=d, out=out)
    wc.check(out[:-13], ref, bound)
    assert (out[-13:] == 5.0).all()


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("many", [False, True])
def test_captured_replayed_and_on_two_streams(gpu_lib, fmt, many):
    note(f"window prefill {fmt} graph and streams")
    rng = np.random.default_rng(12)
    c = Case(rng, *(crowded([500, 31, 90], [130, 20, 90]) if many else ([500, 31, 90], [130, 20, 90])), 8, 2, fmt, 64, 4)
    d = c.device()
    want = wc.prefill(gpu_lib, c, d=d).clone()
    outs = [torch.zeros_like(want) for _ in range(2)]
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        wc.prefill(gpu_lib, c, d=d, out=outs[0])
    for _ in range(4):
        outs[0].zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], want)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for o, st in zip(outs, streams):
        o.zero_()
        st.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(st):
            for _ in range(3):
                wc.prefill(gpu_lib, c, d=d, out=o)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want) and torch.equal(outs[1], want)


@pytest.mark.parametrize("batch", [3968, 4096])
def test_largest_batches(gpu_lib, batch):
    """The most LDS a launch takes, with pairs of waves and past their limit."""
    note(f"window prefill batch {batch}")
    rng = np.random.default_rng(13)
    ctx = rng.integers(1, 40, batch)
    for fmt in ("bf16", "e4m3_block"):
        c = Case(rng, ctx, np.ones(batch, np.int64), 2, 1, fmt, 3000, 1, max_blocks=200)
        ref, bound = c.oracle()
        wc.check(wc.prefill(gpu_lib, c, max_ctx=3200), ref, bound)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("batch", [64, 65])
def test_few_rows_of_many_sequences(gpu_lib, fmt, batch):
    """Row offsets of up to 64 sequences are looked at by the lanes of a wave; some have no rows, some no tokens."""
    note(f"window prefill {fmt} {batch} sequences")
    rng = np.random.default_rng(batch)
    ctx = rng.integers(0, 300, batch)
    rows = np.minimum(rng.integers(0, 4, batch), ctx)
    rows[-1], ctx[-1] = 3, 250
    c = Case(rng, ctx, rows, 5, 1, fmt, 90, 3)
    wc.check(wc.prefill(gpu_lib, c), *c.oracle())


@pytest.mark.parametrize("fmt", ["bf16", "e4m3_block"])
def test_broken_promises_stay_in_bounds(gpu_lib, fmt):
    """Row offsets out of order or past total_q, more rows than tokens, contexts past the largest, ids outside the
    pool: clamped, and rows past the clamped ones are left alone."""
    note(f"window prefill {fmt} broken promises")
    rng = np.random.default_rng(15)
    for many in (False, True):
        ctx, rows = ([40, 200, 64], [10, 20, 5])
        if many:
            ctx, rows = crowded(ctx, rows)
        c = Case(rng, ctx, rows, 4, 2, fmt, 50, 3)
        ref, bound = c.oracle()
        d = c.device()
        d["tables"][1] = 1 << 30                               # (sequence 1's blocks: any of the pool's)
        d["ctx"][2] = 1 << 20                                  # longer than max_context_len: clamped
        got = wc.prefill(gpu_lib, c, d=d).double().cpu().numpy()
        assert (np.abs(got[:10] - ref[:10]) <= bound[:10]).all()
        d = c.device()
        d["ctx"][0] = 4                                        # ten rows of four tokens: six are left alone
        d["q_start"][3:] = 1 << 20                             # ends past total_q
        out = torch.full((c.total, 4, 128), 5.0, dtype=torch.bfloat16, device="cuda")
        wc.prefill(gpu_lib, c, d=d, out=out)
        assert (out[4:10] == 5.0).all() and (out[:4] != 5.0).any()
        d["q_start"][1:] = torch.flip(d["q_start"][1:], (0,))  # out of order
        wc.prefill(gpu_lib, c, d=d, out=out)
        torch.cuda.synchronize()
