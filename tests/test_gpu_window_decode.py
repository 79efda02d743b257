"""window_decode_attention (through the C ABI) against the oracle in float64, within the oracle's bound.

Every token that the query does not see, every unused block and its scale is
NaN, and table entries of blocks without a visible token are -1.
"""
import numpy as np
import pytest
import torch

import window_cases as wc
from window_cases import FMTS, Case

pytestmark = pytest.mark.gpu


def note(msg):
    print(f"[gpu-test] {msg}", flush=True)


LENGTHS = {"short": [1, 0, 2, 15, 16, 17, 31, 33, 64, 65, 100], "mixed": [700, 0, 1, 129, 2048, 1500, 16, 333],
           "one": [1000]}
EDGES = [(1, 0), (1, 1), (2, 5), (16, 0), (17, 16), (31, 33), (64, 4), (65, 64), (100, 1), (256, 130), (5000, 0),
         (5000, 7)]


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("window,n_sink", EDGES)
@pytest.mark.parametrize("lens", list(LENGTHS))
def test_windows(gpu_lib, fmt, window, n_sink, lens):
    note(f"window decode {fmt} window={window} sinks={n_sink} lens={lens}")
    rng = np.random.default_rng(window * 100 + n_sink)
    c = Case(rng, LENGTHS[lens], None, 8, 2, fmt, window, n_sink)
    ref, bound = c.oracle()
    wc.check(wc.decode(gpu_lib, c), ref, bound)
    # equal slices of the stream, cut segments merged on every level
    unit = 32 if fmt == "bf16" else 64
    wc.check(wc.decode(gpu_lib, c, partition_tokens=unit, workgroups_per_cu=2, out_fp32=True), ref, bound)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("hq,hkv", [(1, 1), (3, 3), (16, 1), (10, 2), (64, 8), (64, 4)])
def test_heads(gpu_lib, fmt, hq, hkv):
    note(f"window decode {fmt} heads {hq}/{hkv}")
    rng = np.random.default_rng(hq)
    c = Case(rng, [300, 40, 1, 777], None, hq, hkv, fmt, 111, 20)
    ref, bound = c.oracle()
    wc.check(wc.decode(gpu_lib, c), ref, bound)
    wc.check(wc.decode(gpu_lib, c, max_ctx=777, partition_tokens=64), ref, bound)


@pytest.mark.parametrize("fmt", FMTS)
def test_a_large_batch(gpu_lib, fmt):
    """Over 64 sequences the prologue goes through LDS; segments are cut at workgroup edges."""
    rng = np.random.default_rng(7)
    ctx = np.concatenate([rng.integers(0, 400, 300), [0, 0, 1]])
    note(f"window decode {fmt} batch {len(ctx)}")
    c = Case(rng, ctx, None, 4, 1, fmt, 90, 3)
    ref, bound = c.oracle()
    wc.check(wc.decode(gpu_lib, c), ref, bound)


@pytest.mark.parametrize("fmt", ["bf16", "fp8_e4m3"])
def test_whole_contexts_agree_with_paged_decode(gpu_lib, fmt):
    """A window that hides nothing: the same arithmetic as the call without one, bit for bit."""
    note(f"window decode {fmt} against paged_decode_attention")
    rng = np.random.default_rng(8)
    c = Case(rng, [1, 500, 64, 2000, 0, 31], None, 16, 2, fmt, 2000, 0)
    d = c.device()
    for kw in (dict(), dict(partition_tokens=64)):
        full = gpu_lib.PagedDecoder(6, 16, 2, c.max_blocks, 2000, c.nb, kv_fp8=fmt != "bf16", **kw)
        a, b = full.new_out(), wc.decode(gpu_lib, c, d=d, **kw)
        full(d["q"], d["k"], d["v"], d["tables"], d["ctx"], c.scale, a, d["ks"], d["vs"])
        assert torch.equal(a, b)


def test_long_context_few_tokens_seen(gpu_lib):
    """A quarter of a million tokens, most of them gone from the cache."""
    note("window decode long context")
    rng = np.random.default_rng(9)
    T = 262_144 - 5
    for fmt in FMTS:
        c = Case(rng, [T, 3], None, 4, 1, fmt, 300, 40)
        ref, bound = c.oracle()
        wc.check(wc.decode(gpu_lib, c), ref, bound)


@pytest.mark.parametrize("fmt", FMTS)
def test_repeats_other_shapes_and_streams(gpu_lib, fmt):
    """One workspace for calls of several windows, also between calls without one; every repeat is the same."""
    note(f"window decode {fmt} shared workspace")
    rng = np.random.default_rng(10)
    cases = [Case(rng, rng.integers(1, 900, 20), None, 8, 2, fmt, w, s) for w, s in ((50, 0), (700, 33), (333, 4))]
    decs = [wc.decoder(gpu_lib, c, partition_tokens=64) for c in cases]
    big = max((d.workspace for d in decs), key=lambda t: t.numel())
    for d in decs:
        d.workspace = big
    devs = [c.device() for c in cases]
    first = [wc.decode(gpu_lib, c, dec=d, d=x).clone() for c, d, x in zip(cases, decs, devs)]
    for c, out in zip(cases, first):
        wc.check(out, *c.oracle())
    side = torch.cuda.Stream()
    for _ in range(5):
        for c, d, x, f in zip(cases, decs, devs, first):
            assert torch.equal(wc.decode(gpu_lib, c, dec=d, d=x), f)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        again = [wc.decode(gpu_lib, c, dec=d, d=x) for c, d, x in zip(cases, decs, devs)]
    side.synchronize()
    for a, f in zip(again, first):
        assert torch.equal(a, f)


@pytest.mark.parametrize("fmt", FMTS)
def test_captured_and_replayed(gpu_lib, fmt):
    note(f"window decode {fmt} graph")
    rng = np.random.default_rng(11)
    c = Case(rng, [600, 31, 90, 1200], None, 8, 2, fmt, 128, 4)
    d, dec = c.device(), wc.decoder(gpu_lib, c, partition_tokens=64)
    want = wc.decode(gpu_lib, c, dec=dec, d=d).clone()
    out = torch.zeros_like(want)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        wc.decode(gpu_lib, c, dec=dec, d=d, out=out)
    for _ in range(4):
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        assert torch.equal(wc.decode(gpu_lib, c, dec=dec, d=d), want)


@pytest.mark.parametrize("fmt", ["bf16", "fp8_e4m3"])
def test_infinite_keys(gpu_lib, fmt):
    """Scores of -infinity: zeros where there are no others, no weight where there are."""
    note(f"window decode {fmt} infinite scores")
    rng = np.random.default_rng(12)
    c = Case(rng, [100, 100, 3], None, 4, 1, fmt, 70, 2)
    if fmt == "bf16":
        c.k[:, 0, :, 0] = 0xFF80                  # -infinity in the first dimension
        c.k[c.tables[1, 6], 0, 1, 0] = 0x3F80     # but for one token of the second sequence
    else:
        c.ks[:] = 0.0                             # all scores 0: the mean of the values that are seen
    c.q[:, :, 0] = 0x3F80
    ref, bound = c.oracle()
    if fmt == "bf16":
        assert (ref[[0, 2]] == 0).all() and (ref[1] != 0).any()
    wc.check(wc.decode(gpu_lib, c), ref, bound + 1e-30)
    wc.check(wc.decode(gpu_lib, c, partition_tokens=64, workgroups_per_cu=1), ref, bound + 1e-30)


def test_negative_and_nan_scales(gpu_lib):
    note("window decode: key scales below zero, NaN scales")
    rng = np.random.default_rng(13)
    c = Case(rng, [90, 200], None, 4, 2, "fp8_e4m3", 33, 1)
    c.ks[1] = -c.ks[1]
    wc.check(wc.decode(gpu_lib, c), *c.oracle())
    c.ks[0] = np.nan
    got = wc.decode(gpu_lib, c).float().cpu().numpy()
    assert np.isnan(got[:, :2]).all() and np.isfinite(got[:, 2:]).all()
    c = Case(rng, [90, 200], None, 4, 2, "e4m3_block", 33, 1)
    c.vs[c.tables[1, 11], 1] = 255                # a block that sequence 1 sees, head 1
    got = wc.decode(gpu_lib, c).float().cpu().numpy()
    assert np.isnan(got[1, 2:]).all() and np.isfinite(got[0]).all() and np.isfinite(got[1, :2]).all()


@pytest.mark.parametrize("byte", [1, 40, 127, 200, 235])
def test_scale_bytes_over_the_range(gpu_lib, byte):
    """Values of any size.  Products with a probability that fall below 2^-126 may be flushed, 63 of them at most."""
    note(f"window decode scale byte {byte}")
    rng = np.random.default_rng(byte)
    c = Case(rng, [75], None, 2, 1, "e4m3_block", 60, 3)
    live = np.unique(c.tables[c.tables >= 0])
    c.vs[live] = byte
    if byte == 1:   # below 2^-126 bf16 keeps fewer bits: codes whose values stay normal
        v = c.v[live] & 0x7F
        c.v[live] = np.where(v < 0x7F, np.maximum(v, 0x38), c.v[live])
    ref, bound = c.oracle()
    got = wc.decode(gpu_lib, c, out_fp32=True).double().cpu().numpy()
    assert np.isfinite(got).all()
    assert (np.abs(got - ref) <= bound + 63 * 2.0 ** -126).all()


# one workgroup a segment: one to three units a wave, up to one segment a compute unit, at the
# lines of the rule (18 units at any batch, 24 from 128 segments on 256 compute units, with block
# scales from 160) and past them
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("batch,hkv", [(1, 1), (12, 8), (16, 8), (20, 8), (32, 8), (33, 8), (96, 1)])
@pytest.mark.parametrize("units", [1, 8, 9, 16, 17, 18, 19, 22])
def test_units_a_wave(gpu_lib, fmt, batch, hkv, units):
    note(f"window decode {fmt} batch={batch} heads={hkv} units={units}")
    unit = 32 if fmt == "bf16" else 64
    rng = np.random.default_rng(units)
    window, n_sink = max(units - 1, 1) * unit - 7, 5
    ctx = rng.integers(1, 2 * window + 300, batch)
    ctx[0], ctx[-1] = 2 * window + 300, window
    c = Case(rng, ctx, None, hkv, hkv, fmt, window, n_sink)
    pick = rng.integers(0, hkv)
    out = wc.decode(gpu_lib, c)
    one = Case.__new__(Case)
    one.__dict__.update(c.__dict__)
    one.q, one.k, one.v = c.q[:, pick:pick + 1], c.k[:, pick:pick + 1], c.v[:, pick:pick + 1]
    if fmt != "bf16":
        one.ks, one.vs = (x[:, pick:pick + 1] if fmt == "e4m3_block" else x[pick:pick + 1] for x in (c.ks, c.vs))
    wc.check(out[:, pick:pick + 1], *one.oracle())


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("batch", [3, 300])
def test_nothing_cached(gpu_lib, fmt, batch):
    note(f"window decode {fmt} empty sequences batch={batch}")
    c = Case(np.random.default_rng(14), [0] * batch, None, 4, 1, fmt, 10, 2)
    assert (wc.decode(gpu_lib, c) == 0).all() and (wc.decode(gpu_lib, c, max_ctx=16) == 0).all()


def test_tensors_that_are_elsewhere(gpu_lib):
    """A queries' tensor or a cache in host memory is refused before anything is enqueued."""
    note("window decode, host tensors")
    c = Case(np.random.default_rng(12), [40], None, 4, 2, "bf16", 16, 0)
    d = c.device()
    for name in ("q", "k"):
        with pytest.raises(ValueError):
            wc.decode(gpu_lib, c, d=dict(d, **{name: d[name].cpu()}))
    p = Case(np.random.default_rng(12), [40], [3], 4, 2, "bf16", 16, 0)
    d = p.device()
    with pytest.raises(ValueError):
        wc.prefill(gpu_lib, p, d=dict(d, k=d["k"].cpu()))


@pytest.mark.parametrize("batch,hkv", [(6, 2), (64, 1), (70, 2), (300, 1)])
@pytest.mark.parametrize("lg", [3, 2, 1, 0])
@pytest.mark.parametrize("fmt", FMTS)
def test_segments_apart(gpu_lib, fmt, lg, batch, hkv):
    """Segments of seven or eight units over twice as many workgroups, as many, half or a quarter as many: each takes
    eight, four, two or one slice of its own (300 over the 256 of a device two at most).  Then one segment too short for its slices among them, and empty ones."""
    note(f"window decode {fmt} segments apart lg={lg} batch={batch}")
    rng = np.random.default_rng(13)
    unit = 32 if fmt == "bf16" else 64
    kw = dict(max_ctx=9 * unit, partition_tokens=unit * (8 >> lg))
    lens = [rng.integers(7 * unit, 9 * unit + 1, batch)]
    lens.append(np.where(rng.random(batch) < 0.2, 0, lens[0]))
    lens.append(lens[1].copy())
    lens[2][batch // 2] = unit // 2
    lens.append(np.where(np.arange(batch) == batch - 1, lens[0], 0))
    for ctx in lens:
        c = Case(rng, ctx, None, 4 * hkv, hkv, fmt, 7 * unit, 0, max_blocks=9 * unit // 16)
        d = c.device()
        out = wc.decode(gpu_lib, c, d=d, **kw)
        wc.check(out, *c.oracle())
        assert torch.equal(out, wc.decode(gpu_lib, c, d=d, **kw))
