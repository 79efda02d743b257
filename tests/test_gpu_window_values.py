"""window_prefill_attention: how far a cached value that is not finite may show.

It shows in the rows that see its token, and may show in rows up to 62
positions from those; every other row keeps the bits that it has without it.
Tokens are taken where a wave's last tile holds none that its rows see (pairs
of waves), and where a tile holds the last first token (sink) and tokens that
the window passes.
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


def check(lib, c, T, n, tokens, max_ctx):
    """Sequence 0 of c has T tokens, the last n of them rows; one token at a time is NaN in all its values."""
    see = ow.sees(T, n, c.window, c.n_sink)
    d = c.device()
    want = wc.prefill(lib, c, d=d, max_ctx=max_ctx)[:n].clone()
    assert want.isfinite().all()
    nan = int(np.int16(wc.NAN_CODE[c.fmt])) if c.fmt == "bf16" else 0x7F
    for t in tokens:
        at = d["v"][int(c.tables[0, t // 16])][:, :, t % 16]
        before = at.clone()
        at.fill_(nan)
        got = wc.prefill(lib, c, d=d, max_ctx=max_ctx)[:n]
        at.copy_(before)
        sees = np.flatnonzero(see[:, t])
        assert len(sees)
        bad = got.float().isnan().any(-1).any(-1).cpu().numpy()
        assert bad[sees].all()
        near = np.zeros(n, bool)
        for r in sees:
            near[max(r - 62, 0):r + 63] = True
        assert not bad[~near].any(), f"token {t}: rows {np.flatnonzero(bad & ~near)}"
        far = torch.from_numpy(~near).cuda()
        assert torch.equal(got[far], want[far])


# (query and KV heads) that take pairs of waves with 64 columns, and with 128
PAIRS = {"64": 2, "128": 32}


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("pairs", list(PAIRS))
@pytest.mark.parametrize("window,n_sink", [(1, 2100), (2, 2111), (40, 2100), (2200, 0)])
def test_pairs_of_waves(gpu_lib, fmt, pairs, window, n_sink):
    note(f"window prefill {fmt} NaN value, pairs of waves {pairs}, window={window} sinks={n_sink}")
    rng = np.random.default_rng(window)
    T, n, h = 2304 + 600, 600, PAIRS[pairs]
    c = Case(rng, [T], [n], h, h, fmt, window, n_sink)
    # the first tokens of 64 and of their second halves; a token in mid tile
    check(gpu_lib, c, T, n, [2304, 2336, 2304 + 64 * 3 + 32, 2304 + 64 * 5 + 13, 2304 + 64 * 8 + 32], 16 * c.max_blocks)


# sequences besides the first (3 tokens, no rows), T = n, heads, window: items of 64 and 128
# columns of four waves, 256 of eight, pairs of waves with 64 and 128
VARIANTS = {"64": (64, 600, 1, 100), "128": (0, 600, 64, 100), "256": (0, 1500, 64, 800),
            "pairs 64": (0, 3000, 2, 2100), "pairs 128": (0, 3000, 8, 2100)}


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("variant", list(VARIANTS))
@pytest.mark.parametrize("n_sink", [1, 8, 24, 31, 33, 48])
def test_behind_the_last_sink(gpu_lib, fmt, variant, n_sink):
    note(f"window prefill {fmt} NaN value behind {n_sink} sinks, {variant}")
    more, T, h, window = VARIANTS[variant]
    rng = np.random.default_rng(n_sink)
    c = Case(rng, [T] + [3] * more, [T] + [0] * more, h, h, fmt, window, n_sink)
    check(gpu_lib, c, T, T, sorted({n_sink, n_sink | 15, n_sink | 31, n_sink + 40}), 16 * c.max_blocks)


@pytest.mark.parametrize("variant", list(VARIANTS))
def test_a_scale_of_nan_behind_the_last_sink(gpu_lib, variant):
    """The whole of a block that holds no first token."""
    note(f"window prefill, NaN scale behind the sinks, {variant}")
    more, T, h, window = VARIANTS[variant]
    rng = np.random.default_rng(1)
    c = Case(rng, [T] + [3] * more, [T] + [0] * more, h, h, "e4m3_block", window, 16)
    d = c.device()
    want = wc.prefill(gpu_lib, c, d=d, max_ctx=16 * c.max_blocks)[:T].clone()
    d["vs"][int(c.tables[0, 1])] = 255
    got = wc.prefill(gpu_lib, c, d=d, max_ctx=16 * c.max_blocks)[:T]
    assert got[16:31 + window].isnan().all()             # the rows that see token 31
    assert torch.equal(got[31 + window + 62:], want[31 + window + 62:]) and want.isfinite().all()


@pytest.mark.parametrize("fmt", FMTS)
def test_a_sink_that_is_not_finite(gpu_lib, fmt):
    """Every row from its own position on sees it; tiles whose V a wave takes from a copy give the same."""
    note(f"window prefill {fmt}, a sink that is not finite")
    rng = np.random.default_rng(2)
    T, sink = 600, 5
    c = Case(rng, [T], [T], 64, 64, fmt, 100, 8)
    d = c.device()
    code = {"bf16": 0x7F80}.get(fmt, 0x7F)               # (e4m3 has no infinity)
    d["v"][int(c.tables[0, 0]), :, 7, sink] = code
    got = wc.prefill(gpu_lib, c, d=d, max_ctx=16 * c.max_blocks)
    assert (got[sink:, :, 7] == float("inf")).all() if fmt == "bf16" else got[sink:, :, 7].isnan().all()
    rest = torch.arange(128, device="cuda") != 7
    assert got[:, :, rest].isfinite().all()


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("n_sink", [5, 40])
def test_one_sequence_after_the_other(gpu_lib, fmt, n_sink):
    """Workgroups that take several items, each with its own copy of the last sink's tile."""
    note(f"window prefill {fmt}, many items a workgroup, {n_sink} sinks")
    rng = np.random.default_rng(3)
    lens = [500, 700, 333, 650, 900, 120]
    c = Case(rng, lens, lens, 64, 64, fmt, 60, n_sink)
    out = wc.prefill(gpu_lib, c, max_ctx=16 * c.max_blocks)
    one = Case.__new__(Case)
    one.__dict__.update(c.__dict__)
    one.hq = one.hkv = 1
    one.q, one.k, one.v = c.q[:, 9:10], c.k[:, 9:10], c.v[:, 9:10]
    if fmt != "bf16":
        one.ks, one.vs = (x[:, 9:10] if fmt == "e4m3_block" else x[9:10] for x in (c.ks, c.vs))
    wc.check(out[:, 9:10].contiguous(), *one.oracle())


@pytest.mark.parametrize("batch", [720, 722, 3424, 3425])
def test_the_lists_of_large_batches(gpu_lib, batch):
    """Two workgroups to a unit and one, pairs of waves and none: at the lines of their LDS."""
    note(f"window prefill, {batch} sequences")
    rng = np.random.default_rng(4)
    ctx = rng.integers(1, 40, batch)
    ctx[batch // 2] = 150
    rows = np.ones(batch, np.int64)
    rows[batch // 2] = 150
    for fmt, window in (("bf16", 3000), ("e4m3_block", 20)):
        c = Case(rng, ctx, rows, 2, 1, fmt, window, 3, max_blocks=200)
        wc.check(wc.prefill(gpu_lib, c, max_ctx=3200), *c.oracle())


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("window,n_sink", [(768, 512), (768, 513), (769, 0), (5, 1275), (5, 1276)])
def test_lines_of_short_windows(gpu_lib, fmt, window, n_sink):
    """Items of 128 columns up to 768 tokens of window and 1,280 with the sinks, of 256 beyond."""
    note(f"window prefill {fmt}, window {window} and {n_sink} sinks")
    rng = np.random.default_rng(5)
    c = Case(rng, [1500] * 4, [256] * 4, 64, 64, fmt, window, n_sink)
    out = wc.prefill(gpu_lib, c, max_ctx=16 * c.max_blocks)
    one = Case.__new__(Case)
    one.__dict__.update(c.__dict__)
    one.q, one.k, one.v = c.q[:, 33:34], c.k[:, 33:34], c.v[:, 33:34]
    if fmt != "bf16":
        one.ks, one.vs = (x[:, 33:34] if fmt == "e4m3_block" else x[33:34] for x in (c.ks, c.vs))
    wc.check(out[:, 33:34].contiguous(), *one.oracle())
