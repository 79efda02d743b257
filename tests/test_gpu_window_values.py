"""window_prefill_attention: how far a cached value that is not finite may show.

It shows in the rows that see its token, and may show in rows up to 62
positions from those; every other row keeps the bits that it has without it.
Tokens are taken where a wave's last tile holds none that its rows see (pairs
of waves).
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
