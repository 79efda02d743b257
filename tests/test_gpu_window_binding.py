"""The Python binding of the window and block-scale operators: one tensor in host memory at a time is refused, and
tensors of other types that hold the same bits give the same results."""
import numpy as np
import pytest
import torch

import window_cases as wc
from window_cases import FMTS, Case

pytestmark = pytest.mark.gpu


def note(msg):
    print(f"[gpu-test] {msg}", flush=True)


@pytest.mark.parametrize("fmt", FMTS)
def test_attention_arguments_in_host_memory(gpu_lib, fmt):
    note(f"window attention {fmt}, host tensors")
    rng = np.random.default_rng(1)
    for rows, call in ((None, wc.decode), ([1, 5], wc.prefill)):
        c = Case(rng, [40, 9], rows, 4, 2, fmt, 16, 1)
        d = {k: v for k, v in c.device().items() if v is not None}
        for name in d:
            with pytest.raises(ValueError, match="current device"):
                call(gpu_lib, c, d=dict(c.device(), **{name: d[name].cpu()}))
        with pytest.raises(ValueError, match="current device"):
            call(gpu_lib, c, d=c.device(), out=torch.zeros((c.total, 4, 128), dtype=torch.bfloat16))
    c = Case(rng, [40, 9], None, 4, 2, fmt, 16, 1)
    dec = wc.decoder(gpu_lib, c)
    dec.workspace = dec.workspace.cpu()
    with pytest.raises(ValueError, match="current device"):
        wc.decode(gpu_lib, c, dec=dec)


@pytest.mark.parametrize("fmt", FMTS)
def test_attention_types_that_hold_the_same_bits(gpu_lib, fmt):
    note(f"window attention {fmt}, other types")
    rng = np.random.default_rng(2)
    for rows, call in ((None, wc.decode), ([1, 5], wc.prefill)):
        c = Case(rng, [40, 9], rows, 4, 2, fmt, 16, 1)
        d = c.device()
        want = call(gpu_lib, c, d=d)
        kv = torch.bfloat16 if fmt == "bf16" else torch.float8_e4m3fn
        e = dict(d, q=d["q"].view(torch.bfloat16), k=d["k"].view(kv), v=d["v"].view(kv))
        if fmt == "e4m3_block":
            e.update({n: d[n].view(torch.float8_e8m0fnu) for n in ("ks", "vs")})
        assert torch.equal(call(gpu_lib, c, d=e), want)
        out = torch.zeros((c.total, 4, 128), dtype=torch.int16, device="cuda")
        assert torch.equal(call(gpu_lib, c, d=d, out=out).view(torch.bfloat16), want)
