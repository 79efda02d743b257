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


def test_write_arguments_in_host_memory(gpu_lib):
    note("scaled cache write, host tensors")
    nb, hkv, hq = 5, 2, 4
    on = lambda *s, dtype=torch.bfloat16: torch.zeros(s, dtype=dtype, device="cuda")  # noqa: E731
    u8 = dict(dtype=torch.uint8)
    args = dict(q=on(3, hq, 128), k=on(3, hkv, 128), v=on(3, hkv, 128), cos_sin=on(9, 128, dtype=torch.float32),
                positions=on(3, dtype=torch.int32), slots=torch.arange(3, device="cuda"), q_out=on(3, hq, 128),
                k_blocks=on(nb, hkv, 16, 128, **u8), v_blocks=on(nb, hkv, 128, 16, **u8), k_scale=on(nb, hkv, **u8),
                v_scale=on(nb, hkv, **u8), q_weight=on(128), k_weight=on(128))
    shape = gpu_lib.qk_shape(3, hq, hkv, nb, 9, block_scales=True)
    for name, t in args.items():
        with pytest.raises(ValueError, match="current device"):
            gpu_lib.qk_norm_rope_append_scaled(**dict(args, **{name: t.cpu()}), shape=shape)
    assert (args["k_scale"] == 0).all() and (args["v_scale"] == 0).all()
    gpu_lib.qk_norm_rope_append_scaled(**dict(args, k_blocks=args["k_blocks"].view(torch.float8_e4m3fn),
                                              k_scale=args["k_scale"].view(torch.float8_e8m0fnu)), shape=shape)
    torch.cuda.synchronize()
    assert (args["k_scale"][0] == 1).all() and (args["v_scale"][0] == 1).all()   # (zeros take the least byte)
