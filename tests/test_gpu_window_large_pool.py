"""Caches of more than 4 GiB: blocks behind the first 2^32 bytes are read and written as those before them."""
import numpy as np
import pytest
import torch

import window_cases as wc
from window_cases import Case

pytestmark = pytest.mark.gpu

HKV, NB = 4, 560_000     # 4.6 GB of K and as much of V, one byte a value


@pytest.fixture(scope="module")
def pool():
    k = torch.zeros((NB, HKV, 16, 128), dtype=torch.uint8, device="cuda")
    v = torch.zeros((NB, HKV, 128, 16), dtype=torch.uint8, device="cuda")
    yield k, v
    del k, v
    torch.cuda.empty_cache()


def high(c, d, pool):
    """The case's cache as the last blocks of the pool."""
    k, v = pool
    first = NB - c.nb
    k[first:], v[first:] = d["k"], d["v"]
    big = dict(d, k=k, v=v, tables=torch.where(d["tables"] >= 0, d["tables"] + first, d["tables"]))
    if c.fmt == "e4m3_block":
        for n in ("ks", "vs"):
            big[n] = torch.full((NB, HKV), 255, dtype=torch.uint8, device="cuda")
            big[n][first:] = d[n]
    return big


@pytest.mark.parametrize("fmt", ["fp8_e4m3", "e4m3_block"])
def test_attention(gpu_lib, pool, fmt):
    print(f"[gpu-test] large pool attention {fmt}", flush=True)
    rng = np.random.default_rng(1)
    c = Case(rng, [100, 700, 33], None, 8, HKV, fmt, 90, 5)
    d = c.device()
    want = [wc.decode(gpu_lib, c, d=d, **kw) for kw in ({}, dict(partition_tokens=64))]
    p = Case(rng, [400, 700] + [3] * 64, [100, 90] + [0] * 64, 8, HKV, fmt, 90, 5)
    f = Case(rng, [400, 700], [10, 9], 8, HKV, fmt, 90, 5)
    pd, fd = p.device(), f.device()
    wants = [wc.prefill(gpu_lib, p, d=pd), wc.prefill(gpu_lib, f, d=fd)]
    for x, dd, ws in ((c, d, want), (p, pd, wants[:1]), (f, fd, wants[1:])):
        big, nb = high(x, dd, pool), x.nb
        x.nb = NB
        got = [wc.decode(gpu_lib, x, d=big, **kw) for kw in ({}, dict(partition_tokens=64))] if x is c else [
            wc.prefill(gpu_lib, x, d=big)]
        x.nb = nb
        for a, b in zip(got, ws):
            assert torch.equal(a, b)


def test_append(gpu_lib, pool):
    print("[gpu-test] large pool append", flush=True)
    k, v = pool
    k.zero_(), v.zero_()
    rows, n = 40, 6
    first = NB - n
    g = torch.Generator(device="cuda").manual_seed(1)
    new = torch.randn((2, rows, HKV, 128), generator=g, device="cuda").to(torch.bfloat16)
    t = torch.arange(rows, device="cuda")
    outs = []
    for base, (kc, vc) in ((first, pool), (0, [torch.zeros_like(x[:n]) for x in pool])):
        kc[base:base + n], vc[base:base + n] = 0, 0
        ks, vs = (torch.full((len(kc), HKV), 119, dtype=torch.uint8, device="cuda") for _ in range(2))
        sh = gpu_lib.qk_shape(rows, 0, HKV, len(kc), 100, rotary_dim=0, block_scales=True)
        gpu_lib.qk_norm_rope_append_scaled(None, new[0], new[1], None, t.int(), t + 16 * base + 5, None, kc, vc, ks, vs,
                                           sh)
        torch.cuda.synchronize()
        outs.append([x[base:base + n].clone() for x in (kc, vc, ks, vs)])
    for a, b in zip(*outs):
        assert torch.equal(a, b)
    assert outs[0][0].any() and not k[:first].any()
