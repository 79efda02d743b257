"""Small paged caches for the tests of windows and block scales: everything that no row sees is poisoned."""
import numpy as np
import torch

import workloads
from oracle import window as ow

FMTS = ["bf16", "fp8_e4m3", "e4m3_block"]
NAN_CODE = {"bf16": 0x7FC0, "fp8_e4m3": 0x7F, "e4m3_block": 0x7F}


def codes(rng, fmt, shape, spread=1.0):
    x = rng.standard_normal(shape).astype(np.float32) * spread
    return workloads.to_bf16_codes(x) if fmt == "bf16" else workloads.to_e4m3_codes(x * 93.0)


class Case:
    """ctx[s] cached tokens, the last rows[s] of them query rows (rows None: decode, one row a sequence).

    Hidden tokens, unused blocks and their scales are NaN; table entries of
    blocks without a token that some row sees are -1."""

    def __init__(self, rng, ctx, rows, hq, hkv, fmt, window, n_sink, spare=5, max_blocks=None, spread=1.0):
        self.fmt, self.hq, self.hkv, self.window, self.n_sink = fmt, hq, hkv, window, n_sink
        self.ctx = np.asarray(ctx, np.int32)
        self.rows = None if rows is None else np.asarray(rows, np.int32)
        b = len(ctx)
        n = np.minimum(1, self.ctx) if rows is None else self.rows
        blocks = -(-self.ctx // 16)
        self.nb = int(blocks.sum()) + spare
        self.max_blocks = max(int(blocks.max(initial=0)), 1) if max_blocks is None else max_blocks
        perm = rng.permutation(self.nb)
        self.tables = np.full((b, self.max_blocks), -1, np.int32)
        dead = np.ones((self.nb, 16), bool)
        at = 0
        for s in range(b):
            some = ow.sees(int(self.ctx[s]), int(n[s]), window, n_sink).any(0)
            for j in range(blocks[s]):
                here = some[16 * j:16 * j + 16]
                if here.any():
                    self.tables[s, j] = perm[at]
                    dead[perm[at], :len(here)] = ~here
                at += 1
        self.k, self.v = codes(rng, fmt, (self.nb, hkv, 16, 128), spread), codes(rng, fmt, (self.nb, hkv, 128, 16))
        blk, slot = np.nonzero(dead)
        self.k[blk, :, slot, :] = NAN_CODE[fmt]
        self.v[blk, :, :, slot] = NAN_CODE[fmt]
        self.ks = self.vs = None
        if fmt == "fp8_e4m3":
            self.ks, self.vs = ((rng.random(hkv) * 0.01 + 0.006).astype(np.float32) for _ in range(2))
        elif fmt == "e4m3_block":
            self.ks, self.vs = (rng.integers(118, 123, (self.nb, hkv)).astype(np.uint8) for _ in range(2))
            for x in (self.ks, self.vs):
                x[dead.all(1)] = 255
        self.total = b if rows is None else int(self.rows.sum())
        self.q = workloads.to_bf16_codes(rng.standard_normal((self.total, hq, 128)).astype(np.float32))
        self.q_start = None if rows is None else np.concatenate([[0], np.cumsum(self.rows)]).astype(np.int32)
        self.scale = 128 ** -0.5

    def oracle(self):
        return ow.window_attention(self.q, self.k, self.v, self.tables, self.ctx, self.q_start, self.scale, self.window,
                                   self.n_sink, self.fmt, self.ks, self.vs)

    def device(self):
        return {n: dev(getattr(self, n)) for n in ("q", "k", "v", "tables", "ctx", "ks", "vs", "q_start")}


def dev(a):
    if a is None:
        return None
    a = np.ascontiguousarray(a)
    return torch.from_numpy(a.view(np.int16) if a.dtype == np.uint16 else a).cuda()


def decoder(lib, c, max_ctx=None, **kw):
    return lib.WindowDecoder(len(c.ctx), c.hq, c.hkv, c.max_blocks, int(c.ctx.max(initial=0)) if max_ctx is None else
                             max_ctx, c.nb, c.window, c.n_sink, kv_fp8=c.fmt != "bf16",
                             block_scales=c.fmt == "e4m3_block", **kw)


def decode(lib, c, dec=None, d=None, out=None, **kw):
    d = c.device() if d is None else d
    dec = decoder(lib, c, **kw) if dec is None else dec
    out = torch.full((c.total, c.hq, 128), 77.0, dtype=dec.out_dtype, device="cuda") if out is None else out
    dec(d["q"], d["k"], d["v"], d["tables"], d["ctx"], c.scale, out, d["ks"], d["vs"])
    return out


def prefill_shape(lib, c, max_ctx=None, **kw):
    return lib.prefill_shape(len(c.ctx), c.hq, c.hkv, c.max_blocks, int(c.ctx.max()) if max_ctx is None else max_ctx,
                             c.nb, c.total, kv_fp8=c.fmt != "bf16", block_scales=c.fmt == "e4m3_block", **kw)


def prefill(lib, c, d=None, out=None, out_fp32=False, **kw):
    d = c.device() if d is None else d
    if out is None:
        out = torch.full((c.total, c.hq, 128), 77.0, dtype=torch.float32 if out_fp32 else torch.bfloat16, device="cuda")
    lib.window_prefill_attention(d["q"], d["k"], d["v"], d["tables"], d["ctx"], d["q_start"], c.scale, c.window,
                                 c.n_sink, out, prefill_shape(lib, c, out_fp32=out_fp32, **kw), d["ks"], d["vs"])
    return out


def check(out, ref, bound):
    got = out.double().cpu().numpy()
    assert np.isfinite(got).all()
    over = np.abs(got - ref) / bound
    assert over.max() <= 1.0, f"{over.max():.2f} of the bound at {np.unravel_index(over.argmax(), over.shape)}"
