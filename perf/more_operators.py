"""Timed operators: sliding windows with sinks, and a cache with a scale for each block, through the public entry points.

Two things that deployments of a paged cache add to the decode and prefill of
full contexts:
  * layers that see a window: a token attends the `window` tokens up to its
    own, and the sequence's first `sinks` tokens, which stay visible; blocks
    that nothing sees any more have left the table (-1);
  * an e4m3 cache that needs no calibration: each (block, KV head) tile has a
    scale of its own, a power of two held as one exponent byte (E8M0), set when
    its tokens are written and raised when a later token of the block needs it.
Three operators carry them:
  decode   WindowDecoder: one query token a sequence
  prefill  window_prefill_attention: chunks of prompts, or a few drafts in a row
  append   qk_norm_rope_append_scaled: RMS norm and rotation of queries and keys
           and the write of K and V into the cache with block scales
Each cache type meets each form of attention: bf16, e4m3 with a scale for each
head, e4m3 with block scales; a window as long as the longest context is none.
Sizes are those of this library's deployments (64 query / 8 KV heads, 64 / 4
heads, pools with C_max 8K and 64K, chunks of 2,048 tokens) and of their small,
ragged and lightly loaded ends.

A case is a dict of plain values:
  kind                     "decode", "prefill" or "append"
  batch, hq, hkv, c_max
  cache                    "bf16", "head" (e4m3, a scale for each head) or
                           "block" (e4m3, a scale for each block and head)
  window, sinks            window 0: the whole context
  evicted                  blocks that no row sees are not in the table
  lens, lens_seed          how cached lengths are drawn (see lengths()); they
                           belong to the case, values belong to the seed
  rows                     new tokens of a sequence (decode: 1)
  ragged                   each sequence has 1 .. rows new tokens
  prompt                   new tokens are whole prompts instead
  idle                     decode: every idle-th sequence is empty
  pad                      append: rows behind the last sequence, in no slot
  norm, rotary, paired     append: with the two norms; rotated dimensions; the
                           pairs are neighbours (else halves)
  fused                    append: q, k and v are slices of one projection
"""
import math

import numpy as np
import torch

own = False

BLOCK = 16
DIM = 128
SCALE = 1.0 / math.sqrt(DIM)
E4M3_MAX = 448.0
EPS = 1e-6

LLAMA = dict(hq=64, hkv=8)
QWEN = dict(hq=64, hkv=4)


def _case(name, kind, lens, batch, c_max, lens_seed=0, **more):
    return dict(dict(name=name, kind=kind, lens=lens, batch=batch, c_max=c_max, lens_seed=lens_seed, cache="block",
                     window=0, sinks=0, evicted=False, rows=1, ragged=False, prompt=False, idle=0, pad=0, norm=False,
                     rotary=DIM, paired=False, fused=False), **more)


def listed():
    return [
        # A handful of short chats on a small model with a short window.
        _case("decode_window_tiny_bf16", "decode", "uniform", 3, 512, 1, cache="bf16", window=96, sinks=1, hq=8, hkv=2),
        # The short pool at its full batch, a windowed layer.
        _case("decode_window_short_bf16", "decode", "lognormal", 128, 8192, 2, cache="bf16", window=1024, sinks=4,
              **LLAMA),
        # The long pool: what has left the window has left the cache too.
        _case("decode_window_long_fp8", "decode", "pareto", 64, 65536, 3, cache="head", window=4096, sinks=64,
              evicted=True, **QWEN),
        # The short pool of the fp8 deployment, uncalibrated, whole contexts; a
        # batch captured larger than it is.
        _case("decode_scaled_short", "decode", "lognormal", 256, 8192, 4, idle=17, **QWEN),
        # Few long sequences, window and block scales together.
        _case("decode_window_scaled_long", "decode", "pareto", 16, 65536, 5, window=2048, sinks=16, evicted=True,
              **LLAMA),
        # Four chunks of long prompts in a windowed layer: work for the matrix cores.
        _case("prefill_window_chunks_bf16", "prefill", "chunks", 4, 32768, 6, cache="bf16", window=4096, sinks=4,
              rows=2048, **LLAMA),
        # Fresh prompts of ragged lengths, a short window without sinks.
        _case("prefill_window_prompts_fp8", "prefill", "lognormal", 11, 8192, 7, cache="head", window=512, prompt=True,
              **QWEN),
        # Chunks over an uncalibrated cache, whole contexts.
        _case("prefill_scaled_chunks", "prefill", "chunks", 3, 8192, 8, rows=2048, **QWEN),
        # A few drafts in a row of each sequence, checked in one pass.
        _case("prefill_window_scaled_drafts", "prefill", "uniform", 24, 2048, 9, window=256, sinks=4, rows=6,
              ragged=True, hq=16, hkv=4),
        # An ordinary decode step's write: one token into each sequence's last block.
        _case("append_scaled_decode", "append", "uniform", 256, 512, 10, norm=True, **QWEN),
        # Drafted tokens: blocks that are begun, crossed and ended.
        _case("append_scaled_drafts", "append", "uniform", 96, 1024, 11, rows=7, ragged=True, fused=True, **LLAMA),
        # Prompts of ragged lengths, in a batch padded to a captured size.
        _case("append_scaled_prompts", "append", "lognormal", 9, 8192, 12, prompt=True, pad=61, fused=True, **LLAMA),
    ]


def lengths(case):
    """(tokens cached before the call's own, tokens the call adds), int64 [batch] each.

    For attention the added tokens are in the cache already."""
    rng = np.random.default_rng(case["lens_seed"])
    n, c_max = case["batch"], case["c_max"]
    if case["lens"] == "lognormal":  # prompts of median 600 tokens and up to 428 generated ones
        t = np.clip(np.rint(rng.lognormal(math.log(600.0), 1.2, n)), 16, 8192) + rng.integers(1, 429, n)
    elif case["lens"] == "pareto":  # alpha 1.5 between 8,192 tokens and c_max
        t = np.floor(8192 / (1.0 - rng.random(n) * (1.0 - (8192 / c_max) ** 1.5)) ** (1 / 1.5))
    elif case["lens"] == "chunks":  # chunks that end anywhere in the prompt, its end among them
        t = np.concatenate([[c_max], np.exp(rng.uniform(math.log(min(case["rows"], c_max)), math.log(c_max), n - 1))])
    else:
        t = rng.integers(1, c_max + 1, n)
    t = np.clip(t, 1, c_max).astype(np.int64)
    if case["prompt"]:
        return np.zeros(n, dtype=np.int64), t
    new = np.full(n, case["rows"], dtype=np.int64)
    if case["ragged"]:
        new = rng.integers(1, case["rows"] + 1, n)
    if case["idle"]:
        at = np.arange(n) % case["idle"] == case["idle"] - 1
        t[at] = new[at] = 0
    new = np.minimum(new, t)
    return t - new, new


def _window(case):
    return case["window"] or case["c_max"]


def _blocks(case):
    """Of each sequence: its blocks, the first one that the window of its first row reaches, sink blocks before that."""
    ctx, new = lengths(case)
    first = np.maximum(ctx + 1 - _window(case), 0) // BLOCK
    return -(-(ctx + new) // BLOCK), first, np.minimum(-(-case["sinks"] // BLOCK), first)


def _pool(case):
    """Blocks of the pool."""
    every, first, head = _blocks(case)
    used = int((every - first + head).sum() if case["evicted"] else every.sum())
    return used + 1 + used // 8 + case["batch"]


def _seen(case):
    """(tokens that some row of each sequence sees, pairs of a row and a token that it sees)"""
    ctx, new = lengths(case)
    w, s = _window(case), case["sinks"]
    lo = np.maximum(ctx + 1 - w, 0)
    pairs = 0
    for c, n in zip(ctx.tolist(), new.tolist()):
        p = np.arange(c, c + n)
        pairs += int((np.minimum(p + 1, w) + np.minimum(s, np.maximum(p + 1 - w, 0))).sum())
    return int((ctx + new - lo + np.minimum(s, lo)).sum()), pairs


def work(case):
    hq, hkv = case["hq"], case["hkv"]
    eb, kv_token = (2 if case["cache"] == "bf16" else 1), hkv * DIM * 2
    rows = int(lengths(case)[1].sum())
    if case["kind"] == "append":
        return {"bytes": rows * (hq * DIM * 4 + kv_token * (2 + eb) + case["rotary"] * 4 + 12),
                "flops": rows * (hq + hkv) * DIM * (7 if case["norm"] else 3)}
    tokens, pairs = _seen(case)
    scales = tokens // BLOCK * hkv * 2 if case["cache"] == "block" else 0
    return {"bytes": tokens * kv_token * eb + scales + max(rows, 1) * hq * DIM * 4, "flops": 4 * DIM * hq * pairs}


def draw(rng):
    """rng: a random.Random"""
    most = {}
    for c in listed():
        w = work(c)
        old = most.get(c["kind"], {"bytes": 0, "flops": 0})
        most[c["kind"]] = {k: max(w[k], old[k]) for k in w}
    kind = rng.choice(["decode", "decode", "prefill", "prefill", "append"])
    log = lambda lo, hi: round(math.exp(rng.uniform(math.log(lo), math.log(hi))))  # noqa: E731
    while True:
        hkv = rng.choice([1, 2, 3, 4, 8, 8])
        group = rng.choice([1, 2, 4, 5, 7, 8, 8, 12, 16])
        c = _case("", kind, rng.choice(["uniform", "lognormal"]), log(1, 512), log(64, 65536), rng.randrange(1 << 30),
                  hkv=hkv, hq=hkv * group)
        del c["name"]
        if kind == "append":
            c["c_max"] = log(64, 4096)
            c["prompt"] = rng.random() < 0.4
            if not c["prompt"] and rng.random() < 0.6:
                c["rows"] = log(2, 64)
            c["pad"] = rng.choice([0, 0, 5, 40])
            c["norm"], c["paired"], c["fused"] = rng.random() < 0.5, rng.random() < 0.3, rng.random() < 0.5
            c["rotary"] = rng.choice([DIM, DIM, 64, 32])
        else:
            c["cache"] = rng.choice(["bf16", "head", "block"])
            if c["cache"] != "block" or rng.random() < 0.5:
                c["window"] = log(16, 8192)
                c["sinks"] = rng.choice([0, 1, 4, 4, 17, 64, 200])
                c["evicted"] = rng.random() < 0.5
            if c["c_max"] > 16384 and rng.random() < 0.7:
                c["lens"] = "pareto"
            if kind == "decode":
                c["idle"] = rng.choice([0, 0, 3, 20])
            else:
                c["batch"] = log(1, 64)
                c["rows"] = log(1, 2048)
                c["prompt"] = rng.random() < 0.3
                if c["rows"] >= 256 and rng.random() < 0.6:
                    c["lens"] = "chunks"
        c["ragged"] = c["rows"] > 1 and rng.random() < 0.5
        if c["lens"] == "lognormal" and c["c_max"] < 2048:
            c["lens"] = "uniform"
        if c["prompt"] and c["lens"] in ("chunks", "pareto"):
            c["lens"] = "uniform"
        w, (every, first, head), new = work(c), _blocks(c), lengths(c)[1]
        span = int((every - first + head).max()) * BLOCK
        padded = c["batch"] * span * max(hkv * DIM, c["hq"] * int(new.max())) * 4 if kind != "append" else 0
        size = _pool(c) * hkv * BLOCK * DIM * 2 * (2 if c["cache"] == "bf16" else 1)
        if all(w[k] <= most[kind][k] for k in w) and padded <= 14e9 and size <= (1.2e9 if kind == "append" else 8e9):
            if new.any():
                return c


# ------------------------------------------------------------------ inputs

def _inputs(case, seed):
    """Every input of the pass, on the GPU, from the seed alone."""
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    rng = np.random.default_rng(seed)
    ctx, new = lengths(case)
    b, hq, hkv, nb = case["batch"], case["hq"], case["hkv"], _pool(case)
    max_blocks = -(-case["c_max"] // BLOCK)
    up = lambda a, t: torch.from_numpy(np.ascontiguousarray(a, dtype=t)).to(dev)  # noqa: E731
    every, first, head = _blocks(case)
    perm = rng.permutation(nb).astype(np.int32)
    tables = np.full((b, max_blocks), -1, dtype=np.int32)
    at = 0
    for s in range(b):
        kept = np.arange(every[s])
        if case["evicted"]:
            kept = np.concatenate([kept[:head[s]], kept[first[s]:]])
        tables[s, kept] = perm[at:at + len(kept)]
        at += len(kept)
    x = dict(ks=None, vs=None, nb=nb, rows=int(new.sum()))

    def normal(*shape):
        return torch.randn(shape, generator=g, device=dev, dtype=torch.bfloat16)

    def cache(*shape):
        if case["cache"] == "bf16":
            return normal(*shape)
        t = torch.empty(shape, dtype=torch.uint8, device=dev)
        for i in range(0, nb, 8192):  # unit-variance values over a scale near 1 / 93
            part = torch.randn((min(8192, nb - i),) + shape[1:], generator=g, device=dev) * 93.0
            t[i:i + 8192] = part.clamp_(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn).view(torch.uint8)
        return t

    x["k"], x["v"] = cache(nb, hkv, BLOCK, DIM), cache(nb, hkv, DIM, BLOCK)
    if case["cache"] == "head":  # per-head scales of an amax near 4.5 standard deviations
        x["ks"], x["vs"] = ((4.5 + torch.rand(hkv, generator=g, device=dev)) / E4M3_MAX for _ in range(2))
    elif case["cache"] == "block":  # 2^-7 and 2^-6, a few louder and quieter tiles
        for n in ("ks", "vs"):
            u = torch.rand((nb, hkv), generator=g, device=dev)
            x[n] = (118 + (u > 0.03).int() + (u > 0.1).int() + (u > 0.5).int() + (u > 0.95).int()).to(torch.uint8)

    seq = np.repeat(np.arange(b), new)
    q_start = np.concatenate([[0], np.cumsum(new)])
    pos = ctx[seq] + np.arange(len(seq)) - q_start[seq]
    if case["kind"] != "append":
        x |= dict(q=normal(max(len(seq), b) if case["kind"] == "decode" else len(seq), hq, DIM),
                  tables=up(tables, np.int32), ctx=up(ctx + new, np.int32), q_start=up(q_start, np.int32),
                  span=int((every - first + head).max()), most_rows=int(new.max()))
        return x
    pad, rows = case["pad"], len(pos) + case["pad"]
    slots = tables[seq, pos // BLOCK].astype(np.int64) * BLOCK + pos % BLOCK
    x["slots"] = up(np.concatenate([slots, np.full(pad, -1)]), np.int64)
    x["pos"] = up(np.concatenate([pos, np.full(pad, -1)]), np.int32)
    # projections differ in size from head to head
    loud = torch.exp(0.5 * torch.randn((1, hq + 2 * hkv, 1), generator=g, device=dev)).to(torch.bfloat16)
    qkv = (normal(rows, hq + 2 * hkv, DIM) * loud).view(rows, -1)
    x["q"], x["k_new"], x["v_new"] = (t.view(rows, -1, DIM) for t in
                                      qkv.split([hq * DIM, hkv * DIM, hkv * DIM], dim=1))
    if not case["fused"]:
        x["q"], x["k_new"], x["v_new"] = (x[n].contiguous() for n in ("q", "k_new", "v_new"))
    half = case["rotary"] // 2
    turn = torch.arange(case["c_max"], device=dev, dtype=torch.float64)[:, None] \
        * 500000.0 ** (-torch.arange(half, device=dev, dtype=torch.float64) / half)
    x["cos_sin"] = torch.cat([turn.cos(), turn.sin()], dim=1).float()
    x["qw"] = x["kw"] = None
    if case["norm"]:
        x["qw"], x["kw"] = (1 + 0.2 * normal(DIM) for _ in range(2))
    return x


def prepare(case, seed):
    x = _inputs(case, seed)
    x["case"] = case
    if not own:
        return x
    from paper_2604_08075_amd import binding
    b, hq, hkv, nb, rows = case["batch"], case["hq"], case["hkv"], x["nb"], x["rows"]
    max_blocks = -(-case["c_max"] // BLOCK)
    fp8, scaled = case["cache"] != "bf16", case["cache"] == "block"
    if case["kind"] == "decode":
        x["decoder"] = binding.WindowDecoder(b, hq, hkv, max_blocks, case["c_max"], nb, _window(case), case["sinks"],
                                             kv_fp8=fp8, block_scales=scaled)
        x["out"] = x["decoder"].new_out()
    elif case["kind"] == "prefill":
        x["shape"] = binding.prefill_shape(b, hq, hkv, max_blocks, case["c_max"], nb, rows, kv_fp8=fp8,
                                           block_scales=scaled)
        x["out"] = torch.empty_like(x["q"])
    else:
        x["shape"] = binding.qk_shape(rows + case["pad"], hq, hkv, nb, case["c_max"], rotary_dim=case["rotary"],
                                      interleaved=case["paired"], kv_fp8=True, q_stride=x["q"].stride(0),
                                      k_stride=x["k_new"].stride(0), v_stride=x["v_new"].stride(0), block_scales=True)
        x["q_out"] = torch.zeros((rows + case["pad"], hq, DIM), dtype=torch.bfloat16, device="cuda")
    return x


def _values(case, t):
    """What a cache tensor stands for, in its own type."""
    return t if case["cache"] == "bf16" else t.view(torch.float8_e4m3fn)


def _written(x, case, q):
    """What an append returns: the queries, the caches and their scales."""
    return [q, _values(case, x["k"]), _values(case, x["v"]), x["ks"].view(torch.float8_e8m0fnu),
            x["vs"].view(torch.float8_e8m0fnu)]


def run(x):
    case = x["case"]
    if own:
        return _run_own(x, case)
    return _append(x, case) if case["kind"] == "append" else _attend(x, case)


def _run_own(x, case):
    from paper_2604_08075_amd import binding
    if case["kind"] == "decode":
        return x["decoder"](x["q"], x["k"], x["v"], x["tables"], x["ctx"], SCALE, x["out"], x["ks"], x["vs"])
    if case["kind"] == "prefill":
        binding.window_prefill_attention(x["q"], x["k"], x["v"], x["tables"], x["ctx"], x["q_start"], SCALE,
                                         _window(case), case["sinks"], x["out"], x["shape"], x["ks"], x["vs"])
        return x["out"]
    binding.qk_norm_rope_append_scaled(x["q"], x["k_new"], x["v_new"], x["cos_sin"], x["pos"], x["slots"], x["q_out"],
                                       x["k"], x["v"], x["ks"], x["vs"], x["shape"], x["qw"], x["kw"], EPS)
    return _written(x, case, x["q_out"][:x["rows"]])


# ------------------------------------------------------------------ plain forms

def _attend(x, case):
    hq, hkv, b, dev = case["hq"], case["hkv"], case["batch"], x["q"].device
    group, w, sinks = hq // hkv, _window(case), case["sinks"]
    t = x["ctx"].long()
    if case["kind"] == "decode":  # every sequence has its row, empty ones too
        n_max, n, start = 1, torch.ones_like(t), torch.arange(b, device=dev)
    else:
        n_max, n, start = x["most_rows"], x["q_start"].diff().long(), x["q_start"][:-1].long()
    # the blocks that some row sees: the sinks', then the window's
    first = (t - n + 1 - w).clamp(min=0) // BLOCK
    head = first.clamp(max=-(-sinks // BLOCK))
    j = torch.arange(max(x["span"], 1), device=dev)
    blk = torch.where(j < head[:, None], j, j - head[:, None] + first[:, None])
    ids = x["tables"].gather(1, blk.clamp(max=x["tables"].shape[1] - 1)).clamp(min=0).long()
    k, v = _values(case, x["k"])[ids].float(), _values(case, x["v"])[ids].float()  # [b, blocks, hkv, ..]
    if case["cache"] == "head":
        k, v = k * x["ks"][:, None, None], v * x["vs"][:, None, None]
    elif case["cache"] == "block":
        k = k * torch.exp2(x["ks"][ids].float() - 127)[..., None, None]
        v = v * torch.exp2(x["vs"][ids].float() - 127)[..., None, None]
    k = k.permute(0, 2, 4, 1, 3).reshape(b * hkv, DIM, -1)
    v = v.permute(0, 2, 1, 4, 3).reshape(b * hkv, -1, DIM)
    i = torch.arange(n_max, device=dev)
    row = (start[:, None] + i).clamp(max=x["q"].shape[0] - 1)
    q = x["q"][row].float().view(b, n_max, hkv, group, DIM).permute(0, 2, 1, 3, 4).reshape(b * hkv, -1, DIM) * SCALE
    # the row at position p sees p - w < token <= p, and token < sinks
    token = (blk[:, :, None] * BLOCK + torch.arange(BLOCK, device=dev)).view(b, 1, -1)
    p = (t - n)[:, None, None] + i[:, None]
    see = (token <= p) & ((token > p - w) | (token < sinks))
    z = (q @ k).view(b, hkv, n_max, group, -1).masked_fill_(~see[:, None, :, None], -math.inf)
    z = z.sub_(z.amax(-1, keepdim=True).clamp(min=-1e30)).exp_()
    z = z.div_(z.sum(-1, keepdim=True).clamp(min=1e-30)).view(b * hkv, n_max * group, -1)
    o = (z @ v).view(b, hkv, n_max, group, DIM).permute(0, 2, 1, 3, 4).reshape(b, n_max, hq, DIM)
    return o[i[None, :] < n[:, None]].to(torch.bfloat16)


def _turned(case, t, weight, cs, kind):
    """Norm and rotation of [rows, heads, DIM]."""
    t = t.to(kind)
    if weight is not None:
        t = t * torch.rsqrt(t.square().mean(-1, keepdim=True) + EPS) * weight.to(kind)
    rot = case["rotary"]
    cos, sin = cs.to(kind)[:, None, :].chunk(2, dim=-1)
    a, b = (t[..., 0:rot:2], t[..., 1:rot:2]) if case["paired"] else t[..., :rot].chunk(2, dim=-1)
    y = [a * cos - b * sin, b * cos + a * sin]
    y = torch.stack(y, dim=-1).flatten(-2) if case["paired"] else torch.cat(y, dim=-1)
    return torch.cat([y, t[..., rot:]], dim=-1)


def _exponent(amax):
    """The byte of the smallest power of two, 2^(byte - 127), over which amax is at most 448."""
    m, e = torch.frexp(amax)
    return torch.where(amax > 0, e + 127 - 9 + (m > 0.875), 1).clamp(1, 247)


def _append(x, case):
    n = x["rows"]
    cs = x["cos_sin"][x["pos"][:n].long()]
    q = _turned(case, x["q"][:n], x["qw"], cs, torch.float32).to(torch.bfloat16)
    blk, off = x["slots"][:n] // BLOCK, x["slots"][:n] % BLOCK
    begins = torch.cat([blk.new_ones(1, dtype=torch.bool), blk[1:] != blk[:-1]])
    run, run_blk, run_off = begins.cumsum(0) - 1, blk[begins], off[begins]
    earlier = torch.arange(BLOCK, device=q.device)[None, :] < run_off[:, None]  # tokens of the block that stay
    # (64 bits: whether an amax lies just above or below a power of two)
    k = _turned(case, x["k_new"][:n], x["kw"], cs, torch.float64)
    for new, cache, scale in ((k, x["k"], x["ks"]), (x["v_new"][:n].double(), x["v"].transpose(2, 3), x["vs"])):
        amax = new.new_zeros(len(run_blk), case["hkv"])
        amax.scatter_reduce_(0, run[:, None].expand(-1, case["hkv"]), new.abs().amax(-1), "amax")
        old = scale[run_blk].int() * (run_off > 0)[:, None]
        byte = torch.maximum(_exponent(amax), old)
        tile = cache[run_blk].view(torch.float8_e4m3fn).float()
        shrunk = tile * torch.exp2((old - byte).float())[..., None, None]
        tile = torch.where(earlier[:, None, :, None], shrunk, tile).to(torch.float8_e4m3fn).view(torch.uint8)
        code = (new * torch.exp2((127 - byte).double())[run][..., None]).float().to(torch.float8_e4m3fn)
        tile[run, :, off] = code.view(torch.uint8)
        cache[run_blk] = tile
        scale[run_blk] = byte.to(torch.uint8)
    return _written(x, case, q)


# ------------------------------------------------------------------ from the definitions, in 64 bits

def exact(case, seed):
    x = _inputs(case, seed)
    return _exact_append(x, case) if case["kind"] == "append" else _exact_attend(x, case)


def _exact_cache(case, t):
    return t.double() if case["cache"] == "bf16" else t.view(torch.float8_e4m3fn).double()


def _exact_attend(x, case):
    hq, hkv = case["hq"], case["hkv"]
    group = hq // hkv
    out = torch.zeros(x["q"].shape, dtype=torch.float64, device=x["q"].device)
    q_start = list(range(case["batch"] + 1)) if case["kind"] == "decode" else x["q_start"].tolist()
    for s, t in enumerate(x["ctx"].tolist()):
        r0, r1 = q_start[s], q_start[s + 1]
        p = torch.arange(t - (r1 - r0), t, device=out.device)[:, None]
        tokens = torch.arange(t, device=out.device)
        lo = max(0, t - (r1 - r0) + 1 - _window(case))
        tokens = tokens[(tokens >= lo) | (tokens < case["sinks"])]
        if len(tokens) == 0:
            continue
        ids, off = x["tables"][s].long()[tokens // BLOCK], tokens % BLOCK
        hidden = (tokens > p) | ((tokens <= p - _window(case)) & (tokens >= case["sinks"]))
        for g in range(hkv):
            k, v = _exact_cache(case, x["k"][ids, g, off]), _exact_cache(case, x["v"][ids, g, :, off])
            if case["cache"] == "head":
                k, v = k * x["ks"][g].double(), v * x["vs"][g].double()
            elif case["cache"] == "block":
                k = k * 2.0 ** (x["ks"][ids, g].double() - 127)[:, None]
                v = v * 2.0 ** (x["vs"][ids, g].double() - 127)[:, None]
            q = x["q"][r0:r1, g * group:(g + 1) * group].double()
            z = torch.einsum("rhd,td->rht", q, k) * SCALE
            z = torch.softmax(z.masked_fill(hidden[:, None], -math.inf), dim=-1)
            out[r0:r1, g * group:(g + 1) * group] = torch.einsum("rht,td->rhd", z, v)
    return out


def _exact_append(x, case):
    n, rot, half = x["rows"], case["rotary"], case["rotary"] // 2
    angle = x["cos_sin"][x["pos"][:n].long()].double()
    outs = []
    for t, w in ((x["q"], x["qw"]), (x["k_new"], x["kw"])):
        t = t[:n].double()
        if w is not None:
            t = t / (t.pow(2).sum(-1, keepdim=True) / DIM + EPS).sqrt() * w.double()
        y = t.clone()
        for d in range(half):
            i, j = (2 * d, 2 * d + 1) if case["paired"] else (d, d + half)
            c, s = angle[:, None, d], angle[:, None, half + d]
            y[..., i] = t[..., i] * c - t[..., j] * s
            y[..., j] = t[..., j] * c + t[..., i] * s
        outs.append(y)
    slots = x["slots"][:n].tolist()
    ends = [r for r in range(1, n) if slots[r] // BLOCK != slots[r - 1] // BLOCK] + [n]
    if len(ends) > 20000:
        return None
    caches = [_exact_cache(case, x["k"]), _exact_cache(case, x["v"]).transpose(2, 3).clone()]
    for new, cache, bytes_ in zip((outs[1], x["v_new"][:n].double()), caches, (x["ks"], x["vs"])):
        scale = torch.exp2(bytes_.double() - 127)
        r0 = 0
        for r1 in ends:
            block, at = slots[r0] // BLOCK, slots[r0] % BLOCK
            want = torch.exp2(torch.ceil(torch.log2(new[r0:r1].abs().amax((0, 2)) / E4M3_MAX))).clamp(min=2.0 ** -126)
            if at:
                want = torch.maximum(want, scale[block])
                cache[block, :, :at] *= (scale[block] / want)[:, None, None]
            cache[block, :, at:at + r1 - r0] = (new[r0:r1] / want[:, None]).transpose(0, 1)
            r0 = r1
    return [outs[0], caches[0], caches[1].transpose(2, 3), None, None]
