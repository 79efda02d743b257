"""Timed operators: a step that verifies drafted tokens, through the package's public entry points.

Speculative serving adds a tree of drafted tokens to every sequence and
checks all of them in one pass of the model.  Four operators carry such a
step over this library's paged cache:
  tables  kv_tables_step: block tables, slot maps, positions and tree masks
          from the requests' lengths, against a ring of free blocks
  rope    qk_norm_rope_append: RMS norm of each query and key head, rotary
          position embedding, K and V written into their cache slots
  tree    TreeDecoder: attention of the drafted tokens over the cache, each
          over the committed tokens and its own ancestors
  accept  kv_cache_accept: the accepted path's K and V moved to the front of
          the drafted slots, in every layer

The same calls with one token a sequence, or with the tokens of a prompt, are
the ordinary decode and prefill steps; the cases hold those ends too.  Sizes
are those of this library's deployments (64 query / 8 KV heads with a bf16
cache, 64 / 4 heads with an e4m3 cache, pools with C_max 8K and 64K) and of
their small, ragged and lightly loaded ends.

A case is a dict of plain values:
  kind                     "tables", "rope", "tree" or "accept"
  batch, hq, hkv, c_max, fp8
  lens, lens_seed          how cached lengths are drawn (see lengths()); they
                           belong to the case, values belong to the seed
  draft                    drafted tokens of a sequence; 0: ordinary tokens
  ragged                   each sequence drafts 1 .. draft tokens
  prompt                   tables, rope: whole prompts instead of one token
  done, tight              tables: every done-th sequence ends; the ring holds
                           too few blocks for the last sequences
  pad                      rope: rows behind the last sequence, in no slot
  norm, rotary, paired     rope: with the two norms; rotated dimensions; the
                           pairs are neighbours (else halves)
  fused                    rope: q, k and v are slices of one projection
  layers                   accept: caches that one call moves
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

LLAMA = dict(hq=64, hkv=8, fp8=False)
QWEN = dict(hq=64, hkv=4, fp8=True)


def _case(name, kind, lens, batch, c_max, lens_seed=0, **more):
    return dict(dict(name=name, kind=kind, lens=lens, batch=batch, c_max=c_max, lens_seed=lens_seed, draft=0,
                     ragged=False, prompt=False, done=0, tight=False, pad=0, norm=False, rotary=DIM, paired=False,
                     fused=False, layers=1), **more)


def listed():
    return [
        # An ordinary decode step of the short pool: one token a sequence, every
        # sixteenth or so takes a block.  Latency is all there is.
        _case("tables_decode", "tables", "lognormal", 256, 8192, 1, done=37, **QWEN),
        # A step that verifies trees: parents become masks and depths.
        _case("tables_trees", "tables", "lognormal", 96, 8192, 2, draft=32, ragged=True, done=16, **LLAMA),
        # A burst of fresh prompts, more than the pool can take.
        _case("tables_prompts", "tables", "lognormal", 512, 8192, 3, prompt=True, tight=True, **LLAMA),
        # A quiet decode step's rotation and cache write, no norms.
        _case("rope_decode_bf16", "rope", "uniform", 19, 1024, 4, fused=True, **LLAMA),
        # Drafts of the fp8 deployment: norms, rotation, e4m3 encoding.
        _case("rope_drafts_fp8", "rope", "uniform", 256, 512, 5, draft=7, norm=True, **QWEN),
        # Prompts of ragged lengths, in a batch padded to a captured size.
        _case("rope_prompts_bf16", "rope", "lognormal", 9, 8192, 6, prompt=True, pad=61, fused=True, **LLAMA),
        # A handful of short chats on a small model.
        _case("tree_tiny_bf16", "tree", "uniform", 3, 512, 7, draft=5, ragged=True, hq=8, hkv=2, fp8=False),
        # The short pool at its full batch, eight drafted tokens each.
        _case("tree_short_bf16", "tree", "lognormal", 128, 8192, 8, draft=8, **LLAMA),
        # The long pool, wide trees: enough queries to feed the matrix cores.
        _case("tree_long_bf16", "tree", "pareto", 16, 65536, 9, draft=32, **LLAMA),
        # The short pool of the fp8 deployment, GQA 16, ragged trees.
        _case("tree_short_fp8", "tree", "lognormal", 256, 8192, 10, draft=13, ragged=True, **QWEN),
        # The accepted paths of the short pool, sixteen layers in one call.
        _case("accept_short_bf16", "accept", "uniform", 128, 128, 11, draft=16, layers=16, **LLAMA),
        # The same for a few sequences of the fp8 deployment.
        _case("accept_quiet_fp8", "accept", "uniform", 5, 256, 12, draft=9, ragged=True, layers=6, **QWEN),
    ]


def lengths(case):
    """(tokens cached before the call's own, tokens the call adds), int64 [batch] each.

    For "tree" and "accept" the added tokens are in the cache already."""
    rng = np.random.default_rng(case["lens_seed"])
    n, c_max = case["batch"], case["c_max"]
    if case["lens"] == "lognormal":  # prompts of median 600 tokens and up to 428 generated ones
        t = np.clip(np.rint(rng.lognormal(math.log(600.0), 1.2, n)), 16, 8192) + rng.integers(1, 429, n)
    elif case["lens"] == "pareto":  # alpha 1.5 between 8,192 tokens and c_max
        t = np.floor(8192 / (1.0 - rng.random(n) * (1.0 - (8192 / c_max) ** 1.5)) ** (1 / 1.5))
    else:
        t = rng.integers(1, c_max + 1, n)
    t = np.clip(t, 1, c_max).astype(np.int64)
    if case["prompt"]:
        return np.zeros(n, dtype=np.int64), t
    new = np.full(n, max(case["draft"], 1), dtype=np.int64)
    if case["ragged"]:
        new = rng.integers(1, case["draft"] + 1, n)
    new = np.minimum(new, t)
    return t - new, new


def words(case):
    return (case["draft"] + 63) // 64


def _ends(case):
    """Which sequences are over (tables)."""
    at = np.arange(case["batch"])
    return at % case["done"] == case["done"] - 1 if case["done"] else at < 0


def _pool(case):
    """Blocks of the pool."""
    ctx, new = lengths(case)
    used = int((-(-(ctx + new) // BLOCK)).sum())
    return used + 1 + used // 8 + case["batch"]


def work(case):
    ctx, new = lengths(case)
    eb, hq, hkv, b = (1 if case["fp8"] else 2), case["hq"], case["hkv"], case["batch"]
    kv_token = hkv * DIM * 2
    if case["kind"] == "tables":
        end = _ends(case)
        rows = int(new[~end].sum())
        blocks = int((-(-(ctx + new) // BLOCK) - -(-ctx // BLOCK))[~end].sum() + (-(-ctx // BLOCK))[end].sum())
        return {"bytes": rows * (12 + 8 * words(case) + (4 if case["draft"] else 0)) + b * 28 + 8 * blocks, "flops": 0}
    if case["kind"] == "rope":
        rows = int(new.sum())
        return {"bytes": rows * (hq * DIM * 4 + kv_token * (2 + eb) + case["rotary"] * 4 + 12),
                "flops": rows * (hq + hkv) * DIM * (7 if case["norm"] else 3)}
    if case["kind"] == "tree":
        pairs = int((new * ctx + new).sum())
        return {"bytes": int((ctx + new).sum()) * kv_token * eb + int(new.sum()) * (hq * DIM * 4 + 8 * words(case)),
                "flops": 4 * DIM * hq * pairs}
    moved = sum(m for _, m in _paths(case))
    return {"bytes": max(2 * moved * kv_token * eb * case["layers"], 4 * b), "flops": 0}


def _paths(case):
    """The accepted drafts of each sequence, and how many of them change their slot (accept).

    A path starts at the root; what follows lies behind the accepted count."""
    rng = np.random.default_rng(case["lens_seed"] + 1)
    out = []
    for n in lengths(case)[1].tolist():
        a = 1 + int(rng.integers(0, (n + 1) // 2))
        tail = np.sort(rng.choice(np.arange(a, n), size=a - 1, replace=False)) if a > 1 else np.arange(0)
        out.append((np.concatenate([[0], tail]).astype(np.int32), a - 1))
    return out


def draw(rng):
    """rng: a random.Random"""
    most = {}
    for c in listed():
        w = work(c)
        old = most.get(c["kind"], {"bytes": 0, "flops": 0})
        most[c["kind"]] = {k: max(w[k], old[k]) for k in w}
    kind = rng.choice(["tables", "rope", "tree", "tree", "tree", "accept"])
    log = lambda lo, hi: round(math.exp(rng.uniform(math.log(lo), math.log(hi))))  # noqa: E731
    while True:
        hkv = rng.choice([1, 2, 3, 4, 8, 8])
        group = rng.choice([1, 2, 4, 5, 7, 8, 8, 12, 16])
        c = _case("", kind, rng.choice(["uniform", "lognormal"]), log(1, 512), 0, rng.randrange(1 << 30), hkv=hkv,
                  hq=hkv * group, fp8=rng.random() < 0.5)
        del c["name"]
        c["ragged"] = rng.random() < 0.6
        if kind == "tables":
            c["c_max"] = log(64, 16384)
            c["prompt"] = rng.random() < 0.4
            if not c["prompt"] and rng.random() < 0.6:
                c["draft"] = log(2, 128)
            c["done"] = rng.choice([0, 5, 16, 50])
            c["tight"] = rng.random() < 0.3
        elif kind == "rope":
            c["c_max"] = log(64, 4096)
            c["prompt"] = rng.random() < 0.5
            if not c["prompt"] and rng.random() < 0.6:
                c["draft"] = log(2, 64)
            c["pad"] = rng.choice([0, 0, 5, 40])
            c["norm"], c["paired"], c["fused"] = rng.random() < 0.5, rng.random() < 0.3, rng.random() < 0.5
            c["rotary"] = rng.choice([DIM, DIM, 64, 32])
        elif kind == "tree":
            c["c_max"] = log(64, 65536)
            c["draft"] = log(1, 128)
            if c["c_max"] > 16384 and rng.random() < 0.7:
                c["lens"] = "pareto"
        else:
            c["c_max"], c["batch"] = log(32, 512), log(1, 256)
            c["draft"], c["layers"], c["lens"] = log(2, 64), log(1, 20), "uniform"
        if c["lens"] == "lognormal" and c["c_max"] < 2048:
            c["lens"] = "uniform"
        c["ragged"] = c["ragged"] and c["draft"] > 0
        w, t = work(c), sum(lengths(c))
        padded = c["batch"] * int(t.max()) * max(hkv * DIM, c["hq"] * c["draft"]) * 4 if kind == "tree" else 0
        size = _pool(c) * hkv * BLOCK * DIM * 2 * (1 if c["fp8"] else 2) * c["layers"] if kind != "tables" else 0
        if all(w[k] <= most[kind][k] for k in w) and padded <= 9e9 and size <= (8e9 if kind == "tree" else 1.2e9):
            return c


# ------------------------------------------------------------------ inputs

def _parents(new, rng):
    """Trees of a beam-like shape: a token's parent lies in the first half of those before it."""
    i = np.concatenate([np.arange(n) for n in new]) if len(new) else np.arange(0)
    lo, hi = (i - 1) // 4, (i - 1) // 2
    p = lo + np.floor(rng.random(len(i)) * (hi - lo + 1)).astype(np.int64)
    return np.where(i == 0, -1, p).astype(np.int32)


def _masks(parents, new, w):
    """Ancestors and self of every row as bits, int64 [rows, w]."""
    out = np.zeros((len(parents), w), dtype=np.uint64)
    at = 0
    for n in new.tolist():
        for i in range(n):
            if parents[at + i] >= 0:
                out[at + i] = out[at + parents[at + i]]
            out[at + i, i // 64] |= np.uint64(1 << (i % 64))
        at += n
    return out.view(np.int64)


def _inputs(case, seed):
    """Every input of the pass, on the GPU, from the seed alone."""
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    rng = np.random.default_rng(seed)
    ctx, new = lengths(case)
    b, hq, hkv, nb = case["batch"], case["hq"], case["hkv"], _pool(case)
    max_blocks = -(-case["c_max"] // BLOCK)
    up = lambda a, t: torch.from_numpy(np.ascontiguousarray(a, dtype=t)).to(dev)  # noqa: E731
    perm = rng.permutation(nb).astype(np.int32)
    x = dict(ks=None, vs=None, nb=nb, rows=int(new.sum()))

    if case["kind"] == "tables":
        end = _ends(case)
        owned = -(-ctx // BLOCK)
        spare = (rng.random(b) < 0.2) & (ctx > 0)  # a block left over from refused drafts
        owned = np.minimum(owned + spare, max_blocks)
        n_owned = int(owned.sum())
        tables = np.full((b, max_blocks), -1, dtype=np.int32)
        at = 0
        for s in range(b):
            tables[s, :owned[s]] = perm[at:at + owned[s]]
            at += owned[s]
        need = int(np.maximum(-(-(ctx + new) // BLOCK) - owned, 0)[~end].sum())
        free = nb - n_owned
        if case["tight"]:
            free = min(free, need * 7 // 8)
        head = int(rng.integers(0, nb))
        ring = np.zeros(nb, dtype=np.int32)
        ring[(head + np.arange(free)) % nb] = perm[n_owned:n_owned + free]
        x["rows"] = int(new[~end].sum())
        new = np.where(end, -1, new)
        x |= dict(ctx=up(ctx, np.int32), owned=up(owned, np.int32), new=up(new, np.int32), ring=up(ring, np.int32),
                  free=up([head, free], np.int32), tables=up(tables, np.int32), parents=None)
        if case["draft"]:
            x["parents"] = up(_parents(np.maximum(new, 0), rng), np.int32)
        return x

    tables = np.full((b, max_blocks), -1, dtype=np.int32)
    at = 0
    for s, t in enumerate((ctx + new).tolist()):
        n = -(-t // BLOCK)
        tables[s, :n] = perm[at:at + n]
        at += n
    q_start = np.concatenate([[0], np.cumsum(new)])
    if case["fp8"]:  # per-head scales of an amax near 4.5 standard deviations
        x["ks"], x["vs"] = ((4.5 + torch.rand(hkv, generator=g, device=dev)) / E4M3_MAX for _ in range(2))

    def normal(*shape):
        return torch.randn(shape, generator=g, device=dev, dtype=torch.bfloat16)

    def cache(*shape):
        if not case["fp8"]:
            return normal(*shape)
        t = torch.empty(shape, dtype=torch.uint8, device=dev)
        for i in range(0, nb, 8192):  # unit-variance values over a scale of 1 / 93, saturating
            part = torch.randn((min(8192, nb - i),) + shape[1:], generator=g, device=dev) * 93.0
            t[i:i + 8192] = part.clamp_(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn).view(torch.uint8)
        return t

    x["k"] = [cache(nb, hkv, BLOCK, DIM) for _ in range(case["layers"])]
    x["v"] = [cache(nb, hkv, DIM, BLOCK) for _ in range(case["layers"])]
    seq = np.repeat(np.arange(b), new)
    pos = ctx[seq] + np.arange(len(seq)) - q_start[seq]
    if case["kind"] == "rope":
        pad = case["pad"]
        slots = tables[seq, pos // BLOCK].astype(np.int64) * BLOCK + pos % BLOCK
        if case["draft"]:  # a drafted token's position is its depth's
            par = _parents(new, rng)
            depth = np.zeros(len(par), dtype=np.int64)
            for i, p in enumerate(par.tolist()):
                if p >= 0:
                    depth[i] = depth[q_start[seq[i]] + p] + 1
            pos = ctx[seq] + depth
        x["slots"] = up(np.concatenate([slots, np.full(pad, -1)]), np.int64)
        x["pos"] = up(np.concatenate([pos, np.full(pad, -1)]), np.int32)
        rows = len(pos) + pad
        if case["fused"]:
            qkv = normal(rows, (hq + 2 * hkv) * DIM)
            x["q"], x["k_new"], x["v_new"] = (t.view(rows, -1, DIM) for t in
                                              qkv.split([hq * DIM, hkv * DIM, hkv * DIM], dim=1))
        else:
            x["q"], x["k_new"], x["v_new"] = normal(rows, hq, DIM), normal(rows, hkv, DIM), normal(rows, hkv, DIM)
        half = case["rotary"] // 2
        turn = torch.arange(case["c_max"], device=dev, dtype=torch.float64)[:, None] \
            * 500000.0 ** (-torch.arange(half, device=dev, dtype=torch.float64) / half)
        x["cos_sin"] = torch.cat([turn.cos(), turn.sin()], dim=1).float()
        x["qw"] = x["kw"] = None
        if case["norm"]:
            x["qw"], x["kw"] = (1 + 0.2 * normal(DIM) for _ in range(2))
        return x

    x |= dict(tables=up(tables, np.int32), ctx=up(ctx + new, np.int32), q_start=up(q_start, np.int32),
              max_ctx=int((ctx + new).max()), max_new=int(new.max()))
    if case["kind"] == "tree":
        x["q"] = normal(len(seq), hq, DIM)
        x["mask"] = up(_masks(_parents(new, rng), new, words(case)), np.int64)
    else:
        paths = _paths(case)
        most = max(len(p) for p, _ in paths)
        acc = np.full((b, most), -1, dtype=np.int32)
        for s, (p, _) in enumerate(paths):
            acc[s, :len(p)] = p
        x["accepted"], x["n_accepted"] = up(acc, np.int32), up([len(p) for p, _ in paths], np.int32)
    return x


def prepare(case, seed):
    x = _inputs(case, seed)
    x["case"] = case
    if not own:
        return x
    from paper_2604_08075_amd import binding
    b, hq, hkv, nb, rows = case["batch"], case["hq"], case["hkv"], x["nb"], x["rows"]
    max_blocks = -(-case["c_max"] // BLOCK)
    empty = lambda *s, dtype=torch.int32: torch.empty(s, dtype=dtype, device="cuda")  # noqa: E731
    if case["kind"] == "tables":
        x["shape"] = binding.tables_shape(b, max_blocks, nb, rows, mask_words=words(case))
        x |= dict(ctx_out=empty(b), owned_out=empty(b), free_out=empty(2), q_start=empty(b + 1), pos=empty(rows),
                  slots=empty(rows, dtype=torch.int64), granted=empty(b), mask=None)
        if case["draft"]:
            x["mask"] = empty(rows, words(case), dtype=torch.int64)
    elif case["kind"] == "rope":
        x["shape"] = binding.qk_shape(rows + case["pad"], hq, hkv, nb, case["c_max"], rotary_dim=case["rotary"],
                                      interleaved=case["paired"], kv_fp8=case["fp8"], q_stride=x["q"].stride(0),
                                      k_stride=x["k_new"].stride(0), v_stride=x["v_new"].stride(0))
        x["q_out"] = torch.zeros((rows + case["pad"], hq, DIM), dtype=torch.bfloat16, device="cuda")
    elif case["kind"] == "tree":
        x["decoder"] = binding.TreeDecoder(b, hq, hkv, max_blocks, case["c_max"], nb, rows, mask_words=words(case),
                                           kv_fp8=case["fp8"])
        x["out"] = x["decoder"].new_out()
    else:
        x["shape"] = binding.tree_shape(b, hq, hkv, max_blocks, case["c_max"], nb, rows, kv_fp8=case["fp8"])
        x["layers"] = binding.CacheLayers(x["k"], x["v"])
        x["ctx_out"] = empty(b)
    return x


def _values(case, t):
    """What a cache tensor stands for, in its own type."""
    return t.view(torch.float8_e4m3fn) if case["fp8"] else t


def run(x):
    case = x["case"]
    if own:
        return _run_own(x, case)
    return {"tables": _tables, "rope": _rope, "tree": _tree, "accept": _accept}[case["kind"]](x, case)


def _run_own(x, case):
    from paper_2604_08075_amd import binding
    kind = case["kind"]
    if kind == "tables":
        binding.kv_tables_step(x["ctx"], x["owned"], x["new"], x["ring"], x["free"], x["tables"], x["ctx_out"],
                               x["owned_out"], x["free_out"], x["q_start"], x["slots"], x["pos"], x["granted"],
                               x["shape"], x["parents"], x["mask"])
        outs = [x["tables"], x["ctx_out"], x["owned_out"], x["ring"], x["free_out"], x["q_start"], x["slots"],
                x["pos"], x["granted"]]
        return outs + [x["mask"]] if case["draft"] else outs
    if kind == "rope":
        binding.qk_norm_rope_append(x["q"], x["k_new"], x["v_new"], x["cos_sin"], x["pos"], x["slots"], x["q_out"],
                                    x["k"][0], x["v"][0], x["shape"], x["qw"], x["kw"], EPS, x["ks"], x["vs"])
        return [x["q_out"][:x["rows"]], _values(case, x["k"][0]), _values(case, x["v"][0])]
    if kind == "tree":
        return x["decoder"](x["q"], x["k"][0], x["v"][0], x["tables"], x["ctx"], x["q_start"], x["mask"], SCALE,
                            x["out"], x["ks"], x["vs"])
    binding.kv_cache_accept(x["layers"], x["tables"], x["ctx"], x["q_start"], x["accepted"], x["n_accepted"],
                            x["ctx_out"], x["shape"])
    return [x["ctx_out"]] + [_values(case, t) for t in x["k"] + x["v"]]


# ------------------------------------------------------------------ plain forms

def _tables(x, case):
    ctx, have, new = x["ctx"].long(), x["owned"].long(), x["new"].long()
    ring, nb, rows = x["ring"], x["nb"], x["rows"]
    dev, (b, max_blocks) = ctx.device, x["tables"].shape
    over, n = new < 0, new.clamp(min=0)
    fits = ctx + n <= max_blocks * BLOCK
    need = torch.where(fits & ~over, ((ctx + n + BLOCK - 1) // BLOCK - have).clamp(min=0), 0)
    upto = need.cumsum(0)
    head, free = x["free"].long()
    granted = fits & ((need == 0) | (upto <= free))
    took = torch.where(granted, need, 0)
    gave = torch.where(over, have, 0)
    # entries of the new blocks; released ids behind the free ones
    j = torch.arange(max_blocks, device=dev)[None, :]
    fresh = (j >= have[:, None]) & (j < (have + took)[:, None])
    at = (head + (upto - need - have)[:, None] + j) % nb
    tables = torch.where(fresh, ring[at], x["tables"])
    back = over[:, None] & (j < have[:, None])
    at = (head + free + (gave.cumsum(0) - gave)[:, None] + j) % nb
    ring_out = torch.cat([ring, ring[:1]]).scatter(0, torch.where(back, at, nb).flatten(), x["tables"].flatten())[:nb]
    # rows
    ends = n.cumsum(0)
    r = torch.arange(rows, device=dev)
    s = torch.searchsorted(ends, r, right=True)
    i = r - (ends - n)[s]
    t = ctx[s] + i
    ok = granted[s]
    block = tables[s, (t // BLOCK).clamp(max=max_blocks - 1)].long()
    slots = torch.where(ok, block * BLOCK + t % BLOCK, -1)
    q_start = torch.cat([ends.new_zeros(1), ends])
    outs = [tables, torch.where(over, 0, torch.where(granted, ctx + n, ctx)), torch.where(over, 0, have + took),
            ring_out, torch.stack([(head + took.sum()) % nb, free - took.sum() + gave.sum()]), q_start]
    if not case["draft"]:
        return [o.int() for o in outs] + [slots, t.int(), granted.int()]
    # ancestors by pointer doubling: `up` is the 2^k-th ancestor's row, or the row behind the last
    par = x["parents"].long()
    up = torch.cat([torch.where(par >= 0, r - i + par, rows), r.new_full((1,), rows)])
    bit = torch.arange(64 * words(case), device=dev)
    seen = torch.cat([i[:, None] == bit, torch.zeros((1, len(bit)), dtype=torch.bool, device=dev)])
    depth = (up < rows).long()
    for _ in range(max(1, (case["draft"] - 1).bit_length())):
        seen = seen | seen[up]
        depth = depth + depth[up]
        up = up[up]
    mask = (seen[:rows].view(rows, -1, 64).long() << torch.arange(64, device=dev)).sum(-1)
    return [o.int() for o in outs] + [slots, (ctx[s] + depth[:rows]).int(), granted.int(), mask]


def _turned(case, t, weight, cs, double=False):
    """Norm and rotation of [rows, heads, DIM], in 32 (or 64) bits."""
    t = t.double() if double else t.float()
    if weight is not None:
        t = t * torch.rsqrt(t.square().mean(-1, keepdim=True) + EPS) * weight.to(t.dtype)
    rot = case["rotary"]
    cos, sin = cs.to(t.dtype)[:, None, :].chunk(2, dim=-1)
    a, b = (t[..., 0:rot:2], t[..., 1:rot:2]) if case["paired"] else t[..., :rot].chunk(2, dim=-1)
    y = [a * cos - b * sin, b * cos + a * sin]
    y = torch.stack(y, dim=-1).flatten(-2) if case["paired"] else torch.cat(y, dim=-1)
    return torch.cat([y, t[..., rot:]], dim=-1)


def _encode(case, t, scale):
    """[rows, hkv, DIM] in the cache's type."""
    if not case["fp8"]:
        return t.to(torch.bfloat16)
    t = (t.float() / scale[:, None]).clamp(-E4M3_MAX, E4M3_MAX)
    return t.to(torch.float8_e4m3fn).view(torch.uint8)


def _rope(x, case):
    n = x["rows"]
    cs = x["cos_sin"][x["pos"][:n].long()]
    blk, off = x["slots"][:n] // BLOCK, x["slots"][:n] % BLOCK
    q = _turned(case, x["q"][:n], x["qw"], cs).to(torch.bfloat16)
    k = _turned(case, x["k_new"][:n], x["kw"], cs)
    x["k"][0][blk, :, off] = _encode(case, k, x["ks"])
    x["v"][0][blk, :, :, off] = _encode(case, x["v_new"][:n], x["vs"])
    return [q, _values(case, x["k"][0]), _values(case, x["v"][0])]


def _tree(x, case):
    hq, hkv, dev = case["hq"], case["hkv"], x["q"].device
    group, b, t_max, n_max = hq // hkv, case["batch"], x["max_ctx"], x["max_new"]
    ids = x["tables"][:, :-(-t_max // BLOCK)].clamp(min=0).long()
    k, v = _values(case, x["k"][0])[ids].float(), _values(case, x["v"][0])[ids].float()
    k = k.permute(0, 2, 1, 3, 4).reshape(b * hkv, -1, DIM)[:, :t_max]
    v = v.permute(0, 2, 1, 4, 3).reshape(b * hkv, -1, DIM)[:, :t_max]
    if case["fp8"]:
        k, v = k * x["ks"].repeat(b)[:, None, None], v * x["vs"].repeat(b)[:, None, None]
    # the drafted rows, padded to the longest tree
    start, n = x["q_start"][:-1].long(), x["q_start"].diff().long()
    i = torch.arange(n_max, device=dev)
    row = (start[:, None] + i).clamp(max=x["q"].shape[0] - 1)
    q = x["q"][row].float().view(b, n_max, hkv, group, DIM).permute(0, 2, 1, 3, 4).reshape(b * hkv, -1, DIM) * SCALE
    # token t is drafted token t - (T - n)
    t = torch.arange(t_max, device=dev)
    j = t[None, :] - (x["ctx"].long() - n)[:, None]
    bits = x["mask"][row].gather(2, (j // 64).clamp(0, words(case) - 1)[:, None].expand(b, n_max, t_max))
    see = (j < 0)[:, None] | (((bits >> (j % 64)[:, None]) & 1) == 1) & (j < n[:, None])[:, None]
    z = q @ k.transpose(1, 2).contiguous()
    z = z.view(b, hkv, n_max, group, t_max).masked_fill_(~see[:, None, :, None], -math.inf)
    z = z.sub_(z.amax(-1, keepdim=True)).exp_()
    z = z.div_(z.sum(-1, keepdim=True)).view(b * hkv, -1, t_max)
    o = (z @ v).view(b, hkv, n_max, group, DIM).permute(0, 2, 1, 3, 4).reshape(b, n_max, hq, DIM)
    return o[i[None, :] < n[:, None]].to(torch.bfloat16)


def _accept(x, case):
    n = x["q_start"].diff()
    base = (x["ctx"] - n).long()
    j = torch.arange(x["accepted"].shape[1], device=base.device)
    s = (j[None, :] < x["n_accepted"][:, None]).nonzero()[:, 0]
    j = (j[None, :] < x["n_accepted"][:, None]).nonzero()[:, 1]
    src, dst = base[s] + x["accepted"][s, j], base[s] + j
    sb, db = x["tables"][s, src // BLOCK].long(), x["tables"][s, dst // BLOCK].long()
    for k, v in zip(x["k"], x["v"]):
        k[db, :, dst % BLOCK] = k[sb, :, src % BLOCK]
        v[db, :, :, dst % BLOCK] = v[sb, :, :, src % BLOCK]
    return [(base + x["n_accepted"]).int()] + [_values(case, t) for t in x["k"] + x["v"]]


# ------------------------------------------------------------------ from the definitions, in 64 bits

def exact(case, seed):
    x = _inputs(case, seed)
    return {"tables": _exact_tables, "rope": _exact_rope, "tree": _exact_tree, "accept": _exact_accept}[
        case["kind"]](x, case)


def _exact_tables(x, case):
    """One request after the other, as a scheduler on the host would."""
    ctx, have, new, ring, tables = (x[n].cpu().numpy().astype(np.int64) for n in ("ctx", "owned", "new", "ring",
                                                                                "tables"))
    nb, (head, free) = x["nb"], x["free"].tolist()
    left, tail, first = free, free, head
    q_start, slots, pos, granted, masks = [0], [], [], [], []
    for s in range(case["batch"]):
        if new[s] < 0:
            ring[(head + tail + np.arange(have[s])) % nb] = tables[s, :have[s]]
            tail += have[s]
            ctx[s] = have[s] = 0
            granted.append(1)
            q_start.append(q_start[-1])
            continue
        want = ctx[s] + new[s]
        need = max(0, -(-want // BLOCK) - have[s]) if want <= tables.shape[1] * BLOCK else 0
        ok = want <= tables.shape[1] * BLOCK and (need == 0 or need <= left)
        if need > 0:  # the first that does not fit closes the line
            left = left - need if ok else -1
        if ok:
            tables[s, have[s]:have[s] + need] = ring[(first + np.arange(need)) % nb]
            first, have[s] = first + need, have[s] + need
        t = ctx[s] + np.arange(new[s])
        slots.append(tables[s, t // BLOCK] * BLOCK + t % BLOCK if ok else np.full(new[s], -1))
        if case["draft"]:
            par = x["parents"][q_start[-1]:q_start[-1] + new[s]].cpu().numpy()
            masks.append(_masks(par, new[s:s + 1], words(case)))
            t = ctx[s] + np.array([sum(bin(w & (2 ** 64 - 1)).count("1") for w in m) for m in masks[-1].tolist()]) - 1
        pos.append(t)
        q_start.append(q_start[-1] + new[s])
        granted.append(int(ok))
        ctx[s] = want if ok else ctx[s]
    outs = [tables, ctx, have, ring, np.array([first % nb, tail - (first - head)]), np.array(q_start)]
    outs = [o.astype(np.int32) for o in outs] + [np.concatenate(slots).astype(np.int64),
                                                 np.concatenate(pos).astype(np.int32), np.array(granted, np.int32)]
    return outs + [np.concatenate(masks)] if case["draft"] else outs


def _exact_cache(case, t):
    return t.view(torch.float8_e4m3fn).double() if case["fp8"] else t.double()


def _exact_rope(x, case):
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
    blk, off = x["slots"][:n] // BLOCK, x["slots"][:n] % BLOCK
    k, v = _exact_cache(case, x["k"][0]), _exact_cache(case, x["v"][0])
    new = [outs[1], x["v_new"][:n].double()]
    if case["fp8"]:
        new = [(t / s.double()[:, None]).clamp(-E4M3_MAX, E4M3_MAX) for t, s in zip(new, (x["ks"], x["vs"]))]
    k[blk, :, off], v[blk, :, :, off] = new
    return [outs[0], k, v]


def _exact_tree(x, case):
    hq, hkv = case["hq"], case["hkv"]
    group = hq // hkv
    out = torch.empty(x["q"].shape, dtype=torch.float64, device=x["q"].device)
    q_start, mask = x["q_start"].tolist(), x["mask"].cpu().numpy().view(np.uint64)
    for s, t in enumerate(x["ctx"].tolist()):
        r0, r1 = q_start[s], q_start[s + 1]
        n = r1 - r0
        ids = x["tables"][s, :-(-t // BLOCK)].long()
        k, v = _exact_cache(case, x["k"][0][ids]), _exact_cache(case, x["v"][0][ids])
        if case["fp8"]:
            k, v = k * x["ks"].double()[:, None, None], v * x["vs"].double()[:, None, None]
        k = k.permute(1, 0, 2, 3).reshape(hkv, -1, DIM)[:, :t]
        v = v.permute(1, 0, 3, 2).reshape(hkv, -1, DIM)[:, :t]
        tree = np.array([[(int(mask[r, c // 64]) >> (c % 64)) & 1 for c in range(n)] for r in range(r0, r1)], bool)
        hidden = torch.zeros((n, t), dtype=torch.bool, device=k.device)
        hidden[:, t - n:] = torch.from_numpy(~tree).to(k.device)
        for h in range(hq):
            z = (x["q"][r0:r1, h].double() * SCALE) @ k[h // group].t()
            out[r0:r1, h] = torch.softmax(z.masked_fill_(hidden, -math.inf), dim=-1) @ v[h // group]
    return out


def _exact_accept(x, case):
    base = x["ctx"].cpu().numpy().astype(np.int64) - np.diff(x["q_start"].cpu().numpy())
    tables = x["tables"].cpu().numpy()
    sb, so, db, do = [], [], [], []
    for s, (path, _) in enumerate(_paths(case)):
        for j, i in enumerate(path.tolist()):
            sb.append(tables[s, (base[s] + i) // BLOCK])
            so.append((base[s] + i) % BLOCK)
            db.append(tables[s, (base[s] + j) // BLOCK])
            do.append((base[s] + j) % BLOCK)
    sb, so, db, do = (torch.tensor(np.array(a, dtype=np.int64), device="cuda") for a in (sb, so, db, do))
    outs = [base + np.array([len(p) for p, _ in _paths(case)])]
    outs[0] = outs[0].astype(np.int32)
    for t in x["k"]:
        t[db, :, do] = t[sb, :, so]
        outs.append(_exact_cache(case, t))
    for t in x["v"]:
        t[db, :, :, do] = t[sb, :, :, so]
        outs.append(_exact_cache(case, t))
    return outs
