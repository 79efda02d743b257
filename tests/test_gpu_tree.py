"""tree_decode_attention (through the C ABI) against the oracle in float64, within the bound that the oracle derives."""
import numpy as np
import pytest
import torch

import workloads
from oracle import numerics, tree

pytestmark = pytest.mark.gpu


def note(msg):
    print(f"[gpu-test] {msg}", flush=True)


def tree_masks(rng, counts, words, kind):
    """uint64 [sum(counts), words]"""
    rows = []
    for n in counts:
        m = []
        for i in range(n):
            if kind == "chain":
                x = (2 << i) - 1
            elif kind == "tree":
                x = (m[int(rng.integers(i // 3, i))] if i else 0) | 1 << i
            elif kind == "none":
                x = 0
            else:   # any bits, those past the drafts too
                x = int.from_bytes(rng.bytes(8 * words), "little")
            m.append(x)
        rows += [[(x >> (64 * w)) & (2 ** 64 - 1) for w in range(words)] for x in m]
    return np.array(rows, np.uint64).reshape(-1, words)


def call(lib, w, d, mask, words, max_ctx=None, ws=None, q_start=None, total_q=None):
    qs = w.meta["q_start"] if q_start is None else q_start
    total_q = int(qs[-1]) if total_q is None else total_q
    dec = lib.TreeDecoder(w.batch, w.n_q_heads, w.n_kv_heads, w.max_blocks_per_seq, max_ctx or w.c_max, w.num_blocks,
                          total_q, words, w.kv_format == "fp8_e4m3")
    dec.workspace.fill_(255)   # any content will do
    out = torch.full((total_q, w.n_q_heads, 128), float("nan"), dtype=torch.bfloat16, device="cuda")
    dm = torch.from_numpy(mask.view(np.int64)).cuda()
    dq = torch.from_numpy(np.asarray(qs, np.int32)).cuda()
    args = (d["q"], d["k"][0], d["v"][0], d["block_tables"], d["context_lens"], dq, dm, w.scale)
    dec(*args, out, d["k_scale"], d["v_scale"])
    again = torch.full_like(out, float("nan"))
    dec(*args, again, d["k_scale"], d["v_scale"])
    torch.cuda.synchronize()
    assert torch.equal(out.view(torch.int16), again.view(torch.int16))
    return out.float().cpu().numpy()


def check(lib, chunks, hq, hkv, fmt, words, kind, seed, c_max=None, max_ctx=None):
    c_max = c_max or max(max(t for _, t in chunks), 1)
    note(f"tree {fmt} heads={hq}/{hkv} words={words} {kind} chunks={chunks[:6]}")
    rng = np.random.default_rng(seed)
    w = workloads.make_prefill(chunks, hq, hkv, c_max=c_max, kv_format=fmt, seed=seed)
    mask = tree_masks(rng, [n for n, _ in chunks], words, kind)
    got = call(lib, w, workloads.to_device(w), mask, words, max_ctx)
    ref, bound = tree.tree_attention(w.q_bits, w.k_store.dense(), w.v_store.dense(), w.block_tables, w.context_lens,
                                     w.meta["q_start"], mask, w.scale, fmt, w.k_scale, w.v_scale)
    assert np.isfinite(got).all()
    ratio = np.abs(got - ref) / bound
    note(f"  largest error {np.abs(got - ref).max():.2e}, {ratio.max():.2f} of its bound")
    assert ratio.max() <= 1.0


FMT = ["bf16", "fp8_e4m3"]


@pytest.mark.parametrize("fmt", FMT)
@pytest.mark.parametrize("T", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 129, 200, 513])
def test_lengths(gpu_lib, T, fmt):
    check(gpu_lib, [(min(n, T), T) for n in (1, 3, 8)], 8, 2, fmt, 1, "tree", T)


@pytest.mark.parametrize("fmt", FMT)
@pytest.mark.parametrize("hq,hkv", [(1, 1), (4, 4), (3, 1), (10, 2), (16, 2), (14, 2), (32, 2), (64, 1), (70, 1)])
def test_head_groups(gpu_lib, hq, hkv, fmt):
    check(gpu_lib, [(1, 90), (5, 33), (7, 7), (0, 12), (4, 0 + 4)], hq, hkv, fmt, 1, "tree", hq)


@pytest.mark.parametrize("fmt", FMT)
@pytest.mark.parametrize("n", [2, 4, 6, 8, 9, 16, 17, 31, 32, 33, 50, 64])
def test_tree_sizes(gpu_lib, n, fmt):
    check(gpu_lib, [(n, 150), (n // 2, 77), (n, n)], 8, 1, fmt, 1, "tree", n)


@pytest.mark.parametrize("fmt", FMT)
@pytest.mark.parametrize("words,n", [(2, 65), (2, 128), (3, 190), (4, 256), (4, 10), (3, 1)])
def test_mask_words(gpu_lib, words, n, fmt):
    check(gpu_lib, [(n, n + 60), (n, n), (1, 40)], 2, 1, fmt, words, "tree", n)


@pytest.mark.parametrize("fmt", FMT)
@pytest.mark.parametrize("kind", ["chain", "none", "any"])
def test_mask_kinds(gpu_lib, kind, fmt):
    check(gpu_lib, [(9, 64), (9, 9), (1, 1), (40, 71), (64, 64), (33, 100)], 8, 2, fmt, 1, kind, 3)
    check(gpu_lib, [(70, 90), (128, 128), (100, 333)], 4, 2, fmt, 2, kind, 4)


@pytest.mark.parametrize("fmt", FMT)
@pytest.mark.parametrize("chunks,hq,hkv", [
    ([(6, 9000)], 8, 1),                                       # one long sequence: split over the device
    ([(3, 5000), (1, 17), (8, 2600), (2, 2)], 16, 2),
    ([(16, 3000), (16, 100), (5, 1400)], 16, 1),               # 256 columns
    ([(40, 2100), (33, 40), (1, 900)], 16, 1),                 # more columns than one tile holds
    ([(2, 300)] * 40, 16, 4), ([(1, 64)] * 300, 2, 2), ([(12, 700)] * 20, 16, 2)])
def test_long_and_many(gpu_lib, chunks, hq, hkv, fmt):
    check(gpu_lib, chunks, hq, hkv, fmt, 1, "tree", len(chunks), c_max=9100)


@pytest.mark.parametrize("fmt", FMT)
def test_short_limit(gpu_lib, fmt):
    """The same small batch under the limits of a short and of a long pool."""
    for c_max in (64, 512, 1024, 65536):
        check(gpu_lib, [(4, 60), (1, 9), (6, 33)], 8, 2, fmt, 1, "tree", 8, c_max=c_max)


@pytest.mark.parametrize("fmt", FMT)
@pytest.mark.parametrize("seed", range(12))
def test_random_shapes(gpu_lib, seed, fmt):
    rng = np.random.default_rng(100 + seed)
    hkv = int(rng.choice([1, 2, 3, 4]))
    g = int(rng.choice([1, 2, 4, 5, 8, 12, 16]))
    words = int(rng.integers(1, 3))
    chunks = []
    for _ in range(int(rng.integers(1, 9))):
        t = int(np.exp(rng.uniform(0, np.log(1200))))
        chunks.append((min(t, int(rng.integers(0, 2 + 20 * words))), t))
    if sum(n for n, _ in chunks) == 0:
        chunks[0] = (1, max(chunks[0][1], 1))
    check(gpu_lib, chunks, hkv * g, hkv, fmt, words, str(rng.choice(["tree", "any", "chain"])), seed)


@pytest.mark.parametrize("fmt", FMT)
def test_values_that_are_not_finite(gpu_lib, fmt):
    """NaN and infinities in drafts: rows that do not see them keep their bits, rows that do follow the formula."""
    note(f"tree, values that are not finite, {fmt}")
    chunks = [(6, 40), (33, 150), (5, 5)]
    w = workloads.make_prefill(chunks, 8, 2, c_max=160, kv_format=fmt, seed=21)
    rng = np.random.default_rng(21)
    mask = tree_masks(rng, [n for n, _ in chunks], 1, "tree")
    d = workloads.to_device(w)
    clean = call(gpu_lib, w, d, mask, 1)
    K, V = w.k_store.dense().copy(), w.v_store.dense().copy()
    nan, inf = (0x7FC0, 0x7F80) if fmt == "bf16" else (0x7F, 0xFF)
    hit = []
    for s, j, what, dims, code in ((0, 2, "v", slice(None), nan), (1, 5, "v", slice(3, 4), inf), (1, 20, "k", 9, nan),
                                   (2, 4, "v", slice(100, 128), nan), (1, 5, "v", slice(77, 78), nan)):
        n, T = chunks[s]
        t = T - n + j
        b = w.block_tables[s][t // 16]
        if what == "v":
            V[b, 1, dims, t % 16] = code
        else:
            K[b, 1, t % 16, dims] = code
        hit.append((s, j))
    conv = (lambda x: torch.from_numpy(x.view(np.int16))) if fmt == "bf16" else torch.from_numpy
    d["k"], d["v"] = conv(K)[None].cuda(), conv(V)[None].cuda()
    got = call(gpu_lib, w, d, mask, 1)
    qs = w.meta["q_start"]
    ref, bound = tree.tree_attention(w.q_bits, K, V, w.block_tables, w.context_lens, qs, mask, w.scale, fmt, w.k_scale,
                                     w.v_scale)
    touched = np.zeros(got.shape[0], bool)
    for s, j in hit:
        see = tree.bits(mask[qs[s]:qs[s + 1]], chunks[s][0])[:, j]
        touched[qs[s]:qs[s + 1]] |= see
    assert 0 < touched.sum() < len(touched)
    assert np.array_equal(got[~touched], clean[~touched])
    assert np.array_equal(got[:, :4], clean[:, :4])       # KV head 0 holds no such value
    a, b = got[touched][:, 4:], ref[touched][:, 4:]
    assert np.array_equal(np.isfinite(a), np.isfinite(b))
    if fmt == "bf16":   # (an infinity times a probability is that infinity, unless a NaN joins)
        assert np.array_equal(np.isnan(a), np.isnan(b))
    ok = np.isfinite(b)
    assert (np.abs(a[ok] - b[ok]) <= bound[touched][:, 4:][ok]).all()


def test_rows_and_sequences_outside_the_promises(gpu_lib):
    """Clamped lengths: nothing outside the buffers is written, rows past a sequence's drafts stay as they were."""
    note("tree, values out of range")
    chunks = [(5, 40), (8, 30), (4, 70)]
    w = workloads.make_prefill(chunks, 4, 2, c_max=80, seed=31)
    d = workloads.to_device(w)
    mask = tree_masks(np.random.default_rng(0), [n for n, _ in chunks], 1, "chain")
    good = call(gpu_lib, w, d, mask, 1)
    # padded: rows behind the last sequence
    d2 = dict(d, q=torch.cat([d["q"], d["q"][:3]]))
    padded = call(gpu_lib, w, d2, np.concatenate([mask, mask[:3]]), 1, q_start=w.meta["q_start"], total_q=20)
    assert np.array_equal(padded[:17], good) and np.isnan(padded[17:]).all()
    # a sequence with more rows than tokens (8 rows, 6 tokens), and one past the limit of the shape
    d3 = dict(d, context_lens=torch.tensor([40, 6, 10 ** 9], dtype=torch.int32, device="cuda"))
    got = call(gpu_lib, w, d3, mask, 1)
    assert np.array_equal(got[:5], good[:5]) and np.isfinite(got[5:11]).all() and np.isnan(got[11:13]).all()
    # row offsets out of order and out of range
    # (clamped, the last sequence's range is all seventeen rows, the first one's too)
    got = call(gpu_lib, w, d, mask, 1, q_start=[0, 5, -3, 10 ** 9], total_q=17)
    assert np.isfinite(got).all()
    # block ids outside the pool are clamped
    bad = d["block_tables"].clone()
    bad[1, 0], bad[1, 1] = -1, 2 ** 31 - 1
    got = call(gpu_lib, w, dict(d, block_tables=bad), mask, 1)
    assert np.array_equal(got[:5], good[:5]) and np.array_equal(got[13:], good[13:])


def test_large_block_indices(gpu_lib):
    """Offsets past 32 bits: blocks at the far end of a cache of more than 4 GiB."""
    note("tree, far blocks")
    chunks = [(4, 100), (2, 37)]
    w = workloads.make_prefill(chunks, 4, 2, c_max=128, seed=41)
    mask = tree_masks(np.random.default_rng(1), [4, 2], 1, "tree")
    d = workloads.to_device(w)
    near = call(gpu_lib, w, d, mask, 1)
    far = 600000                       # 600,000 blocks of 8 KiB: 4.9 GB each for K and V
    nb = w.num_blocks
    big = {}
    for name in ("k", "v"):
        big[name] = torch.empty((1, far + nb) + tuple(d[name].shape[2:]), dtype=torch.int16, device="cuda")
        big[name][0, far:] = d[name][0]
    w.num_blocks = far + nb
    bt = torch.where(d["block_tables"] >= 0, d["block_tables"] + far, -1)
    got = call(gpu_lib, w, dict(d, block_tables=bt, **big), mask, 1)
    assert np.array_equal(got, near)


def test_key_scale_of_zero(gpu_lib):
    note("tree, e4m3 with a key scale of 0")
    chunks = [(3, 50), (4, 4)]
    w = workloads.make_prefill(chunks, 4, 2, c_max=64, kv_format="fp8_e4m3", seed=51)
    w.k_scale = w.k_scale * np.float32([0, 1])
    mask = tree_masks(np.random.default_rng(2), [3, 4], 1, "tree")
    mask[4] = 0
    got = call(gpu_lib, w, workloads.to_device(w), mask, 1)
    ref, bound = tree.tree_attention(w.q_bits, w.k_store.dense(), w.v_store.dense(), w.block_tables, w.context_lens,
                                     w.meta["q_start"], mask, w.scale, "fp8_e4m3", w.k_scale, w.v_scale)
    assert (np.abs(got - ref) <= bound).all()


@pytest.mark.parametrize("fmt", FMT)
@pytest.mark.parametrize("T,n,t", [(70, 3, 66), (70, 3, 64), (70, 3, 2), (40, 8, 31), (33, 1, 0), (2500, 4, 2495), (2500, 4, 700)])
def test_committed_values_that_are_not_finite(gpu_lib, T, n, t, fmt):
    """A committed token's V that is not finite reaches every row, wherever it lies beside the drafts."""
    note(f"tree, committed token {t} of {T} not finite, {fmt}")
    w = workloads.make_prefill([(n, T), (n, T)], 4, 2, c_max=T, kv_format=fmt, seed=61)
    mask = tree_masks(np.random.default_rng(3), [n, n], 1, "tree")
    d = workloads.to_device(w)
    clean = call(gpu_lib, w, d, mask, 1)
    V = w.v_store.dense().copy()
    V[w.block_tables[1][t // 16], 0, 5:7, t % 16] = 0x7FC0 if fmt == "bf16" else 0x7F
    d["v"] = (torch.from_numpy(V.view(np.int16)) if fmt == "bf16" else torch.from_numpy(V))[None].cuda()
    got = call(gpu_lib, w, d, mask, 1)
    hit = np.zeros(got.shape, bool)
    hit[n:, :2, 5:7] = True
    assert np.isnan(got[hit]).all() and np.array_equal(got[~hit], clean[~hit])


def test_key_scale_below_zero(gpu_lib):
    """The formula holds for any scale: hidden tokens stay hidden under a negative one."""
    note("tree, e4m3 with key scales below 0")
    chunks = [(3, 50), (4, 4), (9, 700)]
    w = workloads.make_prefill(chunks, 4, 2, c_max=704, kv_format="fp8_e4m3", seed=52)
    w.k_scale = w.k_scale * np.float32([-1, -0.5])
    w.v_scale = w.v_scale * np.float32([1, -2])
    mask = tree_masks(np.random.default_rng(2), [3, 4, 9], 1, "tree")
    mask[4] = 0
    got = call(gpu_lib, w, workloads.to_device(w), mask, 1)
    ref, bound = tree.tree_attention(w.q_bits, w.k_store.dense(), w.v_store.dense(), w.block_tables, w.context_lens,
                                     w.meta["q_start"], mask, w.scale, "fp8_e4m3", w.k_scale, w.v_scale)
    assert (np.abs(got - ref) <= bound).all()


@pytest.mark.parametrize("fmt", FMT)
@pytest.mark.parametrize("B", [7, 300, 1200])
def test_row_offsets_out_of_order(gpu_lib, B, fmt):
    """Offsets below one before them count as the largest so far: the same bits as with those, and no row has two owners."""
    note(f"tree, row offsets out of order, B={B} {fmt}")
    rng = np.random.default_rng(B)
    chunks = [(int(rng.integers(0, 4)), int(rng.integers(3, 40))) for _ in range(B)]
    w = workloads.make_prefill(chunks, 2, 1, c_max=48, kv_format=fmt, seed=B)
    qs = np.asarray(w.meta["q_start"], np.int64)
    total = int(qs[-1])
    bad = qs.copy()
    at = rng.choice(B - 1, 3 + B // 50, replace=False) + 1
    bad[at] = rng.integers(-5, total + 1, len(at))
    bad[B // 2], bad[0] = -2 ** 31, min(2, total)
    bad[B - 1] = 2 ** 31 - 1 if B > 500 else bad[B - 1]
    ordered = np.minimum(np.maximum.accumulate(np.maximum(bad, 0)), total)
    assert (np.diff(bad) < 0).any() and (ordered != qs).any()
    mask = tree_masks(rng, [total], 1, "any")
    d = workloads.to_device(w)
    got = call(gpu_lib, w, d, mask, 1, q_start=bad, total_q=total)
    want = call(gpu_lib, w, d, mask, 1, q_start=ordered, total_q=total)
    assert np.array_equal(got, want, equal_nan=True)
    n = np.diff(ordered)
    # (at most as many rows as a sequence has tokens)
    assert np.isfinite(want).any() and np.isnan(want).all((1, 2)).sum() == total - np.minimum(n, [t for _, t in chunks]).sum()


@pytest.mark.parametrize("fmt", FMT)
@pytest.mark.parametrize("T,n", [(40, 3), (70, 9), (5, 5), (2600, 4)])
def test_scores_of_minus_infinity_give_zeros(gpu_lib, T, n, fmt):
    """Rows whose scores are all -infinity are zero, whatever V holds; the other heads keep their bits."""
    note(f"tree, scores of -infinity, T={T} n={n} {fmt}")
    w = workloads.make_prefill([(n, T), (n, T)], 4, 2, c_max=T, kv_format=fmt, seed=71)
    mask = tree_masks(np.random.default_rng(7), [n, n], 1, "tree")
    K, V = w.k_store.dense().copy(), w.v_store.dense().copy()
    one, nan = (0x3F80, 0x7FC0) if fmt == "bf16" else (0x38, 0x7F)
    K[:, 0] = one                          # KV head 0: every key is 1, the first sequence's queries are -infinity
    w.q_bits[:n, :2] = 0xFF80
    conv = (lambda x: torch.from_numpy(x.view(np.int16))) if fmt == "bf16" else torch.from_numpy
    d = workloads.to_device(w)
    d["k"] = conv(K)[None].cuda()
    clean = call(gpu_lib, w, d, mask, 1)
    assert (clean[:n, :2] == 0).all() and np.isfinite(clean).all() and (clean[n:] != 0).any()
    for t in (0, T - n, T - 1):            # committed and drafted
        V[w.block_tables[0][t // 16], 0, 3:5, t % 16] = nan
    if fmt == "bf16":
        V[w.block_tables[0][(T - n) // 16], 0, 9, (T - n) % 16] = 0x7F80
    d["v"] = conv(V)[None].cuda()
    assert np.array_equal(call(gpu_lib, w, d, mask, 1), clean)


def test_key_scale_that_is_not_a_number(gpu_lib):
    """A row that sees no token is zero under any scale; the other rows of that KV head are NaN."""
    note("tree, e4m3 with a key scale of NaN")
    chunks = [(3, 50), (4, 4), (9, 700)]
    w = workloads.make_prefill(chunks, 4, 2, c_max=704, kv_format="fp8_e4m3", seed=53)
    mask = tree_masks(np.random.default_rng(2), [3, 4, 9], 1, "tree")
    mask[4] = 0
    good = call(gpu_lib, w, workloads.to_device(w), mask, 1)
    w.k_scale = w.k_scale * np.float32([np.nan, 1])
    got = call(gpu_lib, w, workloads.to_device(w), mask, 1)
    assert np.array_equal(got[:, 2:], good[:, 2:]) and (good[4] == 0).all()
    assert (got[4, :2] == 0).all() and np.isnan(np.delete(got[:, :2], 4, axis=0)).all()
