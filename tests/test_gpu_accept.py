"""kv_cache_accept (through the C ABI) against the oracle: codes are moved, so the whole caches must be equal."""
import numpy as np
import pytest
import torch

from oracle import tree

pytestmark = pytest.mark.gpu


def note(msg):
    print(f"[gpu-test] {msg}", flush=True)


def dev(a):
    a = np.ascontiguousarray(a)
    return torch.from_numpy(a.view(np.int16) if a.dtype == np.uint16 else a).cuda()


def check(lib, rng, chunks, hkv, fmt, layers, paths, n_accepted=None, holes=False):
    note(f"accept {fmt} heads={hkv} layers={layers} chunks={chunks[:5]}")
    B = len(chunks)
    mb = max(-(-t // 16) for _, t in chunks) + 1
    nb = B * mb + 5
    bt = rng.permutation(nb)[:B * mb].reshape(B, mb).astype(np.int32)
    if holes:
        bt[0, 0], bt[B - 1, :] = -1, nb + 3
    qs = np.concatenate([[0], np.cumsum([n for n, _ in chunks])]).astype(np.int32)
    ctx = np.array([t for _, t in chunks], np.int32)
    most = max(max(len(p) for p in paths), 1)
    acc = np.full((B, most), -1, np.int32)
    for s, p in enumerate(paths):
        acc[s, :len(p)] = p
    n_acc = np.array([len(p) for p in paths] if n_accepted is None else n_accepted, np.int32)
    t = np.uint16 if fmt == "bf16" else np.uint8
    ks = [rng.integers(0, np.iinfo(t).max + 1, (nb, hkv, 16, 128)).astype(t) for _ in range(layers)]
    vs = [rng.integers(0, np.iinfo(t).max + 1, (nb, hkv, 128, 16)).astype(t) for _ in range(layers)]
    dk, dv = [dev(x) for x in ks], [dev(x) for x in vs]
    out = dev(np.full(B, -9, np.int32))
    shape = lib.tree_shape(B, hkv, hkv, mb, mb * 16, nb, int(qs[-1]), kv_fp8=fmt != "bf16")
    lib.kv_cache_accept(lib.CacheLayers(dk, dv), dev(bt), dev(ctx), dev(qs), dev(acc), dev(n_acc), out, shape)
    torch.cuda.synchronize()
    for l in range(layers):
        wk, wv, wc = tree.accept(ks[l], vs[l], bt, ctx, qs, acc, n_acc)
        assert np.array_equal(dk[l].cpu().numpy().view(t), wk) and np.array_equal(dv[l].cpu().numpy().view(t), wv)
    assert np.array_equal(out.cpu().numpy(), wc)


def path(rng, n, a):
    return np.sort(rng.choice(n, size=min(a, n), replace=False)).tolist()


FMT = ["bf16", "fp8_e4m3"]


@pytest.mark.parametrize("fmt", FMT)
@pytest.mark.parametrize("hkv,layers", [(1, 1), (2, 3), (8, 2), (3, 5)])
def test_random_paths(gpu_lib, hkv, layers, fmt):
    rng = np.random.default_rng(hkv + layers)
    chunks = [(n, n + int(rng.integers(0, 60))) for n in (1, 2, 5, 9, 16, 17, 40, 64, 0, 33)]
    check(gpu_lib, rng, chunks, hkv, fmt, layers, [path(rng, n, int(rng.integers(0, n + 1))) for n, _ in chunks])


@pytest.mark.parametrize("fmt", FMT)
def test_long_paths(gpu_lib, fmt):
    """Paths longer than a wave's lanes, sources that are targets of later moves, and whole chains."""
    rng = np.random.default_rng(1)
    chunks = [(200, 230), (130, 130), (256, 300), (100, 555)]
    check(gpu_lib, rng, chunks, 2, fmt, 2, [path(rng, 200, 150), list(range(130)), list(range(1, 256)),
                                            path(rng, 100, 64)])


def test_more_layers_than_one_launch_takes(gpu_lib):
    rng = np.random.default_rng(2)
    check(gpu_lib, rng, [(5, 20), (3, 9)], 1, "bf16", 70, [[0, 2, 4], [1]])


def test_broken_paths_are_cut(gpu_lib):
    rng = np.random.default_rng(3)
    chunks = [(8, 30), (8, 30), (8, 30), (8, 30), (8, 30), (70, 90)]
    paths = [[0, 3, 3, 5], [2, 1], [-4, 2], [1, 8, 9], [0, 2, 5, 6], list(range(1, 67)) + [60, 68]]
    check(gpu_lib, rng, chunks, 2, "bf16", 1, paths, n_accepted=[4, 2, 2, 3, 99, 68])
    check(gpu_lib, rng, chunks, 2, "fp8_e4m3", 1, paths, n_accepted=[4, 2, 2, -3, 0, 65])


def test_blocks_outside_the_pool_are_left(gpu_lib):
    rng = np.random.default_rng(4)
    chunks = [(20, 30), (20, 40), (9, 9)]
    check(gpu_lib, rng, chunks, 2, "bf16", 2, [path(rng, 20, 12), path(rng, 20, 12), [3, 5]], holes=True)
