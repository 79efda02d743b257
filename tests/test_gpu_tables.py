"""kv_tables_step (through the C ABI) against the oracle: whole numbers, so every output must be equal."""
import numpy as np
import pytest
import torch

from oracle import tables

pytestmark = pytest.mark.gpu


def note(msg):
    print(f"[gpu-test] {msg}", flush=True)


def dev(a, dtype=np.int32):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=dtype)).cuda()


def run(lib, ctx, owned, new, ring, head, count, tb, rows, parents=None, words=0, repeat=1):
    B, mb = tb.shape
    d = dict(ctx=dev(ctx), owned=dev(owned), new=dev(new), ring=dev(ring), st=dev([head, count]), tb=dev(tb))
    e = lambda *s, dtype=torch.int32: torch.full(s, -7, dtype=dtype, device="cuda")  # noqa: E731
    o = dict(ctx=e(B), owned=e(B), state=e(2), q_start=e(B + 1), slots=e(rows, dtype=torch.int64), positions=e(rows),
             granted=e(B))
    mask = e(rows, words, dtype=torch.int64) if words else None
    par = dev(parents) if parents is not None else None
    for _ in range(repeat):
        lib.kv_tables_step(d["ctx"], d["owned"], d["new"], d["ring"], d["st"], d["tb"], o["ctx"], o["owned"],
                           o["state"], o["q_start"], o["slots"], o["positions"], o["granted"],
                           lib.tables_shape(B, mb, len(ring), rows, words), par, mask)
    torch.cuda.synchronize()
    got = {k: v.cpu().numpy() for k, v in dict(o, ring=d["ring"], tables=d["tb"]).items()}
    if words:
        got["mask"] = mask.cpu().numpy().view(np.uint64)
    return got


def same(got, want):
    for k, v in got.items():
        assert np.array_equal(v, want[k]), k


def state(rng, B, mb, free):
    owned = rng.integers(0, mb + 1, B)
    ctx = np.maximum(owned * 16 - rng.integers(0, 40, B), 0)
    nb = int(owned.sum()) + free + 3
    ids = rng.permutation(nb)
    tb = np.full((B, mb), -1)
    at = 0
    for s in range(B):
        tb[s, :owned[s]] = ids[at:at + owned[s]]
        at += owned[s]
    head = int(rng.integers(0, nb))
    ring = np.full(nb, -5)
    ring[(head + np.arange(free)) % nb] = ids[at:at + free]
    return ctx, owned, tb, ring, head


@pytest.mark.parametrize("B,mb,free,most,over", [
    (1, 4, 3, 1, 0), (1, 4, 0, 16, 0), (7, 8, 9, 20, 0.3), (64, 32, 40, 1, 0.1), (65, 16, 10, 33, 0.2),
    (256, 20, 300, 1, 0.05), (257, 20, 3000, 300, 0.1), (1024, 6, 800, 12, 0.1), (4096, 5, 2000, 30, 0.02),
    (9, 600, 4000, 9000, 0.2)])
def test_tables(gpu_lib, B, mb, free, most, over):
    note(f"tables B={B} blocks={mb} free={free} up to {most} tokens")
    rng = np.random.default_rng(B + most)
    ctx, owned, tb, ring, head = state(rng, B, mb, free)
    new = np.where(rng.random(B) < over, -1, rng.integers(0, most + 1, B))
    rows = int(np.maximum(new, 0).sum())
    for total, rep in ((rows, 1), (rows + 13, 2), (max(rows - 5, 0), 1)):  # exact, padded (called twice), cut
        want = tables.step(ctx, owned, new, ring, head, free, tb, total)
        same(run(gpu_lib, ctx, owned, new, ring, head, free, tb, total, repeat=rep), want)


@pytest.mark.parametrize("words", [1, 2, 3, 4])
@pytest.mark.parametrize("B", [1, 5, 130])
def test_tables_trees(gpu_lib, B, words):
    note(f"tables with trees B={B} words={words}")
    rng = np.random.default_rng(10 * B + words)
    mb = 40
    ctx, owned, tb, ring, head = state(rng, B, mb, 300)
    new = rng.integers(-1, 64 * words + 1, B)
    new[B // 2] = 64 * words                   # as large as the masks allow
    if B > 3:
        new[1] = 64 * words + 1                # larger: refused
    rows = int(np.maximum(new, 0).sum())
    par = np.concatenate([rng.integers(-1, np.maximum(np.arange(max(n, 0)), 1), max(n, 0)) for n in new])
    first = np.concatenate([[0], np.cumsum(np.maximum(new, 0))])
    n0 = max(new[B // 2], 0)
    par[first[B // 2]:first[B // 2] + n0] = np.arange(n0) - 1                  # one long chain
    if rows > 4:
        par[rng.integers(0, rows, 3)] = [10 ** 6, -3, 2 ** 31 - 1]             # no earlier token: roots
    want = tables.step(ctx, owned, new, ring, head, 300, tb, rows + 3, np.append(par, [0, 0, 0]), words)
    same(run(gpu_lib, ctx, owned, new, ring, head, 300, tb, rows + 3, np.append(par, [0, 0, 0]), words), want)


def test_tables_broken_promises_stay_inside(gpu_lib):
    """Lengths and counts outside their ranges are clamped; guard words around every buffer stay as they were."""
    note("tables, values out of range")
    B, mb, nb, rows = 5, 4, 16, 30
    guard = 64

    def fenced(a, dtype=torch.int32):
        t = torch.full((len(a) + 2 * guard,), -77, dtype=dtype, device="cuda")
        t[guard:-guard] = torch.tensor(a, dtype=dtype, device="cuda")
        return t, t[guard:-guard]

    ins = [[-5, 2 ** 31 - 1, 63, 20, 7], [-1, 2 ** 31 - 1, 0, 99, 1], [2 ** 31 - 1, 3, 1, -9, 12]]
    bufs = [fenced(x) for x in ins] + [fenced(range(nb)), fenced([2 ** 31 - 1, 2 ** 31 - 1]),
                                       fenced([3] * (B * mb)), fenced([0] * B), fenced([0] * B), fenced([0] * 2),
                                       fenced([0] * (B + 1)), fenced([0] * rows, torch.int64), fenced([0] * rows),
                                       fenced([0] * B)]
    gpu_lib.kv_tables_step(*[v for _, v in bufs], gpu_lib.tables_shape(B, mb, nb, rows))
    torch.cuda.synchronize()
    for full, _ in bufs:
        assert (full[:guard] == -77).all() and (full[-guard:] == -77).all()
    q = bufs[9][1].tolist()
    assert q[0] == 0 and q == sorted(q) and q[-1] <= rows


def test_tables_many_steps_on_the_device(gpu_lib):
    """Sixty steps that keep their state on the device, two buffers in turn, as the oracle has them."""
    note("tables, sixty steps")
    rng = np.random.default_rng(5)
    B, mb, nb, rows = 12, 10, 80, 400
    ctx, owned, tb = np.zeros(B, int), np.zeros(B, int), np.full((B, mb), -1)
    ring, head, count = rng.permutation(nb), 7, nb
    bufs = [dict(ctx=dev(ctx), owned=dev(owned), st=dev([head, count])) for _ in range(2)]
    dring, dtb = dev(ring), dev(tb)
    o = dict(q=dev(np.zeros(B + 1)), slots=dev(np.zeros(rows), np.int64), pos=dev(np.zeros(rows)), ok=dev(np.zeros(B)))
    shape = gpu_lib.tables_shape(B, mb, nb, rows)
    for i in range(60):
        new = rng.integers(-1, 30, B)
        a, b = bufs[i % 2], bufs[1 - i % 2]
        gpu_lib.kv_tables_step(a["ctx"], a["owned"], dev(new), dring, a["st"], dtb, b["ctx"], b["owned"], b["st"],
                               o["q"], o["slots"], o["pos"], o["ok"], shape)
        w = tables.step(ctx, owned, new, ring, head, count, tb, rows)
        ctx, owned, ring, tb = w["ctx"], w["owned"], w["ring"], w["tables"]
        head, count = w["state"].tolist()
        torch.cuda.synchronize()
        assert np.array_equal(b["ctx"].cpu().numpy(), ctx) and np.array_equal(b["owned"].cpu().numpy(), owned)
        assert np.array_equal(dring.cpu().numpy(), ring) and np.array_equal(dtb.cpu().numpy(), tb)
        assert b["st"].tolist() == [head, count] and np.array_equal(o["slots"].cpu().numpy(), w["slots"])


def test_tables_trees_of_a_large_batch(gpu_lib):
    """More sequences than one turn of the scan takes, with trees, refusals and sequences that end."""
    note("tables with trees, 1100 sequences")
    rng = np.random.default_rng(77)
    B, mb = 1100, 6
    ctx, owned, tb, ring, head = state(rng, B, mb, 500)
    new = rng.integers(-1, 20, B)
    new[[3, 600, 1099]] = 65                   # larger than the masks: refused
    rows = int(np.maximum(new, 0).sum())
    par = np.concatenate([rng.integers(-1, np.maximum(np.arange(max(n, 0)), 1), max(n, 0)) for n in new])
    want = tables.step(ctx, owned, new, ring, head, 500, tb, rows, par, 1)
    assert 0 < want["granted"].sum() < B
    same(run(gpu_lib, ctx, owned, new, ring, head, 500, tb, rows, par, 1), want)


@pytest.mark.parametrize("B", [1, 6, 300, 700])
def test_tables_owned_counts_below_the_context(gpu_lib, B):
    """A count of blocks below what the cached tokens take stands for that, also where the sequence ends."""
    note(f"tables, owned counts too small, B={B}")
    rng = np.random.default_rng(B)
    mb, free = 12, 200
    ctx, owned, tb, ring, head = state(rng, B, mb, free)
    ctx[0] = 16 * owned[0]
    said = np.where(rng.random(B) < 0.7, rng.integers(-1, 3, B), owned)
    said[0] = 0
    new = np.where(rng.random(B) < 0.5, -1, rng.integers(0, 20, B))
    new[0] = -1
    rows = int(np.maximum(new, 0).sum()) + 1
    want = tables.step(ctx, said, new, ring, head, free, tb, rows)
    held = np.maximum(said, -(-ctx // 16))
    over = new < 0
    took = int((want["owned"] - held)[~over].sum())
    assert want["state"][1] == free - took + int(held[over].sum()) and held[over].sum() > np.maximum(said, 0)[over].sum()
    same(run(gpu_lib, ctx, said, new, ring, head, free, tb, rows, repeat=2), want)
