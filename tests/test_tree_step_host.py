"""Refusals of the operators of a step that verifies drafted tokens (host side only: nothing is launched)."""
import ctypes

import numpy as np
import pytest

EINVAL, ENOMEM, ENOTSUP = -22, -12, -95
P = 4096     # stands for any aligned device pointer; only calls that the host refuses get it


def tables(lib, args=(), sh=(), **kw):
    shape = dict(batch=4, max_blocks_per_seq=8, num_blocks=64, total_rows=10)
    words = dict(kw).pop("mask_words", 0)
    s = lib.tables_shape(**dict(shape, **kw))
    for k, v in dict(sh).items():
        setattr(s, k, v)
    names = ["context", "owned", "new", "parents", "ring", "state", "tables", "context_out", "owned_out", "state_out",
             "q_start", "slots", "positions", "granted", "mask"]
    vals = {n: P + 256 * i for i, n in enumerate(names)}
    if not words:
        vals["parents"] = vals["mask"] = None
    vals.update(dict(args))
    return lib.lib().kv_tables_step(*[vals[n] for n in names], ctypes.byref(s), None)


@pytest.mark.parametrize("kw,sh,code", [
    (dict(batch=-1), {}, EINVAL), (dict(batch=4097), {}, ENOTSUP), (dict(block_size=32), {}, ENOTSUP),
    (dict(max_blocks_per_seq=0), {}, EINVAL), (dict(max_blocks_per_seq=1 << 28), {}, EINVAL),
    (dict(num_blocks=0), {}, EINVAL), (dict(num_blocks=(1 << 30) + 1), {}, EINVAL),
    (dict(total_rows=-1), {}, EINVAL), (dict(total_rows=(1 << 30) + 1), {}, EINVAL),
    (dict(mask_words=5), {}, ENOTSUP), (dict(mask_words=-1), {}, ENOTSUP), ({}, dict(reserved=1), EINVAL)])
def test_tables_shapes_refused(host_lib, kw, sh, code):
    assert tables(host_lib, sh=sh, **kw) == code
    assert host_lib.last_error() != ""


@pytest.mark.parametrize("args,words", [
    (dict(context=None), 0), (dict(owned=None), 0), (dict(new=None), 0), (dict(ring=None), 0), (dict(state=None), 0),
    (dict(tables=None), 0), (dict(q_start=None), 0), (dict(slots=None), 0), (dict(positions=None), 0),
    (dict(granted=None), 0), (dict(parents=None), 1), (dict(mask=None), 1), (dict(parents=P), 0),
    (dict(parents=P, mask=P + 64), 0), (dict(slots=P + 4), 0), (dict(context=P + 2), 0), (dict(mask=P + 4), 1),
    (dict(context=P, context_out=P), 0), (dict(state=P, state_out=P), 0), (dict(owned=P, owned_out=P), 0),
    (dict(new=P, q_start=P), 0), (dict(parents=P, positions=P), 1)])
def test_tables_pointers_refused(host_lib, args, words):
    assert tables(host_lib, args, mask_words=words) == EINVAL
    assert host_lib.lib().kv_tables_step(*[P] * 15, None, None) == EINVAL


def qk(lib, args=(), sh=(), **kw):
    s = lib.qk_shape(**dict(dict(rows=4, n_q_heads=8, n_kv_heads=2, num_blocks=64, n_positions=100), **kw))
    for k, v in dict(sh).items():
        setattr(s, k, v)
    fp8 = bool(kw.get("kv_fp8"))
    vals = dict(q=P, k=P, v=P, qw=None, kw=None, eps=1e-6, cos=P, pos=P, slots=P, out=2 * P, kc=P, vc=P,
                ks=P if fp8 else None, vs=P if fp8 else None)
    vals.update(dict(args))
    return lib.lib().qk_norm_rope_append(*vals.values(), ctypes.byref(s), None)


@pytest.mark.parametrize("kw,sh,code", [
    (dict(head_dim=64), {}, ENOTSUP), (dict(block_size=8), {}, ENOTSUP), ({}, dict(kv_dtype=2), ENOTSUP),
    ({}, dict(reserved=1), EINVAL), ({}, dict(interleaved=2), EINVAL), (dict(rotary_dim=24), {}, ENOTSUP),
    (dict(rotary_dim=144), {}, ENOTSUP), (dict(rotary_dim=-16), {}, ENOTSUP),
    (dict(n_q_heads=0), {}, EINVAL), (dict(n_kv_heads=0), {}, EINVAL), (dict(n_q_heads=65537), {}, EINVAL),
    (dict(rows=-1), {}, EINVAL), (dict(rows=1 << 40), {}, EINVAL), (dict(num_blocks=0), {}, EINVAL),
    (dict(n_positions=0), {}, EINVAL), (dict(q_stride=1016), {}, EINVAL), (dict(k_stride=260), {}, EINVAL),
    (dict(v_stride=-256), {}, EINVAL), (dict(q_stride=1 << 62), {}, EINVAL)])
def test_qk_shapes_refused(host_lib, kw, sh, code):
    assert qk(host_lib, sh=sh, **kw) == code
    assert host_lib.last_error() != ""


@pytest.mark.parametrize("args,kw", [
    (dict(q=None), {}), (dict(k=None), {}), (dict(v=None), {}), (dict(cos=None), {}), (dict(pos=None), {}),
    (dict(slots=None), {}), (dict(out=None), {}), (dict(kc=None), {}), (dict(vc=None), {}), (dict(q=P + 2), {}),
    (dict(slots=P + 4), {}), (dict(pos=P + 2), {}), (dict(ks=P, vs=P), {}), (dict(ks=None), dict(kv_fp8=True)),
    (dict(vs=None), dict(kv_fp8=True)), (dict(out=P), dict(q_stride=2048)), (dict(qw=P + 8), {}),
    (dict(qw=P, eps=-1.0), {}), (dict(kw=P, eps=float("nan")), {}), (dict(kw=P, eps=float("inf")), {})])
def test_qk_pointers_refused(host_lib, args, kw):
    assert qk(host_lib, args, **kw) == EINVAL


def tshape(lib, sh=(), **kw):
    s = lib.tree_shape(**dict(dict(batch=4, n_q_heads=8, n_kv_heads=2, max_blocks_per_seq=8, max_context_len=128,
                                   num_blocks=64, total_q=10), **kw))
    for k, v in dict(sh).items():
        setattr(s, k, v)
    return s


@pytest.mark.parametrize("kw,sh,code", [
    (dict(head_dim=64), {}, ENOTSUP), (dict(block_size=8), {}, ENOTSUP), ({}, dict(kv_dtype=2), ENOTSUP),
    ({}, dict(reserved=1), EINVAL), (dict(batch=-1), {}, EINVAL), (dict(batch=4097), {}, ENOTSUP),
    (dict(mask_words=0), {}, ENOTSUP), (dict(mask_words=5), {}, ENOTSUP), (dict(n_q_heads=9), {}, EINVAL),
    (dict(n_q_heads=0), {}, EINVAL), (dict(n_kv_heads=-2), {}, EINVAL), (dict(n_q_heads=4096, n_kv_heads=2), {}, ENOTSUP),
    (dict(n_q_heads=65536, n_kv_heads=65536), {}, ENOTSUP), (dict(max_blocks_per_seq=7), {}, EINVAL),
    (dict(max_context_len=-1), {}, EINVAL), (dict(num_blocks=0), {}, EINVAL), (dict(num_blocks=1 << 31), {}, EINVAL),
    (dict(max_context_len=(1 << 30) + 1, max_blocks_per_seq=1 << 27), {}, ENOTSUP), (dict(total_q=-1), {}, EINVAL),
    (dict(total_q=1 << 31), {}, EINVAL)])
def test_tree_shapes_refused(host_lib, kw, sh, code):
    s = tshape(host_lib, sh, **kw)
    L = host_lib.lib()
    assert L.tree_decode_workspace_size(ctypes.byref(s)) == 0
    assert L.tree_decode_attention(*[P] * 7, 1.0, None, None, P, ctypes.byref(s), P, 1 << 30, None) == code
    assert host_lib.last_error() != ""
    if code == EINVAL and kw and "total_q" not in kw and "mask_words" not in kw and "n_q_heads" not in kw:
        assert accept(host_lib, shape=s) in (EINVAL, ENOTSUP)


def test_tree_arguments_refused(host_lib):
    L = host_lib.lib()
    s, s8 = tshape(host_lib), tshape(host_lib, kv_fp8=True)
    need = L.tree_decode_workspace_size(ctypes.byref(s))
    assert need > 0

    def call(shape=s, scale=1.0, ks=None, vs=None, out=P, ws=P, n=1 << 30, **ptr):
        names = ["q", "k", "v", "tables", "ctx", "q_start", "mask"]
        vals = [ptr.get(x, P) for x in names]
        return L.tree_decode_attention(*vals, scale, ks, vs, out, ctypes.byref(shape), ws, n, None)

    for name in ("q", "k", "v", "tables", "ctx", "q_start", "mask"):
        assert call(**{name: None}) == EINVAL
        assert call(**{name: P + 2}) == EINVAL
    assert call(mask=P + 4) == EINVAL and call(q=P + 8) == EINVAL and call(out=None) == EINVAL and call(out=P + 8) == EINVAL
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        assert call(scale=scale) == EINVAL
    assert call(ks=P, vs=P) == EINVAL and call(shape=s8) == EINVAL and call(shape=s8, ks=P) == EINVAL
    assert call(ws=None) == EINVAL and call(ws=P + 128) == EINVAL and call(n=need - 1) == ENOMEM
    assert L.tree_decode_attention(*[None] * 7, 1.0, None, None, None, None, None, 0, None) == EINVAL
    empty = tshape(host_lib, batch=0)
    assert L.tree_decode_attention(*[None] * 7, 1.0, None, None, None, ctypes.byref(empty), None, 0, None) == 0
    empty = tshape(host_lib, total_q=0)
    assert L.tree_decode_attention(*[None] * 7, 1.0, None, None, None, ctypes.byref(empty), None, 0, None) == 0


def accept(lib, shape=None, k=(P, 2 * P), v=(3 * P, 4 * P), n=2, max_accept=4, out=9 * P, **ptr):
    arr = lambda x: (ctypes.c_void_p * len(x))(*x) if x is not None else None  # noqa: E731
    names = ["tables", "ctx", "q_start", "accepted", "n_accepted"]
    vals = [ptr.get(x, P + 64 * i) for i, x in enumerate(names)]
    shape = tshape(lib) if shape is None else shape
    return lib.lib().kv_cache_accept(arr(k), arr(v), n, *vals, max_accept, out, ctypes.byref(shape), None)


def test_accept_arguments_refused(host_lib):
    assert accept(host_lib, n=0) == EINVAL and accept(host_lib, n=-1) == EINVAL
    assert accept(host_lib, max_accept=0) == EINVAL
    assert accept(host_lib, k=None) == EINVAL and accept(host_lib, v=None) == EINVAL
    assert accept(host_lib, k=(P, None)) == EINVAL and accept(host_lib, v=(P, P + 2)) == EINVAL
    for name in ("tables", "ctx", "q_start", "accepted", "n_accepted"):
        assert accept(host_lib, **{name: None}) == EINVAL and accept(host_lib, **{name: P + 2}) == EINVAL
    assert accept(host_lib, out=None) == EINVAL and accept(host_lib, out=P + 64) == EINVAL   # the lengths themselves
    for kw, code in ((dict(head_dim=64), ENOTSUP), (dict(block_size=8), ENOTSUP), (dict(batch=-1), EINVAL),
                     (dict(batch=4097), ENOTSUP), (dict(n_q_heads=0, n_kv_heads=0), EINVAL),
                     (dict(max_blocks_per_seq=7), EINVAL), (dict(num_blocks=0), EINVAL), (dict(total_q=-1), EINVAL)):
        assert accept(host_lib, shape=tshape(host_lib, **kw)) == code
    assert accept(host_lib, shape=tshape(host_lib, sh=dict(kv_dtype=7))) == ENOTSUP
    assert accept(host_lib, shape=tshape(host_lib, sh=dict(reserved=7))) == EINVAL
    assert accept(host_lib, shape=tshape(host_lib, batch=0)) == 0
    assert host_lib.lib().kv_cache_accept(None, None, 1, *[None] * 5, 1, None, None, None) == EINVAL


def test_calls_with_nothing_to_do(host_lib):
    assert qk(host_lib, dict(q=None, k=None, v=None, out=None, kc=None, vc=None), rows=0) == 0


def test_binding_refuses_unequal_layers(host_lib):
    with pytest.raises(ValueError):
        host_lib.CacheLayers([np.zeros(1)], [])


def test_same_tensor_twice_refused(host_lib):
    assert accept(host_lib, k=(P, P)) == EINVAL and accept(host_lib, v=(P, P)) == EINVAL       # a layer given twice
    assert accept(host_lib, k=(P, 2 * P), v=(3 * P, P)) == EINVAL and accept(host_lib, k=(P,), v=(P,), n=1) == EINVAL
    many = [P * (i + 1) for i in range(2050)]
    assert accept(host_lib, k=many[:1025], v=many[1025:], n=1025) == ENOTSUP
    assert accept(host_lib, k=many[:1023] + many[:1], v=many[1025:2049], n=1024) == EINVAL
    for a, b in (("context_out", "owned_out"), ("granted", "q_start"), ("ring", "tables"), ("state_out", "granted")):
        assert tables(host_lib, {a: 2 * P, b: 2 * P}) == EINVAL
    assert tables(host_lib, dict(slots=2 * P, mask=2 * P), mask_words=1) == EINVAL
    assert tables(host_lib, dict(ring=2 * P, new=2 * P)) == EINVAL


def test_binding_refuses_a_sliced_path(host_lib):
    import torch
    x = torch.zeros(4, 8, dtype=torch.int32)
    layers = host_lib.CacheLayers([x], [torch.zeros(1)])
    for accepted in (x[:, :3], x[0]):
        with pytest.raises(ValueError):
            host_lib.kv_cache_accept(layers, x, x, x, accepted, x, x, tshape(host_lib))


def test_outputs_that_are_inputs_refused(host_lib):
    L, s = host_lib.lib(), tshape(host_lib)
    rest = [P + 4096 * i for i in range(1, 7)]
    for q, out, ws in ((P, P, 32 * P), (P, 32 * P, P), (P, 32 * P, 32 * P)):
        assert L.tree_decode_attention(q, *rest, 1.0, None, None, out, ctypes.byref(s), ws, 1 << 30, None) == EINVAL
    for name in ("tables", "ctx", "q_start", "accepted", "n_accepted"):
        assert accept(host_lib, out=9 * P, **{name: 9 * P}) == EINVAL
    for name in ("k", "v"):
        assert qk(host_lib, {name: 2 * P}) == EINVAL and "q_out" in host_lib.last_error()


def test_binding_refuses_rows_at_other_strides(host_lib):
    """Slices of one projection with the strides of tensors of their own would read other rows' values."""
    import torch
    rows, hq, hkv = 5, 4, 2
    qkv = torch.zeros(rows, (hq + 2 * hkv) * 128, dtype=torch.bfloat16)
    sliced = qkv.split([hq * 128, hkv * 128, hkv * 128], dim=1)
    own = [x.contiguous() for x in sliced]
    x = torch.zeros(rows, dtype=torch.int64)

    def call(tensors, out=None, n=rows, **strides):
        # (a shape that the library refuses: what gets that far was not refused for its strides)
        s = host_lib.qk_shape(n, hq, hkv, 64, 100, **strides)
        s.reserved = 1
        out = torch.zeros(rows, hq, 128, dtype=torch.bfloat16) if out is None else out
        host_lib.qk_norm_rope_append(*tensors, torch.zeros(100, 128), x, x, out, x, x, s, stream=0)

    wide = dict(q_stride=1024, k_stride=1024, v_stride=1024)
    heads = lambda ts: [t.unflatten(1, (-1, 128)) for t in ts]  # noqa: E731
    for tensors, strides in ((own, {}), (sliced, wide), (heads(own), {}), (heads(sliced), wide),
                             ([t.reshape(-1, 128) for t in own], {}), ([t.flatten() for t in own], {}),
                             ([qkv.flatten()] * 3, wide), ([t[:, None] for t in heads(sliced)], wide),
                             ([t[None] for t in heads(sliced)], wide),
                             ([t.unflatten(0, (1, rows)) for t in sliced], wide)):
        with pytest.raises(host_lib.DpoolError):
            call(tensors, **strides)
    two = torch.zeros(2, 3, (hq + 2 * hkv) * 128)               # rows of two dimensions
    with pytest.raises(host_lib.DpoolError):
        call(two.split([hq * 128, hkv * 128, hkv * 128], dim=2), n=6, **wide)
    with pytest.raises(host_lib.DpoolError):
        call([t[:1] for t in sliced], n=1)                      # one row: no stride to speak of
    for i in range(3):
        for bad in (sliced[i], heads(sliced)[i], own[i][::2], own[i].unflatten(1, (-1, 128)).flip(0).transpose(1, 2),
                    heads(own)[i].transpose(0, 1), own[i][:1].expand(rows, -1)):
            with pytest.raises(ValueError, match="strides"):
                call([bad if j == i else own[j] for j in range(3)])
        with pytest.raises(ValueError, match="strides"):
            call([own[i] if j == i else sliced[j] for j in range(3)], **wide)
        with pytest.raises(ValueError, match="strides"):        # every other row
            call([two[:, ::2].split([hq * 128, hkv * 128, hkv * 128], dim=2)[j] for j in range(3)], n=4, **wide)
    with pytest.raises(ValueError, match="contiguous"):
        call(own, out=torch.zeros(rows, hq, 256, dtype=torch.bfloat16)[..., :128])


def test_binding_takes_rows_that_no_stride_reaches(host_lib):
    """No rows, or the first of many: what lies between rows does not matter then."""
    import torch
    x = torch.zeros(5, dtype=torch.int64)
    qkv = torch.zeros(5, 8 * 128, dtype=torch.bfloat16)
    for rows, given in ((0, qkv[:0]), (0, torch.zeros(0)), (1, qkv), (1, qkv.unflatten(1, (-1, 128)))):
        q, k, v = (given[:, :4], given[:, 4:6], given[:, 6:]) if given.dim() == 3 else (
            (given[:, :512], given[:, 512:768], given[:, 768:]) if given.dim() == 2 else (given,) * 3)
        s = host_lib.qk_shape(rows, 4, 2, 64, 100)
        s.reserved = 1          # refused by the library: got as far as that
        with pytest.raises(host_lib.DpoolError):
            host_lib.qk_norm_rope_append(q, k, v, x, x, x, torch.zeros(5, 4, 128), x, x, s, stream=0)
    s = host_lib.qk_shape(2, 4, 2, 64, 100)
    with pytest.raises(ValueError, match="strides"):
        host_lib.qk_norm_rope_append(qkv[:, :512], qkv[:, 512:768], qkv[:, 768:], x, x, x, torch.zeros(5, 4, 128), x, x,
                                     s, stream=0)


def test_binding_refuses_caches_with_gaps(host_lib):
    """Layers interleaved in one tensor are no caches of their own: tokens would move in other layers' blocks."""
    import torch
    both = torch.zeros(4, 2, 2, 16, 128)
    k, v = [both[:, i] for i in range(2)], [x.contiguous() for x in both.transpose(3, 4).unbind(1)]
    for a, b in ((k, v), (v, k)):
        with pytest.raises(ValueError, match="contiguous"):
            host_lib.CacheLayers(a, b)
    apart = both.transpose(0, 1).contiguous()
    assert host_lib.CacheLayers(list(apart), v).n == 2
