"""Refusals of the window and block-scale operators (host side only: nothing is launched)."""
import ctypes

import pytest

EINVAL, ENOMEM, ENOTSUP = -22, -12, -95
P = 4096     # stands for any aligned device pointer; only calls that the host refuses get it


def decode(lib, args=(), sh=(), window=64, n_sink=4, ws=1 << 30, **kw):
    s = lib.decode_shape(**dict(dict(batch=4, n_q_heads=8, n_kv_heads=2, max_blocks_per_seq=100, max_context_len=1600,
                                     num_blocks=500), **kw))
    for k, v in dict(sh).items():
        setattr(s, k, v)
    fp8 = kw.get("kv_fp8") or kw.get("block_scales")
    vals = dict(q=P, k=P, v=P, tables=P, ctx=P, scale=0.1, window=window, n_sink=n_sink, ks=P if fp8 else None,
                vs=P if fp8 else None, out=2 * P)
    vals.update(dict(args))
    wsp = vals.pop("ws", 4 * P)
    return lib.lib().window_decode_attention(*vals.values(), ctypes.byref(s), wsp, ws, None)


@pytest.mark.parametrize("kw,sh,code", [
    (dict(head_dim=64), {}, ENOTSUP), (dict(block_size=8), {}, ENOTSUP), ({}, dict(kv_dtype=3), ENOTSUP),
    ({}, dict(kv_dtype=-1), ENOTSUP), ({}, dict(out_dtype=2), ENOTSUP), ({}, dict(reserved=1), EINVAL),
    (dict(batch=-1), {}, EINVAL), (dict(batch=4097), {}, ENOTSUP), (dict(n_q_heads=7), {}, EINVAL),
    (dict(n_q_heads=34), {}, ENOTSUP), (dict(max_context_len=1601), {}, EINVAL), (dict(num_blocks=0), {}, EINVAL),
    (dict(window=0), {}, EINVAL), (dict(window=-5), {}, EINVAL), (dict(n_sink=-1), {}, EINVAL),
    (dict(partition_tokens=48), {}, EINVAL), (dict(workgroups_per_cu=9), {}, EINVAL)])
def test_decode_shapes_refused(host_lib, kw, sh, code):
    assert decode(host_lib, sh=sh, **kw) == code
    assert host_lib.last_error().startswith("window_decode")


@pytest.mark.parametrize("args,kw", [
    (dict(q=None), {}), (dict(k=None), {}), (dict(v=None), {}), (dict(tables=None), {}), (dict(ctx=None), {}),
    (dict(out=None), {}), (dict(ks=P, vs=P), {}), (dict(ks=None), dict(kv_fp8=True)),
    (dict(vs=None), dict(block_scales=True)), (dict(q=P + 8), {}), (dict(k=P + 4), {}), (dict(ctx=P + 2), {}),
    (dict(ks=P + 2), dict(kv_fp8=True)), (dict(out=P), {}), (dict(out=4 * P), {}), (dict(q=4 * P), {}),
    (dict(scale=float("nan")), {}), (dict(ws=4 * P + 16), {})])
def test_decode_pointers_refused(host_lib, args, kw):
    assert decode(host_lib, args, **kw) == EINVAL


def test_decode_workspace(host_lib):
    s = host_lib.decode_shape(4, 8, 2, 100, 1600, 500)
    need = host_lib.window_workspace_size(s, 64, 4)
    assert need > 0 and decode(host_lib, ws=need - 1) == ENOMEM and decode(host_lib, dict(ws=None)) == ENOMEM
    assert host_lib.window_workspace_size(s, 0, 4) == 0 and host_lib.window_workspace_size(s, 64, -1) == 0
    # never more than the whole context's, whatever the window and the sinks are
    assert host_lib.window_workspace_size(s, 2 ** 31 - 1, 2 ** 31 - 1) <= host_lib.workspace_size(s)
    with pytest.raises(host_lib.DpoolError):
        host_lib.WindowDecoder(4, 8, 2, 100, 1600, 500, window=0, device="cpu")


def test_empty_batch_is_fine(host_lib):
    assert decode(host_lib, dict(q=None, k=None, v=None, out=None), batch=0) == 0


def test_other_entry_points_refuse_block_scales(host_lib):
    s = host_lib.decode_shape(4, 8, 2, 100, 1600, 500, block_scales=True)
    assert s.kv_dtype == host_lib.KV_FP8_E4M3_BLOCK and host_lib.workspace_size(s) == 0
    assert host_lib.lib().kv_cache_append(*[P] * 8, ctypes.byref(s), None) == ENOTSUP


def prefill(lib, args=(), sh=(), window=64, n_sink=4, **kw):
    s = lib.prefill_shape(**dict(dict(batch=4, n_q_heads=8, n_kv_heads=2, max_blocks_per_seq=100, max_context_len=1600,
                                      num_blocks=500, total_q=90), **kw))
    for k, v in dict(sh).items():
        setattr(s, k, v)
    fp8 = kw.get("kv_fp8") or kw.get("block_scales")
    vals = dict(q=P, k=P, v=P, tables=P, ctx=P, q_start=P, scale=0.1, window=window, n_sink=n_sink,
                ks=P if fp8 else None, vs=P if fp8 else None, out=2 * P)
    vals.update(dict(args))
    return lib.lib().window_prefill_attention(*vals.values(), ctypes.byref(s), None)


@pytest.mark.parametrize("kw,sh,code", [
    (dict(head_dim=64), {}, ENOTSUP), (dict(block_size=8), {}, ENOTSUP), ({}, dict(kv_dtype=3), ENOTSUP),
    ({}, dict(out_dtype=2), ENOTSUP), ({}, dict(reserved=1), EINVAL), ({}, dict(query_tile=16), EINVAL),
    (dict(batch=-1), {}, EINVAL), (dict(batch=4097), {}, ENOTSUP), (dict(n_q_heads=7), {}, EINVAL),
    (dict(max_context_len=1601), {}, EINVAL), (dict(num_blocks=0), {}, EINVAL), (dict(total_q=-1), {}, EINVAL),
    (dict(window=0), {}, EINVAL), (dict(n_sink=-1), {}, EINVAL),
    (dict(max_blocks_per_seq=5000, max_context_len=65537, window=65000, n_sink=25), {}, ENOTSUP),
    (dict(max_blocks_per_seq=1 << 27, max_context_len=(1 << 30) + 1), {}, ENOTSUP)])
def test_prefill_shapes_refused(host_lib, kw, sh, code):
    assert prefill(host_lib, sh=sh, **kw) == code
    assert host_lib.last_error().startswith("window_prefill_attention")


@pytest.mark.parametrize("args,kw", [
    (dict(q=None), {}), (dict(k=None), {}), (dict(v=None), {}), (dict(tables=None), {}), (dict(ctx=None), {}),
    (dict(q_start=None), {}), (dict(out=None), {}), (dict(ks=P, vs=P), {}), (dict(ks=None), dict(kv_fp8=True)),
    (dict(vs=None), dict(block_scales=True)), (dict(q=P + 8), {}), (dict(v=P + 4), {}), (dict(q_start=P + 2), {}),
    (dict(ks=P + 2), dict(kv_fp8=True)), (dict(out=P), {}), (dict(scale=0.0), {}), (dict(scale=float("inf")), {})])
def test_prefill_pointers_refused(host_lib, args, kw):
    assert prefill(host_lib, args, **kw) == EINVAL


def test_chunked_prefill_refuses_block_scales(host_lib):
    s = host_lib.prefill_shape(4, 8, 2, 100, 1600, 500, 90, block_scales=True)
    assert host_lib.lib().chunked_prefill_attention(*[P] * 6, 0.1, P, P, 2 * P, ctypes.byref(s), None) == ENOTSUP


def test_prefill_of_nothing_is_fine(host_lib):
    assert prefill(host_lib, dict(q=None, out=None), total_q=0) == 0


def append(lib, args=(), sh=(), **kw):
    s = lib.qk_shape(**dict(dict(rows=4, n_q_heads=8, n_kv_heads=2, num_blocks=64, n_positions=100,
                                 block_scales=True), **kw))
    for k, v in dict(sh).items():
        setattr(s, k, v)
    vals = dict(q=P, k=P, v=P, qw=None, kw=None, eps=1e-6, cos=P, pos=P, slots=P, out=2 * P, kc=3 * P, vc=4 * P,
                ks=P + 1, vs=P + 3)
    vals.update(dict(args))
    return lib.lib().qk_norm_rope_append_scaled(*vals.values(), ctypes.byref(s), None)


@pytest.mark.parametrize("kw,sh,code", [
    (dict(head_dim=64), {}, ENOTSUP), (dict(block_size=8), {}, ENOTSUP), ({}, dict(kv_dtype=0), ENOTSUP),
    ({}, dict(kv_dtype=1), ENOTSUP), ({}, dict(kv_dtype=3), ENOTSUP), ({}, dict(reserved=1), EINVAL),
    ({}, dict(interleaved=2), EINVAL), (dict(rotary_dim=24), {}, ENOTSUP), (dict(n_q_heads=-1), {}, EINVAL),
    (dict(n_kv_heads=0), {}, EINVAL), (dict(rows=-1), {}, EINVAL), (dict(rows=1 << 40), {}, EINVAL),
    (dict(num_blocks=0), {}, EINVAL), (dict(n_positions=0), {}, EINVAL), (dict(q_stride=1016), {}, EINVAL),
    (dict(k_stride=260), {}, EINVAL), (dict(v_stride=-256), {}, EINVAL)])
def test_append_shapes_refused(host_lib, kw, sh, code):
    assert append(host_lib, sh=sh, **kw) == code
    assert host_lib.last_error().startswith("qk_norm_rope_append_scaled")


@pytest.mark.parametrize("args,kw", [
    (dict(q=None), {}), (dict(k=None), {}), (dict(v=None), {}), (dict(cos=None), {}), (dict(pos=None), {}),
    (dict(slots=None), {}), (dict(out=None), {}), (dict(kc=None), {}), (dict(vc=None), {}), (dict(ks=None), {}),
    (dict(vs=None), {}), (dict(ks=P + 3), {}), (dict(vc=3 * P), {}), (dict(q=P + 2), {}), (dict(slots=P + 4), {}),
    (dict(out=P), dict(q_stride=2048)), (dict(kc=P + 8), {}), (dict(kw=P, eps=-1.0), {})])
def test_append_pointers_refused(host_lib, args, kw):
    assert append(host_lib, args, **kw) == EINVAL


def test_append_of_nothing_is_fine(host_lib):
    assert append(host_lib, dict(q=None, k=None), rows=0) == 0


def test_append_binding_refuses_gaps(host_lib):
    import torch
    q, k = torch.zeros((4, 8, 128), dtype=torch.bfloat16), torch.zeros((4, 2, 128), dtype=torch.bfloat16)
    c, e = torch.zeros((64, 2, 16, 128), dtype=torch.uint8), torch.zeros((64, 2), dtype=torch.uint8)
    s, i = host_lib.qk_shape(4, 8, 2, 64, 100, block_scales=True), torch.zeros(4, dtype=torch.int64)
    call = lambda **kw: host_lib.qk_norm_rope_append_scaled(**dict(dict(  # noqa: E731
        q=q, k=k, v=k, cos_sin=torch.zeros(100, 128), positions=i.int(), slots=i, q_out=torch.zeros_like(q), k_blocks=c,
        v_blocks=torch.zeros_like(c), k_scale=e, v_scale=torch.zeros_like(e), shape=s), **kw))
    for bad in (dict(q_out=torch.zeros((4, 9, 128), dtype=torch.bfloat16)[:, :8]), dict(k=torch.zeros((8, 2, 128))[::2]),
                dict(k_blocks=torch.zeros((64, 4, 16, 128), dtype=torch.uint8)[:, ::2]),
                dict(v_scale=torch.zeros((64, 4), dtype=torch.uint8)[:, :2]), dict(k_scale=torch.zeros(64, 2)),
                dict(q=None, q_out=None, v=torch.zeros((8, 2, 128))[::2]), dict(slots=i.int()), dict(positions=i),
                dict(slots=torch.zeros(8, dtype=torch.int64)[::2]), dict(positions=torch.zeros(8).int()[::2]),
                dict()):  # (nothing but that the tensors are not on a device)
        with pytest.raises(ValueError):
            call(**bad)


def test_attention_binding_refuses_gaps_and_other_types(host_lib):
    import torch
    q, t = torch.zeros((4, 8, 128), dtype=torch.bfloat16), torch.zeros((4, 100), dtype=torch.int32)
    k, v = torch.zeros((50, 2, 16, 128), dtype=torch.uint8), torch.zeros((50, 2, 128, 16), dtype=torch.uint8)
    heads, blocks = torch.zeros(2), torch.zeros((50, 2), dtype=torch.uint8)
    for scaled, good, bad in ((False, heads, blocks), (True, blocks, heads)):
        dec = host_lib.decode_shape(4, 8, 2, 100, 1600, 50, kv_fp8=True, block_scales=scaled)
        pre = host_lib.prefill_shape(4, 8, 2, 100, 1600, 50, 4, kv_fp8=True, block_scales=scaled)
        d = dict(q=q, k_blocks=k, v_blocks=v, block_tables=t, context_lens=t[0], scale=0.1, window=64, n_sink=0,
                 out=torch.zeros_like(q), k_scale=good, v_scale=good)
        for more in (dict(k_scale=bad), dict(v_scale=bad), dict(q=torch.zeros((4, 128, 8)).transpose(1, 2)),
                     dict(block_tables=torch.zeros((4, 200), dtype=torch.int32)[:, ::2]), dict(k_blocks=k[:, :1]),
                     dict(out=torch.zeros((4, 9, 128))[:, :8]), dict(v_scale=torch.zeros((50, 4)).to(good.dtype)[:, ::2]),
                     dict(context_lens=t[0].long()), dict(block_tables=t.long()), dict(context_lens=t[:, 0]), dict()):
            with pytest.raises(ValueError):
                host_lib.window_decode_attention(**dict(d, **more), shape=dec)
            with pytest.raises(ValueError):
                host_lib.window_prefill_attention(**dict(d, **more), q_start=t[0], shape=pre)
        for start in (t[0].long(), t[:, 0]):
            with pytest.raises(ValueError):
                host_lib.window_prefill_attention(**d, q_start=start, shape=pre)


def test_drafted_trees_refuse_block_scales(host_lib):
    s = host_lib.tree_shape(2, 8, 2, 100, 1600, 50, 4, kv_fp8=True)
    s.kv_dtype = host_lib.KV_FP8_E4M3_BLOCK
    assert host_lib.tree_workspace_size(s) == 0
    p = (ctypes.c_void_p * 1)(P)
    o = (ctypes.c_void_p * 1)(2 * P)
    assert host_lib.lib().kv_cache_accept(p, o, 1, P, P, P, P, P, 4, 3 * P, ctypes.byref(s), None) == ENOTSUP
