"""What the Python binding of the window and block-scale operators refuses (host side only: nothing is launched).

Tensors are in host memory; where the device counts, a stand-in says that they
are on device 0.  Every call here has one thing wrong and is refused for it.
"""
import pytest
import torch

B, HQ, HKV, MB, NB, ROWS, CAP = 3, 8, 2, 10, 7, 5, 160


class Stub:
    """A tensor that says it is on another device than it is."""

    def __init__(self, t, dev=0):
        self.t, self.dev = t, dev

    def get_device(self):
        return self.dev

    def __getattr__(self, name):
        return getattr(self.t, name)


def attention(lib, kind, cache):
    """(call, its arguments): a decode or a prefill over a bf16, e4m3 or block-scaled cache."""
    kw = dict(kv_fp8=cache == "head", block_scales=cache == "block")
    rows = B if kind == "decode" else ROWS
    tile = torch.bfloat16 if cache == "bf16" else torch.uint8
    scale = {"bf16": None, "head": torch.zeros(HKV), "block": torch.zeros((NB, HKV), dtype=torch.uint8)}[cache]
    args = dict(q=torch.zeros((rows, HQ, 128), dtype=torch.bfloat16), k_blocks=torch.zeros((NB, HKV, 16, 128), dtype=tile),
                v_blocks=torch.zeros((NB, HKV, 128, 16), dtype=tile), block_tables=torch.zeros((B, MB), dtype=torch.int32),
                context_lens=torch.zeros(B, dtype=torch.int32), out=torch.zeros((rows, HQ, 128), dtype=torch.bfloat16))
    if scale is not None:
        args.update(k_scale=scale, v_scale=scale.clone())
    if kind == "decode":
        args["workspace"] = torch.zeros(1 << 16, dtype=torch.uint8)
        fn, shape = lib.window_decode_attention, lib.decode_shape(B, HQ, HKV, MB, CAP, NB, **kw)
    else:
        args["q_start"] = torch.zeros(B + 1, dtype=torch.int32)
        fn, shape = lib.window_prefill_attention, lib.prefill_shape(B, HQ, HKV, MB, CAP, NB, ROWS, **kw)
    return (lambda **more: fn(**dict(dict(args, scale=0.1, window=64, n_sink=0, shape=shape), **more))), args


CASES = [(k, c) for k in ("decode", "prefill") for c in ("bf16", "head", "block")]


@pytest.mark.parametrize("kind,cache", CASES)
def test_attention_tensors_elsewhere(host_lib, kind, cache):
    call, args = attention(host_lib, kind, cache)
    on = {n: Stub(t) for n, t in args.items()}
    for name in args:
        for dev in (-1, 1):
            with pytest.raises(ValueError, match="current device"):
                call(**dict(on, **{name: Stub(args[name], dev)}))
    with pytest.raises(ValueError, match="current device"):
        call()


@pytest.mark.parametrize("kind,cache", CASES)
def test_attention_other_types(host_lib, kind, cache):
    call, args = attention(host_lib, kind, cache)
    wrong = {"q": (torch.float32, torch.float16, torch.uint8), "out": (torch.float32, torch.float16, torch.uint8),
             "block_tables": (torch.int64, torch.float32, torch.int16), "context_lens": (torch.int64, torch.float32),
             "q_start": (torch.int64, torch.float32)}
    wrong["k_blocks"] = wrong["v_blocks"] = ((torch.float16, torch.float32, torch.uint8, torch.float8_e4m3fn)
                                             if cache == "bf16" else
                                             (torch.bfloat16, torch.int16, torch.float8_e5m2, torch.float8_e4m3fnuz))
    wrong["k_scale"] = wrong["v_scale"] = ((torch.float64, torch.int32, torch.uint8, torch.bfloat16) if cache == "head"
                                           else (torch.float32, torch.float8_e4m3fn, torch.bool))
    for name, types in wrong.items():
        for t in types if name in args else ():
            with pytest.raises(ValueError, match=r"bf16|int32|fp32|exponent"):
                call(**{name: torch.zeros(args[name].shape, dtype=t)})
    shape = (host_lib.decode_shape(B, HQ, HKV, MB, CAP, NB, cache == "head", True, block_scales=cache == "block")
             if kind == "decode" else host_lib.prefill_shape(B, HQ, HKV, MB, CAP, NB, ROWS, cache == "head", True,
                                                             block_scales=cache == "block"))
    with pytest.raises(ValueError, match="out is fp32"):       # a bf16 tensor is half as long
        call(shape=shape)


@pytest.mark.parametrize("kind,cache", CASES)
def test_attention_tensors_that_are_too_small(host_lib, kind, cache):
    call, args = attention(host_lib, kind, cache)
    for name, t in args.items():
        if name != "workspace":                                # (the library looks at its size)
            with pytest.raises(ValueError, match="elements|element more"):
                call(**{name: t.flatten()[:-1]})


@pytest.mark.parametrize("kind,cache", CASES)
def test_attention_tensors_with_gaps(host_lib, kind, cache):
    call, args = attention(host_lib, kind, cache)
    for name, t in args.items():
        with pytest.raises(ValueError, match="contiguous"):
            call(**{name: torch.zeros((*t.shape, 2), dtype=t.dtype)[..., 0]})


@pytest.mark.parametrize("kind,cache", CASES)
def test_attention_types_that_hold_the_same_bits(host_lib, kind, cache):
    """Refused for where they are, and for nothing else."""
    call, args = attention(host_lib, kind, cache)
    same = {"q": (torch.int16, torch.uint16), "out": (torch.int16,)}
    same["k_blocks"] = same["v_blocks"] = ((torch.int16, torch.uint16) if cache == "bf16" else
                                           (torch.int8, torch.float8_e4m3fn))
    if cache == "block":
        same["k_scale"] = same["v_scale"] = (torch.int8, torch.float8_e8m0fnu)
    for name, types in same.items():
        for t in types if name in args else ():
            with pytest.raises(ValueError, match="current device"):
                call(**{name: torch.zeros(args[name].shape, dtype=torch.uint8 if t.itemsize == 1 else torch.int16).view(t)})


# ---------------------------------------------------------------- the cache write

def write(lib, queries=True):
    """(call, its arguments): the write of four rows into a cache with block scales."""
    hq = HQ if queries else 0
    args = dict(k=torch.zeros((4, HKV, 128), dtype=torch.bfloat16), v=torch.zeros((4, HKV, 128), dtype=torch.bfloat16),
                cos_sin=torch.zeros((20, 128)), positions=torch.zeros(4, dtype=torch.int32),
                slots=torch.zeros(4, dtype=torch.int64), k_blocks=torch.zeros((NB, HKV, 16, 128), dtype=torch.uint8),
                v_blocks=torch.zeros((NB, HKV, 128, 16), dtype=torch.uint8),
                k_scale=torch.zeros((NB, HKV), dtype=torch.uint8), v_scale=torch.zeros((NB, HKV), dtype=torch.uint8),
                k_weight=torch.zeros(128, dtype=torch.bfloat16))
    if queries:
        args.update(q=torch.zeros((4, HQ, 128), dtype=torch.bfloat16), q_out=torch.zeros((4, HQ, 128), dtype=torch.bfloat16),
                    q_weight=torch.zeros(128, dtype=torch.bfloat16))
    shape = lib.qk_shape(4, hq, HKV, NB, 20, block_scales=True)
    none = {} if queries else dict(q=None, q_out=None)
    return (lambda **more: lib.qk_norm_rope_append_scaled(**dict(dict(args, shape=shape, **none), **more))), args


@pytest.mark.parametrize("queries", [True, False])
def test_write_tensors_elsewhere(host_lib, queries):
    call, args = write(host_lib, queries)
    on = {n: Stub(t) for n, t in args.items()}
    for name in args:
        for dev in (-1, 1):
            with pytest.raises(ValueError, match="current device"):
                call(**dict(on, **{name: Stub(args[name], dev)}))
    with pytest.raises(ValueError, match="current device"):
        call()


@pytest.mark.parametrize("queries", [True, False])
def test_write_other_types(host_lib, queries):
    call, args = write(host_lib, queries)
    wrong = dict.fromkeys(("q", "q_out", "k", "v", "q_weight", "k_weight"), (torch.float16, torch.float32, torch.uint8))
    wrong.update(dict.fromkeys(("k_blocks", "v_blocks"), (torch.bfloat16, torch.float8_e5m2, torch.float8_e4m3fnuz)))
    wrong.update(dict.fromkeys(("k_scale", "v_scale"), (torch.float32, torch.bool, torch.float8_e4m3fn)))
    wrong.update(cos_sin=(torch.float64, torch.bfloat16, torch.int32), positions=(torch.int64, torch.float32),
                 slots=(torch.int32, torch.float64))
    for name, types in wrong.items():
        for t in types if name in args else ():
            with pytest.raises(ValueError, match="bf16|fp32|int32|exponent"):
                call(**{name: torch.zeros(args[name].shape, dtype=t)})


@pytest.mark.parametrize("queries", [True, False])
def test_write_tensors_that_are_too_small(host_lib, queries):
    call, args = write(host_lib, queries)
    for name, t in args.items():
        small = t[:-1] if name in ("q", "q_out", "k", "v") else t.flatten()[:-1]
        with pytest.raises(ValueError, match="elements|row for each"):
            call(**{name: small})
        with pytest.raises(ValueError, match="elements|row for each"):
            call(**{name: t[:0]})


@pytest.mark.parametrize("queries", [True, False])
def test_write_tensors_with_gaps(host_lib, queries):
    call, args = write(host_lib, queries)
    for name, t in args.items():
        with pytest.raises(ValueError, match="contiguous|strides"):
            call(**{name: torch.zeros((*t.shape, 2), dtype=t.dtype)[..., 0]})


def test_write_without_an_output(host_lib):
    call, _ = write(host_lib)
    with pytest.raises(ValueError, match="q_out"):
        call(q_out=None)


def test_write_types_that_hold_the_same_bits(host_lib):
    call, args = write(host_lib)
    same = dict.fromkeys(("q", "q_out", "k", "v", "q_weight", "k_weight"), (torch.int16, torch.uint16))
    same.update(dict.fromkeys(("k_blocks", "v_blocks"), (torch.int8, torch.float8_e4m3fn)))
    same.update(dict.fromkeys(("k_scale", "v_scale"), (torch.int8, torch.float8_e8m0fnu)))
    for name, types in same.items():
        for t in types:
            with pytest.raises(ValueError, match="current device"):
                call(**{name: torch.zeros(args[name].shape, dtype=torch.uint8 if t.itemsize == 1 else torch.int16).view(t)})
