"""Pins of the quantised cache's oracle: tables written by hand, worked blocks, torch's own e4m3, and the calls' refusals,
which need no GPU."""
import ctypes as C

import numpy as np
import pytest
import torch

import oracle
from paper_2506_19225_amd import vxl


def block(*first, fill=0.0):
    return np.array(list(first) + [fill] * (32 - len(first)))


def test_numbers():
    assert oracle.kvq_numbers("fp4").tolist() == [0, 0.5, 1, 1.5, 2, 3, 4, 6]
    want = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(oracle.kvq_numbers("fp8"), want)


@pytest.mark.parametrize("x,codes,byte", [
    ((6.0, -3.0, 0.25, 0.75, 5.0, 2.5), (7, 13, 0, 2, 6, 4), 127),      # ties: 0.25 -> 0, 0.75 -> 1, 5 -> 4, 2.5 -> 2
    ((6.99, 6.0), (7, 7), 127),                                         # 6.99 rounds to the largest number
    ((7.0, -6.0, 0.5), (6, 13, 0), 128),                                # 7 / 2 -> 4 (tie), -6 / 2 -> -3, 0.5 / 2 -> 0
    ((1.0, -0.0), (6, 8), 125),
    ((0.0, -0.0), (0, 8), 17),
    ((2.0 ** -140, 2.0 ** -111), (0, 1), 17),                           # 2^-111 is 0.5 of the smallest scale
    ((2.0 ** -110, 2.0 ** -109), (2, 4), 17),
    ((1.7499 * 2.0 ** 127,), (7,), 252),
])
def test_blocks_by_hand_fp4(x, codes, byte):
    c, s = oracle.kvq_quantise(block(*x), "fp4")
    assert s.tolist() == [byte] and c[:len(codes)].tolist() == list(codes) and not c[len(codes):].any()


@pytest.mark.parametrize("bad", [np.inf, -np.inf, np.nan, 1.75 * 2.0 ** 127])
@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
def test_blocks_that_are_nan(bad, fmt):
    x = np.concatenate([block(1.0, bad), block(1.0)])
    c, s = oracle.kvq_quantise(x, fmt)
    v = oracle.kvq_values(c, s, fmt)
    assert s[0] == 255 and np.isnan(v[:32]).all() and np.array_equal(v[32:], block(1.0))


def test_fp8_against_torch():
    """Where the scale is known, the codes are torch's conversion to e4m3 (round to nearest, ties to even)."""
    rng = np.random.default_rng(5)
    x = (rng.standard_normal((200, 32)) * np.exp2(rng.integers(-30, 30, size=(200, 1)))).astype(np.float32)
    c, s = oracle.kvq_quantise(x, "fp8")
    y = torch.from_numpy(x * np.exp2(127.0 - s[:, :1].astype(np.float64)).astype(np.float32))
    assert y.abs().amax(1).ge(224).all() and y.abs().amax(1).lt(448).all()
    assert np.array_equal(c, y.to(torch.float8_e4m3fn).view(torch.uint8).numpy())


def test_error_of_a_block():
    """Half a step at most: 2^-4 of the value in e4m3 (normal numbers), a quarter of a block's scale 2^2 in e2m1 below its 6."""
    rng = np.random.default_rng(6)
    x = rng.standard_normal((500, 32))
    for fmt, steps in (("fp8", 16.0), ("fp4", 1.0)):
        c, s = oracle.kvq_quantise(x, fmt)
        scale = np.exp2(s.astype(np.float64) - 127)
        assert (np.abs(oracle.kvq_values(c, s, fmt) - x) <= steps * scale).all()


# ---- what the calls refuse, on the host ---------------------------------------------------------
DESC = vxl.make_desc(28, 4, 128, "bf16")


def arg(rows=0x1000, scales=0x2000, fmt=vxl.KVQ_FP4, capacity=100):
    return vxl.KvqCacheArg(rows, scales, fmt, capacity)


def write(k=0x10000, v=0x20000, n=10, cache=None, first=0, desc=DESC):
    return vxl.lib().vxl_kvq_write(C.byref(desc), k, v, n, C.byref(cache or arg()), first, None)


def read(k=0x10000, v=0x20000, n=10, cache=None, first=0, desc=DESC):
    return vxl.lib().vxl_kvq_read(C.byref(desc), C.byref(cache or arg()), first, n, k, v, None)


@pytest.mark.parametrize("call", [write, read])
def test_refusals_of_write_and_read(call):
    bad = vxl.VXL_ERR_INVALID_ARG
    for kw in (dict(k=None), dict(v=None), dict(k=0x10008), dict(v=0x20004), dict(n=-1), dict(first=-1), dict(first=91),
               dict(n=101), dict(n=2**31 - 1), dict(first=2**31 - 1), dict(k=0x1000), dict(v=0x2000), dict(cache=arg(rows=None)),
               dict(cache=arg(scales=None)), dict(cache=arg(rows=0x1008)), dict(cache=arg(scales=0x2004)), dict(cache=arg(capacity=0)),
               dict(desc=vxl.make_desc(28, 3, 128, "bf16"))):
        assert call(**kw) == bad, kw
    for kw in (dict(cache=arg(fmt=2)), dict(cache=arg(fmt=-1)), dict(desc=vxl.make_desc(28, 4, 96, "bf16"))):
        assert call(**kw) == vxl.VXL_ERR_UNSUPPORTED, kw
    assert call(n=0) == call(n=0, k=None, v=None, first=100) == vxl.VXL_OK
    lib = vxl.lib()
    assert lib.vxl_kvq_write(C.byref(DESC), 0x10000, 0x20000, 1, None, 0, None) == bad
    assert lib.vxl_kvq_write(None, 0x10000, 0x20000, 1, C.byref(arg()), 0, None) == bad
    assert lib.vxl_kvq_read(C.byref(DESC), C.byref(arg()), 0, 1, 0x10000, 0x10000, None) == bad


@pytest.mark.parametrize("call", [write, read])
def test_buffers_that_overlap(call):
    """Ten rows of four heads, 10,240 bytes or parts of a longer tensor, and a cache with 51,200 bytes of codes and 3,200 of scales."""
    bad, at = vxl.VXL_ERR_INVALID_ARG, 0x1000000
    cache = arg(rows=at, scales=at + 0x100000)
    ends = [lo + off for lo, size in ((at, 51200), (at + 0x100000, 3200)) for off in (16 - 10240, -16, 16, size - 16)]
    for p in ends:
        assert call(k=p, v=0x20000, cache=cache) == call(k=0x20000, v=p, cache=cache) == bad, hex(p)
        assert call(k=p, v=0x20000, cache=cache, desc=vxl.make_desc(28, 4, 128, "bf16", token_major=True)) == bad
    long = vxl.make_desc(28, 4, 128, "bf16")                            # (rows of a tensor of 100,000 bytes per head)
    long.q_stride_head = long.kv_stride_head = 50000
    long.q_stride_tok = long.kv_stride_tok = 128
    for g in range(4):
        assert call(k=at - g * 100000 - 9 * 256, v=0x20000, cache=cache, desc=long) == bad
    if call is write:
        for off in (0, 16, 51200 - 16, 16 - 3200):
            assert call(cache=arg(rows=at, scales=at + off)) == bad
    else:
        pair = vxl.make_desc(28, 4, 128, "bf16")                        # (a key and its value side by side, 2,048 bytes a token)
        pair.q_stride_head = pair.kv_stride_head = 128
        pair.q_stride_tok = pair.kv_stride_tok = 1024
        for desc, off in ((DESC, 10240 - 16), (DESC, 16 - 10240), (pair, 1024 - 16), (pair, 16), (pair, 2048 * 9 + 1008), (long, 100000 * 3),
                          (long, 2560 - 16)):
            assert call(k=0x800000, v=0x800000 + off, cache=cache, desc=desc) == bad, off


def test_refusals_without_a_layout():
    lib, c = vxl.lib(), C.byref(arg())
    assert lib.vxl_gather_bilevel_kvq(None, C.byref(DESC), c, None, 0x10, 1, 0x10000, 0x20000, 10, 0x30, None,
                                      None) == vxl.VXL_ERR_INVALID_ARG
    assert lib.vxl_bilevel_decode_kvq(None, C.byref(DESC), 0x10000, 1, 1, c, None, 0x10, 10, 0, 0x20000, None, None, 0x30000,
                                      1 << 20, None) == vxl.VXL_ERR_INVALID_ARG


def test_sizes():
    n = C.c_size_t(7)
    lib = vxl.lib()
    for d, fmt, codes, scales in ((128, vxl.KVQ_FP4, 128, 8), (128, vxl.KVQ_FP8, 256, 8), (64, vxl.KVQ_FP4, 64, 4), (64, vxl.KVQ_FP8, 128, 4)):
        assert lib.vxl_kvq_row_bytes(C.byref(vxl.make_desc(4, 2, d, "f32")), fmt, C.byref(n)) == codes and n.value == scales
    assert lib.vxl_kvq_row_bytes(C.byref(DESC), 2, C.byref(n)) == 0 and n.value == 0
    assert lib.vxl_kvq_row_bytes(None, 0, None) == 0
    for b, t, cap in ((0, 1, 10), (1, 0, 10), (1, 1, 0), (-1, 1, 10)):
        assert vxl.workspace_bytes(vxl.OP_DECODE_KVQ, None, DESC, b, t, cap) == 0
    assert vxl.workspace_bytes(vxl.OP_DECODE_KVQ, None, DESC, 2, 3, 1000) >= 8000


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_sizes_past_64_bits(dtype):
    """Numbers of queries, tokens and heads whose products pass 64 bits (and are 0 there) end in a number, or in the refusal."""
    big = 1 << 30
    for hq, hkv, b, t in ((256, 256, big, big), (512, 256, big, big), (2**31 - 1, 2**31 - 1, 2**31 - 1, 2**31 - 1), (2**31 - 1, 1, 1, 2**31 - 1),
                          (1 << 30, 1, 1 << 15, 1 << 30), (256, 256, 1 << 16, 1 << 20), (4, 2, 65536, 1)):
        desc = vxl.make_desc(hq, hkv, 128, dtype)
        assert vxl.workspace_bytes(vxl.OP_DECODE_KVQ, None, desc, b, t, 100) >= b * 404
        assert vxl.debug_kvq_plan(desc, b, t, 100)[1] == 1


def test_cache_objects():
    with pytest.raises(ValueError, match="format"):
        vxl.KvqCache(DESC, "int4", 10)
    with pytest.raises(ValueError, match="format"):
        vxl.KvqCache(vxl.make_desc(28, 4, 96, "bf16"), "fp4", 10)
    rows, scales = torch.zeros(4, 10, 2, 64, dtype=torch.uint8), torch.zeros(4, 10, 2, 4, dtype=torch.uint8)
    for kw in (dict(), dict(rows=rows), dict(capacity=10, rows=rows, scales=scales)):
        with pytest.raises(ValueError, match="capacity or both"):
            vxl.KvqCache(DESC, "fp4", **kw)
    for r, s in ((rows[:3], scales), (rows, scales[:, :9]), (rows.to(torch.int32), scales), (rows, scales[..., :2])):
        with pytest.raises(ValueError, match="uint8 tensor"):
            vxl.KvqCache(DESC, "fp4", rows=r, scales=s)
    with pytest.raises(AssertionError, match="contiguous CUDA"):
        vxl.KvqCache(DESC, "fp4", rows=rows, scales=scales)
    with pytest.raises(TypeError, match="a quantised cache expected"):
        vxl.native().kvq_write(DESC, None, None, 0, C.c_void_p(0x1000), 0, None)
