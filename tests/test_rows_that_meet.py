"""Which rows of two tensors meet, where a descriptor puts rows of one between rows of the other: calls that are answered by their
checks, or end in a library whose launches fail without a device."""
import ctypes as C

import pytest
import torch

from paper_2506_19225_amd import vxl

BASE, FAR = 1 << 40, 1 << 45


@pytest.fixture(autouse=True)
def no_device():
    if torch.cuda.is_available():
        pytest.skip("made-up addresses are not for a device")


def fused(hq, hkv, d, parts):
    """Rows of a token of hq query and hkv KV heads, `parts` heads in all, side by side."""
    desc = vxl.make_desc(hq, hkv, d, "bf16")
    desc.q_stride_head = desc.kv_stride_head = d
    desc.q_stride_tok = desc.kv_stride_tok = parts * d
    return desc


@pytest.mark.parametrize("heads", [2, 1024, 1025, 5000])
def test_keys_and_values_side_by_side_in_a_tokens_row(heads):
    d, n = 64, 9
    desc = fused(heads, heads, d, 2 * heads)
    cache = vxl.KvqCacheArg(FAR, 2 * FAR, vxl.KVQ_FP8, n)
    read = lambda k, v: vxl.lib().vxl_kvq_read(C.byref(desc), C.byref(cache), 0, n, k, v, None)  # noqa: E731
    row = d * 2
    assert read(BASE, BASE + heads * row) == read(BASE + heads * row, BASE) == vxl.VXL_ERR_HIP
    for off in ((heads - 1) * row, heads * row - 16, heads * row + 16, (3 * heads - 1) * row):
        assert read(BASE, BASE + off) == vxl.VXL_ERR_INVALID_ARG, off
    assert read(BASE, BASE + (2 * heads * (n - 1) + heads) * row) == read(BASE, BASE + 2 * heads * n * row) == vxl.VXL_ERR_HIP


@pytest.mark.parametrize("hq,hkv", [(6, 2), (4096, 512), (4096, 4096)])
def test_queries_and_keys_side_by_side_in_a_tokens_row(hq, hkv):
    d, n = 64, 5
    desc, arg = fused(hq, hkv, d, hq + hkv), vxl.RotaryArg(FAR, d, 0, 1.0, 0)
    rotate = lambda q, k: vxl.lib().vxl_rotate(C.byref(desc), C.byref(arg), 2 * FAR, n, q, k, q, k, None)  # noqa: E731
    row = d * 2
    assert rotate(BASE, BASE + hq * row) == rotate(BASE + hkv * row, BASE) == vxl.VXL_ERR_HIP
    for off in ((hq - 1) * row, hq * row - 16, hq * row + 16):
        assert rotate(BASE, BASE + off) == vxl.VXL_ERR_INVALID_ARG, off
