"""What a vxl_mixed_attend call takes for its sizes, on the host."""
import itertools

import pytest

from paper_2506_19225_amd import vxl


def test_plans_fit_their_calls():
    """Splits no finer than tiles, parts no finer than blocks of query rows, and a workspace for what they leave."""
    for (hq, hkv, d), dtype in itertools.product([(28, 4, 128), (14, 2, 64), (8, 1, 128), (40, 1, 64), (4, 4, 64)], ["bf16", "f32"]):
        desc = vxl.make_desc(hq, hkv, d, dtype)
        for batch, t, cap in itertools.product([1, 3, 64], [1, 4, 7, 64, 1000, 20000], [1, 31, 65, 1000, 18688, 1 << 20]):
            waves, n_split, n_part = vxl.debug_mixed_plan(desc, batch, t, cap)
            rows, units = hq // hkv * t, batch * hkv
            few = rows <= 32
            assert waves in ((0,) if few or dtype == "f32" else (4, 8))
            tile = 64 if waves else 4 * 32                       # (the others: one of 32 keys for each of four waves)
            assert 1 <= n_split <= (cap + tile - 1) // tile
            assert 1 <= n_part <= (1 if few or dtype == "f32" else (rows + 63) // 64)
            need = units * rows * 4 + (n_split > 1) * units * n_split * rows * (d * 4 + 8) + few * units * rows * cap * 4
            need += (n_part > 1) * n_part * units * cap * 4
            have = vxl.workspace_bytes(vxl.OP_MIXED_ATTEND, None, desc, batch, t, cap)
            assert have >= need


def test_no_plan_for_what_is_no_call():
    desc = vxl.make_desc(8, 2, 64, "bf16")
    for batch, t, cap in [(0, 1, 10), (1, 0, 10), (1, 1, 0), (1, 1, -5), (40000, 1, 10), (1, 1 << 29, 10)]:
        with pytest.raises(ValueError):
            vxl.debug_mixed_plan(desc, batch, t, cap)
        assert vxl.workspace_bytes(vxl.OP_MIXED_ATTEND, None, desc, batch, t, cap) == 0


def test_forced_plans_stay_within_their_sizes():
    desc = vxl.make_desc(28, 4, 128, "bf16")
    try:
        vxl.debug_mixed_force(4, 1000, 1000)
        assert vxl.debug_mixed_plan(desc, 1, 40, 300) == (4, 5, 5)
        vxl.debug_mixed_force(8, 2, 3)
        assert vxl.debug_mixed_plan(desc, 1, 40, 300) == (8, 2, 3)
    finally:
        vxl.debug_mixed_force()
    waves, n_split, n_part = vxl.debug_mixed_plan(desc, 1, 40, 300)
    assert n_split <= 5 and n_part <= 5
