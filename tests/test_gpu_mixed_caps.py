"""Capped logits of growing mixed sets: what no token sees has no say in them, and caps far above the logits."""
import numpy as np
import pytest

import oracle
from paper_2506_19225_amd import vxl

from mixed_util import E, attend, check_attend, sets, stored, values

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("t,plan", [(1, (0, 1, 0)), (1, (0, 3, 0)), (4, (0, 2, 0)), (50, (4, 1, 1)), (50, (8, 3, 2))])
@pytest.mark.parametrize("rule", [dict(causal=True, window=500), dict(window=300, n_always=20),
                                  dict(causal=True, slopes=2.0 ** (-8 * (np.arange(8) + 1) / 8) / 512)])
def test_keys_that_no_token_sees_change_no_bit(rule, t, plan, dtype):
    """Empty rows, rows before all windows and behind all tokens, among rows that are seen in every tile, and padding tokens: keys, finite values
    and queries of them small, large (far past the cap), infinite and NaN.  All logits that count are far below the cap."""
    n, cap = 640, 50.0
    rng = np.random.default_rng(t)
    k, v, pos = sets(rng, 1, 2, n, 64, dtype, [n], spread=0.5)
    qd = values(rng, (1, t, 8, 64), dtype)
    q_pos = (1000 + np.arange(t, dtype=np.int32))[None]
    pos[rng.random(pos.shape) < 0.1] = -1
    padding = np.arange(t) % 3 == 1
    q_pos[0, padding] = -1
    weight = rng.random((1, 2, n)).astype(np.float32)
    kind = {x: y for x, y in rule.items() if x != "slopes"}
    unseen = ~np.stack([oracle.visible(q_pos[0], pos[0, g], **kind).any(0) for g in range(2)])
    assert (unseen.reshape(2, -1, 32).mean(2) > 0).all() and (unseen.reshape(2, -1, 32).mean(2) < 1).all()
    for g in range(2):
        s = qd[0, ~padding, 4 * g:4 * g + 4].reshape(-1, 64).astype(np.float64) @ k[0, g][~unseen[g]].T / 8
        assert (np.abs(s) < cap / 8).all()
    results = []
    for size in (0.01, 3.0, 1000.0, np.inf, np.nan):
        k[0][unseen] = stored(rng.choice([-1.0, 1.0], (int(unseen.sum()), 64)).astype(np.float32) * np.float32(size), dtype)
        qd[0, padding] = k[0][unseen][0]
        v[0][unseen] = stored(rng.standard_normal((int(unseen.sum()), 64)).astype(np.float32) * min(np.nan_to_num(size, nan=9.0), 1e30), dtype)
        try:
            vxl.debug_mixed_force(*plan)
            results.append(attend(qd, k, v, [n], dtype, 0.0, q_pos, pos, weight, softcap=cap, **rule))
        finally:
            vxl.debug_mixed_force()
        if size < 1:
            check_attend(results[0], qd, k, v, [n], dtype, 0.0, q_pos, pos, weight, softcap=cap, **rule)
    for got in results[1:]:
        assert all(np.array_equal(x, y) for x, y in zip(got, results[0]))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("t", [1, 4, 50])
@pytest.mark.parametrize("softcap", [2.0 ** 48, 2.0 ** 50, 2.0 ** 55])
def test_caps_far_above_large_logits(softcap, t, dtype):
    """Products of 2^45, whose third power is no number of 32 bits: the one row of such a logit has all the weight, one of its negative none.  The
    logit is off by the roundings of the scale, its unit and their product, of the series' two last steps, and of the unit that it is given in; from 2^-6 of such a cap
    on bf16 sets have the exponential, off by 2^-22 softcap."""
    n = 200
    rng = np.random.default_rng(t)
    k, v, _ = sets(rng, 1, 2, n, 64, dtype, [n])
    qd = np.full((1, t, 8, 64), 2.0 ** 20, np.float32)
    k[:] = 0.0
    k[0, 0, 77], k[0, 1, 130], k[0, :, 5] = 2.0 ** 19, 2.0 ** 19, -2.0 ** 19
    out, lse, weight = attend(qd, k, v, [n], dtype, 0.0, softcap=softcap)
    for h in range(8):
        assert (out[0, :, h] == v[0, h // 4, (77, 130)[h // 4]]).all()
    want = softcap * np.tanh(2.0 ** 42 / softcap)
    by_exp = dtype == "bf16" and 2.0 ** 42 / softcap >= 2.0 ** -6
    assert (np.abs(lse - want) <= 8 * E * want + by_exp * 2.0 ** -22 * softcap).all()
    one = np.zeros((2, n))
    one[0, 77] = one[1, 130] = 4 * t
    assert np.array_equal(weight[0], one)
