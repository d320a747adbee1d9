"""Pins of the oracle of rotary positions and growing mixed sets: closed forms, library special cases, brute force."""
import numpy as np
import pytest
import torch

import oracle


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_by_hand(interleaved):
    x = np.arange(1.0, 7.0)[None]                                  # pairs (1, 3), (2, 4), or (1, 2), (3, 4); 5, 6 stay
    y = oracle.rotate(x, [2], [np.pi / 4, np.pi / 2], interleaved, 0.5)
    pairs = [(0, 1), (2, 3)] if interleaved else [(0, 2), (1, 3)]
    want = x[0].copy()
    for (a, b), turn in zip(pairs, ("quarter", "half")):
        want[a], want[b] = (-x[0, b] / 2, x[0, a] / 2) if turn == "quarter" else (-x[0, a] / 2, -x[0, b] / 2)
    assert np.allclose(y[0], want, atol=1e-15)


def test_rotation_is_relative_and_its_transpose_is_its_gradient():
    rng = np.random.default_rng(1)
    freqs = 1e4 ** (-np.arange(4) / 4)
    q, k = rng.standard_normal((2, 1, 12))
    at = lambda x, p: oracle.rotate(x, [p], freqs)                 # noqa: E731
    assert np.allclose((at(q, 17) * at(k, 5)).sum(), (at(q, 112) * at(k, 100)).sum(), atol=1e-12)
    g = rng.standard_normal((1, 12))
    back = oracle.rotate(g, [9], freqs, magnitude=1.5, transpose=True)
    for i in range(12):
        step = np.zeros((1, 12))
        step[0, i] = 1e-3
        diff = (g * (oracle.rotate(q + step, [9], freqs, magnitude=1.5) - oracle.rotate(q - step, [9], freqs, magnitude=1.5))).sum() / 2e-3
        assert abs(diff - back[0, i]) < 1e-9


def test_attention_without_a_rule_is_the_librarys():
    rng = np.random.default_rng(2)
    q, k, v = rng.standard_normal((2, 3, 6, 8)), rng.standard_normal((2, 2, 11, 8)), rng.standard_normal((2, 2, 11, 8))
    out, lse, w = oracle.attend_mixed(q, k, v, [11, 4])
    for b, n in enumerate((11, 4)):
        want = torch.nn.functional.scaled_dot_product_attention(*(torch.from_numpy(x) for x in (
            q[b].transpose(1, 0, 2), np.repeat(k[b, :, :n], 3, 0), np.repeat(v[b, :, :n], 3, 0)))).numpy()
        assert np.allclose(out[b], want.transpose(1, 0, 2), atol=1e-12)
        assert np.allclose(w[b].sum(1), 9) and (w[b, :, n:] == 0).all()          # 3 tokens of 3 heads give 1 each


def test_visibility_by_hand():
    see = oracle.visible([5, -1, 9], [0, 3, 5, 6, -1, 9], causal=True, window=4, n_always=1)
    assert see.tolist() == [[True, True, True, False, False, False], [False] * 6, [True, False, False, True, False, True]]
    assert oracle.visible([5], [0, 7, -1]).tolist() == [[True, True, False]]


def test_empty_and_broken_rows():
    q, k, v = np.ones((1, 2, 1, 4)), np.ones((1, 1, 3, 4)), np.ones((1, 1, 3, 4))
    k[0, 0, 1], v[0, 0, 1] = np.nan, np.inf
    out, lse, w = oracle.attend_mixed(q, k, v, [3], q_pos=np.array([[0, 1]]), row_pos=np.array([[[0, 1, 7]]]), causal=True)
    assert (out[0, 0] == 1).all() and lse[0, 0, 0] == 2 and np.isnan(out[0, 1]).all() and np.isnan(lse[0, 1, 0])
    assert np.isnan(w[0, 0, :2]).all() and w[0, 0, 2] == 0
    out, lse, w = oracle.attend_mixed(q, np.full_like(k, -np.inf), v, [3])
    assert (out == 0).all() and (lse == -np.inf).all() and (w == 0).all()


def test_eviction_by_hand():
    w = np.array([3.0, np.nan, 1.0, 5.0, 1.0, -0.0, 0.0, np.inf, 2.0], np.float32)
    pos = np.array([10, 11, 12, 13, 14, 15, 16, -1, 18])
    assert oracle.evict_rows(9, w, pos, 18, 4).tolist() == [0, 8, 2, 3]
    assert oracle.evict_rows(9, w, pos, 18, 8).tolist() == [0, 1, 2, 3, 4, 5, 6, 8]
    assert oracle.evict_rows(9, w, pos, 18, 3, n_first=12, n_recent=3).tolist() == [0, 1, 6]
    assert oracle.evict_rows(9, w, pos, 18, 6).tolist() == [0, 8, 2, 3, 4, 5]
    assert oracle.evict_rows(3, w, pos, 18, 9).tolist() == [0, 1, 2] and len(oracle.evict_rows(-4, w, pos, 18, 9)) == 0


def test_without_latest_rows_none_is_held_for_its_position():
    """n_recent = 0: neither without a newest position nor with one that rows lie behind."""
    w, pos = np.array([3.0, 1.0, 2.0, 5.0], np.float32), np.array([9, 11, 4, 6])
    for newest in (0, 5, 11):
        assert oracle.evict_rows(4, w, pos, newest, 2, n_first=0, n_recent=0).tolist() == [0, 3]
