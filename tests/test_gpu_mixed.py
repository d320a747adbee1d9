"""Rotary positions and growing mixed sets on the device, against the float64 oracle."""
import numpy as np
import pytest
import torch

import oracle
from paper_2506_19225_amd import vxl

from mixed_util import DTYPE, E, HALF_STEP, attend, check_attend, check_evict, evict, f32, i32, sets, stored, values

pytestmark = pytest.mark.gpu


# ---- rotary positions ----------------------------------------------------------------------------
def rotary_tol(x, y, freqs, interleaved, magnitude, dtype):
    """Of the two products of a pair: an angle rounded once (2^-25 of half a turn at most, 1.6 E), a sine and cosine off by an ulp, three
    products' roundings; then the result's."""
    half = len(freqs)
    size = np.abs(x).copy()
    first, second = (np.s_[..., 0:2 * half:2], np.s_[..., 1:2 * half:2]) if interleaved else (np.s_[..., :half], np.s_[..., half:2 * half])
    both = size[first] + size[second]
    size[first] = size[second] = both
    tol = 6.6 * E * abs(magnitude) * size + HALF_STEP[dtype] * np.abs(y)
    tol[..., 2 * half:] = 0.0
    return tol


def frequencies(rotary, base=1e6):
    return base ** (-2.0 * np.arange(rotary // 2) / rotary)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,d,n,rotary,interleaved,token_major,far", [
    (28, 4, 128, 33, 128, False, True, 0), (4, 2, 64, 577, 32, True, False, 10), (14, 2, 128, 65, 48, False, False, 900000),
    (8, 1, 64, 1, 64, True, True, 5), (4, 4, 64, 7, 16, False, True, 2 ** 31 - 100), (3, 1, 128, 19, 10, False, True, 77),
    (3, 1, 128, 19, 10, True, False, 77), (2, 2, 64, 5, 2, False, False, 3), (1, 1, 128, 300, 126, True, True, 1)])
@pytest.mark.parametrize("transpose", [False, True])
def test_rotation(dtype, hq, hkv, d, n, rotary, interleaved, token_major, far, transpose):
    rng = np.random.default_rng(n + rotary)
    q, k = values(rng, (hq, n, d), dtype), values(rng, (hkv, n, d), dtype)
    at = (far + rng.integers(0, 99, n)).astype(np.int64)
    at[0] = -3 if far else 0
    freqs, magnitude = frequencies(rotary), 1.0 if n == 33 else 1.1386
    order = (lambda x: np.ascontiguousarray(x.transpose(1, 0, 2))) if token_major else (lambda x: x)
    desc = vxl.make_desc(hq, hkv, d, dtype, token_major=token_major)
    dq, dk = vxl.to_device(order(q), dtype), vxl.to_device(order(k), dtype)
    r = vxl.Rotary(torch.from_numpy(freqs).cuda(), interleaved, magnitude)
    r = r.transposed() if transpose else r
    qo, ko = torch.full_like(dq, 9.0), torch.full_like(dk, 9.0)
    vxl.rotate(desc, r, i32(at), dq, dk, qo, ko)
    for x, y in ((q, qo), (k, ko)):
        want = oracle.rotate(x, at, freqs, interleaved, magnitude, transpose)
        got = y.double().cpu().numpy()
        got = got.transpose(1, 0, 2) if token_major else got
        assert (np.abs(got - want) <= rotary_tol(x, want, freqs, interleaved, magnitude, dtype)).all()
    alone = torch.full_like(dq, 9.0)
    vxl.rotate(desc, r, i32(at), dq, None, alone, None)
    assert torch.equal(alone, qo)
    vxl.rotate(desc, r, i32(at), dq, dk, dq, dk)                   # in place
    assert torch.equal(dq, qo) and torch.equal(dk, ko)


def test_rotation_of_a_fused_projection_in_place():
    """Queries, keys and values of a token side by side, as one projection writes them: the values stay."""
    rng = np.random.default_rng(4)
    hq, hkv, d, n = 6, 2, 64, 41
    x = values(rng, (n, hq + 2 * hkv, d), "bf16")
    dx = vxl.to_device(x, "bf16")
    desc = vxl.make_desc(hq, hkv, d, "bf16")
    desc.q_stride_head = desc.kv_stride_head = d
    desc.q_stride_tok = desc.kv_stride_tok = (hq + 2 * hkv) * d
    freqs = frequencies(d)
    dev = torch.from_numpy(freqs).cuda()
    import ctypes as C
    arg = vxl.RotaryArg(dev.data_ptr(), d, 0, 1.0, 0)
    at = i32(np.arange(n))
    kp = dx.data_ptr() + hq * d * 2
    st = vxl.lib().vxl_rotate(C.byref(desc), C.byref(arg), at.data_ptr(), n, dx.data_ptr(), kp, dx.data_ptr(), kp, vxl._stream(None))
    assert st == vxl.VXL_OK
    got = dx.double().cpu().numpy()
    want = oracle.rotate(x[:, :hq + hkv].transpose(1, 0, 2), np.arange(n), freqs).transpose(1, 0, 2)
    assert np.array_equal(got[:, hq + hkv:], x[:, hq + hkv:])
    tol = rotary_tol(x[:, :hq + hkv], want, freqs, False, 1.0, "bf16")
    assert (np.abs(got[:, :hq + hkv] - want) <= tol).all()


def test_gradient_of_a_rotation():
    """The transposed call is the gradient: against float64 autograd of the formula, and <g, R x> = <R^T g, x>."""
    rng = np.random.default_rng(6)
    hq, hkv, d, n, rotary = 4, 2, 64, 23, 48
    freqs = torch.from_numpy(frequencies(rotary)).cuda()
    desc = vxl.make_desc(hq, hkv, d, "f32")
    q, k, gq, gk = (f32(values(rng, (h, n, d), "f32")) for h in (hq, hkv, hq, hkv))
    at = i32(rng.integers(0, 5000, n))
    r = vxl.Rotary(freqs, magnitude=1.25)
    qo, ko, gqo, gko = (torch.empty_like(x) for x in (q, k, gq, gk))
    vxl.rotate(desc, r, at, q, k, qo, ko)
    vxl.rotate(desc, r.transposed(), at, gq, gk, gqo, gko)
    angle = at.double()[:, None] * freqs
    for x, g, gx, y in ((q, gq, gqo, qo), (k, gk, gko, ko)):
        leaf = x.double().requires_grad_()
        a, b, rest = leaf[..., :rotary // 2], leaf[..., rotary // 2:rotary], leaf[..., rotary:]
        cos, sin = 1.25 * torch.cos(angle), 1.25 * torch.sin(angle)
        torch.cat((a * cos - b * sin, a * sin + b * cos, rest), -1).backward(g.double())
        tol = rotary_tol(g.double().cpu().numpy(), leaf.grad.cpu().numpy(), frequencies(rotary), False, 1.25, "f32")
        assert (np.abs((gx.double() - leaf.grad).cpu().numpy()) <= tol).all()
        lhs, rhs = (g.double() * y.double()).sum(), (gx.double() * x.double()).sum()
        assert abs(float(lhs - rhs)) <= 16 * E * float((g.double().abs() * y.double().abs()).sum() + (gx.double() * x.double()).abs().sum())


# ---- append --------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,d,bsz,t,cap,lens,token_major", [
    (28, 4, 128, 1, 1, 40, [33], True), (4, 2, 64, 3, 5, 17, [17, 5, 9], True), (14, 2, 128, 2, 64, 300, [64, 299], False),
    (2, 2, 64, 4, 3, 8, [2, -5, 10, 0], True), (8, 1, 128, 1, 130, 130, [130], False)])
def test_append(dtype, hq, hkv, d, bsz, t, cap, lens, token_major):
    """Tokens whose row lies before the first or behind the last are not stored; their queries are rotated all the same."""
    rng = np.random.default_rng(t + cap)
    n = bsz * t
    q, k, v = (values(rng, (h, n, d), dtype) for h in (hq, hkv, hkv))
    at = rng.integers(0, 200000, (bsz, t))
    freqs = frequencies(d // 2)
    order = (lambda x: np.ascontiguousarray(x.transpose(1, 0, 2))) if token_major else (lambda x: x)
    desc = vxl.make_desc(hq, hkv, d, dtype, token_major=token_major)
    dq, dk, dv = (vxl.to_device(order(x), dtype) for x in (q, k, v))
    qd = torch.full((bsz, t, hq, d), 9.0, dtype=DTYPE[dtype], device="cuda")
    kmix, vmix = (torch.full((bsz, hkv, cap, d), 9.0, dtype=DTYPE[dtype], device="cuda") for _ in range(2))
    pos, weight = torch.full((bsz, hkv, cap), -7, dtype=torch.int32, device="cuda"), torch.full((bsz, hkv, cap), 9.0, device="cuda")
    r = vxl.Rotary(torch.from_numpy(freqs).cuda())
    vxl.mixed_append(desc, r, i32(at), dq, dk, dv, qd, kmix, vmix, i32(lens), pos, weight)
    turned = [oracle.rotate(x, at.reshape(-1), freqs) for x in (q, k)]
    tols = [rotary_tol(x, y, freqs, False, 1.0, dtype) for x, y in zip((q, k), turned)]
    split = lambda x: x.reshape(x.shape[0], bsz, t, d).transpose(1, 2, 0, 3)       # noqa: E731  [B, T, heads, D]
    assert (np.abs(qd.double().cpu().numpy() - split(turned[0])) <= split(tols[0])).all()
    want_k, want_v, tol = np.full((bsz, hkv, cap, d), 9.0), np.full((bsz, hkv, cap, d), 9.0), np.zeros((bsz, hkv, cap, d))
    want_pos, want_weight = np.full((bsz, hkv, cap), -7), np.full((bsz, hkv, cap), 9.0)
    for b in range(bsz):
        for i in range(t):
            row = lens[b] - t + i
            if 0 <= row < cap:
                want_k[b, :, row], tol[b, :, row], want_v[b, :, row] = split(turned[1])[b, i], split(tols[1])[b, i], split(v)[b, i]
                want_pos[b, :, row], want_weight[b, :, row] = at[b, i], 0
    assert (np.abs(kmix.double().cpu().numpy() - want_k) <= tol).all()
    assert np.array_equal(vmix.double().cpu().numpy(), want_v)
    assert np.array_equal(pos.cpu().numpy(), want_pos) and np.array_equal(weight.cpu().numpy(), want_weight)
    k2, v2, q2 = torch.full_like(kmix, 9.0), torch.full_like(vmix, 9.0), dq.reshape(bsz, t, hq, d) if token_major else torch.empty_like(qd)
    vxl.mixed_append(desc, r, i32(at), dq, dk, dv, q2, k2, v2, i32(lens))       # no positions, no weights; queries in place
    assert torch.equal(k2, kmix) and torch.equal(v2, vmix) and torch.equal(q2, qd)


def test_append_without_a_rotary_copies():
    rng = np.random.default_rng(3)
    desc = vxl.make_desc(6, 2, 64, "bf16", token_major=True)
    q, k, v = (vxl.to_device(values(rng, (4, h, 64), "bf16"), "bf16") for h in (6, 2, 2))
    qd, kmix = torch.zeros(2, 2, 6, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(2, 2, 5, 64, dtype=torch.bfloat16, device="cuda")
    vmix = torch.zeros_like(kmix)
    vxl.mixed_append(desc, None, i32([[1, 2], [3, 4]]), q, k, v, qd, kmix, vmix, i32([2, 5]))
    assert torch.equal(qd, q.view(2, 2, 6, 64))
    assert torch.equal(kmix[0, :, :2], k[:2].transpose(0, 1)) and torch.equal(vmix[1, :, 3:], v[2:].transpose(0, 1))


# ---- attention by position -----------------------------------------------------------------------
HEADS = [(28, 4, 128), (14, 2, 64), (8, 1, 128), (4, 4, 64), (16, 8, 128)]
RULES = {"plain": {}, "causal": dict(causal=True), "window": dict(causal=True, window=37), "band": dict(window=50), "prefix": dict(causal=True, window=9, n_always=40),
         "capped": dict(softcap=15.0, causal=True), "biased": dict(causal=True, slopes=True), "all": dict(softcap=30.0, causal=True, window=100, n_always=4, slopes=True)}


def case(seed, heads, bsz, t, cap, lens, dtype, rule, near=True):
    rng = np.random.default_rng(seed)
    hq, hkv, d = heads
    k, v, pos = sets(rng, bsz, hkv, cap, d, dtype, lens)
    qd = values(rng, (bsz, t, hq, d), dtype)
    q_pos = np.stack([rng.integers(0, 3 * max(int(n), 1), t) if near else 3 * max(int(n), 1) + np.arange(t) for n in lens]).astype(np.int32)
    weight = rng.random((bsz, hkv, cap)).astype(np.float32)
    rule = dict(rule)
    if rule.get("slopes"):
        rule["slopes"] = 2.0 ** (-8 * (np.arange(hq) + 1) / hq)
    return qd, k, v, q_pos, pos, weight, rule


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rule", RULES)
@pytest.mark.parametrize("heads,bsz,t,cap,lens", [
    (HEADS[0], 1, 1, 130, [129]), (HEADS[1], 3, 5, 77, [77, 1, 40]), (HEADS[2], 2, 9, 200, [65, 200]), (HEADS[3], 2, 3, 64, [64, 33]),
    (HEADS[4], 1, 2, 300, [257]), (HEADS[0], 1, 13, 450, [449])])
def test_attention(dtype, rule, heads, bsz, t, cap, lens):
    qd, k, v, q_pos, pos, weight, r = case(cap + t, heads, bsz, t, cap, lens, dtype, RULES[rule])
    got = attend(qd, k, v, lens, dtype, 0.0, q_pos, pos, weight, **r)
    check_attend(got, qd, k, v, lens, dtype, 0.0, q_pos, pos, weight, **r)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,bsz,t,cap,lens,rule", [
    (HEADS[0], 1, 150, 700, [699], "causal"), (HEADS[1], 2, 70, 1500, [1500, 801], "window"), (HEADS[2], 1, 40, 4100, [4099], "capped"),
    (HEADS[0], 2, 1, 5000, [4999, 2600], "causal"), (HEADS[3], 1, 300, 600, [599], "biased"), (HEADS[4], 1, 33, 2049, [2049], "all")])
def test_attention_over_longer_sets(dtype, heads, bsz, t, cap, lens, rule):
    qd, k, v, q_pos, pos, weight, r = case(7 * cap + t, heads, bsz, t, cap, lens, dtype, RULES[rule], near=rule in ("window", "all"))
    got = attend(qd, k, v, lens, dtype, 0.0, q_pos, pos, weight, **r)
    check_attend(got, qd, k, v, lens, dtype, 0.0, q_pos, pos, weight, **r)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("t", [1, 3, 40])
def test_attention_without_positions(dtype, t):
    """Every row of the set is seen: vxl_bilevel_decode's result (with a cap: of its own)."""
    qd, k, v, _, _, weight, _ = case(t, HEADS[0], 2, t, 333, [333, 90], dtype, {})
    for softcap in (0.0, 20.0):
        got = attend(qd, k, v, [333, 90], dtype, 0.11, None, None, weight, softcap=softcap)
        check_attend(got, qd, k, v, [333, 90], dtype, 0.11, None, None, weight, softcap=softcap)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("t", [1, 6, 50])
def test_lengths_and_padding(dtype, t):
    """Empty sets, an overflow report, a length past the buffers, one row; padding tokens, empty rows with NaN in them, a window
    that leaves nothing."""
    lens = [0, -17, 1, 500, 90]
    qd, k, v, q_pos, pos, weight, _ = case(t + 50, HEADS[1], 5, t, 90, lens, dtype, {})
    q_pos[3, ::2] = -1
    pos[3, :, 5:70:3] = -2
    k[3, :, 5:70:3], v[3, :, 5:70:3] = np.nan, np.inf
    q_pos[4] = 10 ** 9
    for rule in (dict(causal=True), dict(causal=True, window=5, n_always=2)):
        got = attend(qd, k, v, lens, dtype, 0.0, q_pos, pos, weight, **rule)
        check_attend(got, qd, k, v, lens, dtype, 0.0, q_pos, pos, weight, **rule)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("t", [1, 4, 50])
def test_numbers_that_are_none(dtype, t):
    """Infinities and NaN in keys and values: those that a token does not see do not matter to it, those that it sees do as in the formulas."""
    n = 150
    qd, k, v, _, pos, weight, _ = case(t + 90, HEADS[1], 1, t, n, [n], dtype, {})
    pos[:] = np.arange(n)
    q_pos = np.linspace(20, n - 10, t).astype(np.int32)[None]
    k[0, 0, 100], v[0, 0, 60, 3], v[0, 0, 61, 4], v[0, 0, 40, 5], v[0, 1, n - 1] = np.nan, np.inf, -np.inf, np.nan, np.nan
    v[0, 1, 70, 9], v[0, 1, 71, 9] = np.inf, -np.inf
    k[0, 1, n - 2] = np.inf
    rule = dict(causal=True)
    got = attend(qd, k, v, [n], dtype, 0.0, q_pos, pos, weight, **rule)
    check_attend(got, qd, k, v, [n], dtype, 0.0, q_pos, pos, weight, **rule)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_logits_of_minus_infinity_and_large_ones(dtype):
    qd, k, v, q_pos, pos, weight, _ = case(5, HEADS[3], 1, 3, 70, [70], dtype, {})
    qd[:] = np.abs(qd) + 0.1
    k[0, 0], k[0, 1, ::2] = -np.inf, -np.inf
    k[0, 2] *= 300
    qd, k = stored(qd, dtype), stored(k, dtype)                    # (what the device is given)
    got = attend(qd, k, v, [70], dtype, 0.0, None, None, weight)
    check_attend(got, qd, k, v, [70], dtype, 0.0, None, None, weight)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("t,n", [(1, 700), (50, 700)])
def test_weights_in_place_and_the_same_bits(dtype, t, n):
    qd, k, v, q_pos, pos, weight, _ = case(t, HEADS[0], 2, t, n, [n, n - 9], dtype, {})
    desc = vxl.make_desc(28, 4, 128, dtype)
    dq, dk, dv = (vxl.to_device(x, dtype) for x in (qd, k, v))
    rule, at, rows, lens = vxl.ScoreRule(causal=True, softcap=25.0), i32(q_pos), i32(pos), i32([n, n - 9])
    ws = vxl.alloc_workspace(vxl.workspace_bytes(vxl.OP_MIXED_ATTEND, None, desc, 2, t, n))
    results = []
    for _ in range(3):
        w, out, lse = f32(weight), torch.empty_like(dq), torch.empty(2, t, 28, device="cuda")
        vxl.mixed_attend(desc, rule, dq, at, dk, dv, lens, rows, out, lse, w, w, ws)
        results.append((out, lse, w))
    for r in results[1:]:
        assert all(torch.equal(x, y) for x, y in zip(r, results[0]))
    other, alone = torch.empty_like(results[0][2]), torch.empty_like(dq)
    other.copy_(f32(weight))
    vxl.mixed_attend(desc, rule, dq, at, dk, dv, lens, rows, alone, None, f32(weight), other, ws)
    assert torch.equal(other, results[0][2]) and torch.equal(alone, results[0][0])
    vxl.mixed_attend(desc, rule, dq, at, dk, dv, lens, rows, alone, None, None, None, ws)      # (no weights wanted)
    assert torch.equal(alone, results[0][0])
    none = torch.full_like(other, 5.0)
    vxl.mixed_attend(desc, rule, dq, at, dk, dv, lens, rows, alone, None, None, none, ws)      # (from 0)
    given = int((results[0][1][1] > -np.inf).sum())            # (a token and head that see a row give 1)
    assert abs(float(none[1, :, :n - 9].double().sum()) - given) < 1e-4 * given and (none[1, :, n - 9:] == 5).all()


# ---- eviction ------------------------------------------------------------------------------------
def evict_case(seed, bsz, hkv, cap, d, dtype, lens, kind):
    rng = np.random.default_rng(seed)
    k, v, pos = sets(rng, bsz, hkv, cap, d, dtype, lens)
    w = np.exp(rng.standard_normal((bsz, hkv, cap))).astype(np.float32)
    if kind == "ties":
        w = rng.integers(0, 3, w.shape).astype(np.float32) * np.where(rng.random(w.shape) < 0.5, -0.0, 1.0).astype(np.float32)
    elif kind == "equal":
        w[:] = 0.25
    elif kind == "special":
        w = rng.choice(np.array([np.nan, np.inf, -np.inf, -0.0, 0.0, 1e-45, -1e-45, 3e38, -3e38, -1.5, 2.0], np.float32), w.shape)
        pos[rng.random(pos.shape) < 0.1] = -1
    return k, v, w, pos


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("kind", ["random", "ties", "equal", "special"])
@pytest.mark.parametrize("dtype,bsz,hkv,cap,d,lens,keep,n_first,n_recent", [
    ("bf16", 1, 4, 300, 128, [300], 200, 4, 16), ("f32", 3, 2, 90, 64, [90, 0, 13], 13, 17, 0), ("bf16", 2, 1, 77, 64, [-4, 500], 76, 0, 0),
    ("f32", 1, 2, 65, 128, [65], 1, 0, 0), ("bf16", 2, 2, 64, 128, [64, 63], 0, 0, 3), ("bf16", 1, 2, 1200, 64, [1111], 900, 2000, 100),
    ("bf16", 1, 1, 1, 64, [1], 5, 0, 1), ("f32", 1, 3, 2500, 64, [2400], 64, 64, 64)])
def test_eviction(in_place, kind, dtype, bsz, hkv, cap, d, lens, keep, n_first, n_recent):
    k, v, w, pos = evict_case(cap + keep, bsz, hkv, cap, d, dtype, lens, kind)
    newest = np.array([pos[b].max() + b for b in range(bsz)])
    check_evict(k, v, lens, w, pos, newest, keep, n_first, n_recent, dtype, in_place=in_place)


@pytest.mark.parametrize("kind", ["random", "equal", "special"])
@pytest.mark.parametrize("cap,keep", [(20011, 5000), (20011, 20000), (40000, 17), (140000, 16384)])
def test_eviction_of_long_sets(kind, cap, keep):
    lens = [cap - 3, cap // 2]
    k, v, w, pos = evict_case(cap, 2, 2, cap, 64, "bf16", lens, kind)
    check_evict(k, v, lens, w, pos, np.array([3 * cap, 2 * cap]), keep, 5, 70, "bf16", out_cap=keep)
    check_evict(k, v, lens, w, pos, None, keep, 0, 0, "bf16", in_place=True)


# ---- together ------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_generation_over_a_set_that_grows_and_is_cut_back(dtype):
    """A prompt of 120 rows, then 60 tokens one at a time, the set cut to 100 rows whenever 140 are reached, all in place; compared after
    every token with the oracle run on the device's own state of before, and at the end with the attention weights of all steps."""
    rng = np.random.default_rng(11)
    hq, hkv, d, cap, n = 14, 2, 64, 144, 120
    desc = vxl.make_desc(hq, hkv, d, dtype, token_major=True)
    freqs = frequencies(d)
    rotary = vxl.Rotary(torch.from_numpy(freqs).cuda())
    rule = vxl.ScoreRule(causal=True, softcap=20.0, window=90, n_always=4)
    kind = dict(causal=True, softcap=20.0, window=90, n_always=4)
    kmix, vmix = (torch.full((1, hkv, cap, d), float("nan"), dtype=DTYPE[dtype], device="cuda") for _ in range(2))
    row_pos, weight = torch.full((1, hkv, cap), -1, dtype=torch.int32, device="cuda"), torch.full((1, hkv, cap), 3.0, device="cuda")
    ws_a = vxl.alloc_workspace(vxl.workspace_bytes(vxl.OP_MIXED_ATTEND, None, desc, 1, n, cap))
    ws_e = vxl.alloc_workspace(vxl.workspace_bytes(vxl.OP_MIXED_EVICT, None, desc, 1, 0, cap))
    length, seen, cuts = 0, 0, 0
    for step in range(61):
        t = n if step == 0 else 1
        q, k, v = (vxl.to_device(values(rng, (t, h, d), dtype), dtype) for h in (hq, hkv, hkv))
        length += t
        lens, at = i32([length]), i32(np.arange(seen, seen + t)[None])
        qd, out, lse = torch.empty(1, t, hq, d, dtype=DTYPE[dtype], device="cuda"), torch.empty(1, t, hq, d, dtype=DTYPE[dtype], device="cuda"), \
            torch.empty(1, t, hq, device="cuda")
        vxl.mixed_append(desc, rotary, at, q, k, v, qd, kmix, vmix, lens, row_pos, weight)
        before = weight.cpu().numpy().copy()
        vxl.mixed_attend(desc, rule, qd, at, kmix, vmix, lens, row_pos, out, lse, weight, weight, ws_a)
        if step % 7 < 2:
            host = [x.float().cpu().numpy() for x in (qd, kmix, vmix)]
            got = tuple(x.double().cpu().numpy() for x in (out, lse, weight))
            check_attend(got, *host, [length], dtype, 0.0, at.cpu().numpy(), row_pos.cpu().numpy(), before, **kind)
        seen += t
        if length == 140:
            want = [oracle.evict_rows(length, weight[0, g].cpu().numpy(), row_pos[0, g].cpu().numpy(), seen - 1, 100, 4, 16) for g in range(hkv)]
            old = row_pos.cpu().numpy().copy()
            vxl.mixed_evict(desc, kmix, vmix, lens, weight, row_pos, i32([seen - 1]), 100, 4, 16, kmix, vmix, weight, row_pos, lens, ws_e)
            length = int(lens)
            assert length == 100
            for g in range(hkv):
                assert np.array_equal(row_pos[0, g, :100].cpu().numpy(), old[0, g, want[g]])
                assert set(range(4)) <= set(row_pos[0, g, :100].tolist()) and set(range(seen - 16, seen)) <= set(row_pos[0, g, :100].tolist())
            cuts += 1
    assert cuts == 2 and seen == 180
