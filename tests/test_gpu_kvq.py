"""The quantised KV cache on the device: codes and values bit for bit against the oracle's definition, gathered sets exactly,
the decode in place against float64 attention over the values that the cache stands for, with bounds counted from the
roundings that the path makes."""
import ctypes as C

import numpy as np
import pytest
import torch

import oracle
from paper_2506_19225_amd import vxl, workloads as wl

from gpu_util import gpu_decode, kept_rows, make_layout
from kvq_util import FORMATS, device_cache, pack, quantised, random_rows

pytestmark = pytest.mark.gpu
DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}


def same_bits(a, b):
    return a.dtype == b.dtype and a.shape == b.shape and torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


# ---- write and read ------------------------------------------------------------------------------
def write_and_read(k, v, dtype, fmt, token_major=False, first=0, capacity=None):
    """k, v float32 [Hkv, n, D]: written at `first`, compared with the oracle, read back and compared again."""
    hkv, n, d = k.shape
    capacity = first + n if capacity is None else capacity
    desc = vxl.make_desc(hkv, hkv, d, dtype, token_major=token_major)
    cache = vxl.KvqCache(desc, fmt, capacity)
    cache.rows.fill_(0x5a)
    cache.scales.fill_(0xa5)
    order = (lambda x: x.transpose(1, 0, 2)) if token_major else (lambda x: x)
    dk, dv = vxl.to_device(order(k), dtype), vxl.to_device(order(v), dtype)
    vxl.kvq_write(desc, dk, dv, cache, first)
    rows, scales, wk, wv = quantised(k, v, fmt)
    want_rows, want_scales = np.full(cache.rows.shape, 0x5a, np.uint8), np.full(cache.scales.shape, 0xa5, np.uint8)
    want_rows[:, first:first + n], want_scales[:, first:first + n] = rows, scales
    got_rows, got_scales = cache.rows.cpu().numpy(), cache.scales.cpu().numpy()
    assert np.array_equal(got_scales, want_scales)
    assert np.array_equal(got_rows, want_rows)
    k2, v2 = torch.full_like(dk, 3.0), torch.full_like(dv, 3.0)
    vxl.kvq_read(desc, cache, k2, v2, first)
    for got, want in ((k2, wk), (v2, wv)):
        got, want = got.double().cpu().numpy(), order(want)
        assert np.array_equal(np.isnan(got), np.isnan(want))
        assert np.array_equal(got[~np.isnan(want)], want[~np.isnan(want)])
        assert np.array_equal(np.signbit(got[~np.isnan(want)]), np.signbit(want[~np.isnan(want)]))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hkv,n,d,token_major,first,spare", [
    (4, 1, 128, True, 37, 5), (2, 3, 64, False, 0, 0), (1, 130, 128, False, 1, 0), (3, 67, 64, True, 9, 1), (8, 33, 128, True, 0, 3)])
def test_rows_written_and_read(fmt, dtype, hkv, n, d, token_major, first, spare):
    rng = np.random.default_rng(n * d + hkv)
    k, v = random_rows(rng, (hkv, n, d), dtype), random_rows(rng, (hkv, n, d), dtype)
    write_and_read(k, v, dtype, fmt, token_major, first, first + n + spare)


@pytest.mark.parametrize("fmt", FORMATS)
def test_every_bf16_number(fmt):
    """All 65,536 bit patterns: in blocks of 32 neighbours, and each beside a larger one, so that every number is the largest of
    a block once and is rounded against other scales too."""
    bits = np.arange(65536, dtype=np.uint32)
    x = (bits << 16).view(np.float32)
    with np.errstate(invalid="ignore"):
        y = np.where(np.isfinite(x), x, 1.0).astype(np.float32).reshape(-1, 32)
    mixed = y[np.argsort((bits * 40503) % 65536).reshape(-1, 32) // 32, np.arange(32)]
    mixed[:, 0] = np.abs(mixed[:, 0])
    near = np.concatenate([y.reshape(-1, 64), (y * np.float32(0.5)).reshape(-1, 64)], 0)
    near[:, 5] = wl.round_to_bf16((near[:, 6].astype(np.float64) * 5).clip(-2.0e38, 2.0e38).astype(np.float32))
    for rows in (x.reshape(1, -1, 64), mixed.reshape(1, -1, 64), wl.round_to_bf16(near)[None]):
        write_and_read(rows, rows[:, ::-1].copy(), "bf16", fmt)


@pytest.mark.parametrize("fmt", FORMATS)
def test_fp32_numbers_at_the_borders(fmt):
    """Ties, numbers a step to either side of them, the bound of a block's scale, subnormals, the largest, zeros, NaN."""
    numbers = oracle.kvq_numbers(fmt)
    ties = np.concatenate([numbers, (numbers[1:] + numbers[:-1]) / 2]).astype(np.float32)
    around = np.concatenate([ties, np.nextafter(ties, np.float32(9e9)), np.nextafter(ties, np.float32(-9e9))])
    around = np.concatenate([around, -around])
    rng = np.random.default_rng(8)
    blocks = []
    for e in (-149, -126, -112, -110, -60, -1, 0, 40, 110):
        for top in (numbers[-1], 1.75 * 2.0 ** np.floor(np.log2(numbers[-1]) - 1), 3.5):
            row = rng.choice(around, size=128).astype(np.float64) * 2.0 ** e
            row[rng.integers(0, 4) * 32:][:32][3] = top * 2.0 ** e
            blocks.append(row.astype(np.float32))
    special = np.zeros((8, 128), np.float32)
    special[0, 3:5] = np.inf, 1.0
    special[1, 40] = np.nan
    special[2, 70] = np.float32(1.75 * 2.0 ** 127)
    special[3, 70] = np.nextafter(np.float32(1.75 * 2.0 ** 127), np.float32(0))
    special[4] = -0.0
    special[5, ::7] = 1.0e-45
    special[6, 100] = np.finfo(np.float32).max
    x = np.concatenate([np.stack(blocks), special])[None]
    write_and_read(x, x[:, ::-1].copy(), "f32", fmt)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_part_of_a_longer_tensor(dtype):
    """Rows 11..50 of a head-major tensor, by its strides, into rows 100..139; then one row, and none."""
    rng = np.random.default_rng(77)
    hkv, n, d = 3, 90, 64
    k, v = random_rows(rng, (hkv, n, d), dtype), random_rows(rng, (hkv, n, d), dtype)
    desc = vxl.make_desc(hkv, hkv, d, dtype)
    desc.q_stride_head = desc.kv_stride_head = n * d
    desc.q_stride_tok = desc.kv_stride_tok = d
    cache = vxl.KvqCache(desc, "fp4", 150)
    cache.rows.zero_(), cache.scales.zero_()
    dk, dv = vxl.to_device(k, dtype), vxl.to_device(v, dtype)
    at = lambda t, r: t.view(-1)[r * d:]                                        # noqa: E731
    vxl.kvq_write(desc, at(dk, 11), at(dv, 11), cache, 100, 40)
    vxl.kvq_write(desc, at(dk, 89), at(dv, 89), cache, 149, 1)
    vxl.kvq_write(desc, at(dk, 0), at(dv, 0), cache, 0, 0)
    rows, scales, wk, _ = quantised(k, v, "fp4")
    got = cache.rows.cpu().numpy()
    assert np.array_equal(got[:, 100:140], rows[:, 11:51]) and np.array_equal(got[:, 149], rows[:, 89])
    assert not got[:, :100].any() and not got[:, 140:149].any()
    assert np.array_equal(cache.scales.cpu().numpy()[:, 100:140], scales[:, 11:51])
    for start, count in ((51, 40), (89, 2), (0, 91)):                           # rows that the tensors do not hold
        with pytest.raises(vxl.VxlError) as e:
            vxl.kvq_write(desc, at(dk, start), at(dv, start), cache, 0, count)
        assert e.value.status == vxl.VXL_ERR_INVALID_ARG
        with pytest.raises(vxl.VxlError) as e:
            vxl.kvq_read(desc, cache, at(dk, start), at(dv, start), 0, count)
        assert e.value.status == vxl.VXL_ERR_INVALID_ARG
    back = torch.zeros_like(dk)
    vxl.kvq_read(desc, cache, at(back, 20), at(torch.zeros_like(dk), 20), 100, 40)
    got = back.double().cpu().numpy()
    assert np.array_equal(got[:, 20:60], wk[:, 11:51]) and not got[:, :20].any() and not got[:, 60:].any()


# ---- prompts -------------------------------------------------------------------------------------
def prompt(rng, dtype, hkv, d, fmt, lay, pooled):
    """Plain rows of a prompt, its caches on the device and the values that they stand for (dense, sparse)."""
    k, v = random_rows(rng, (hkv, lay.n_tokens, d), dtype), random_rows(rng, (hkv, lay.n_tokens, d), dtype)
    desc = vxl.make_desc(hkv, hkv, d, dtype)
    rows, scales, wk, wv = quantised(k, v, fmt)
    cache = device_cache(desc, fmt, rows, scales, spare=3)
    if not pooled:
        return cache, None, (wk, wv), None
    ksp, vsp = (random_rows(rng, (hkv, max(int(lay.sparse_offsets[-1]), 1), d), dtype) for _ in range(2))
    rows, scales, wks, wvs = quantised(ksp, vsp, fmt)
    return cache, device_cache(desc, fmt, rows, scales, spare=2), (wk, wv), (wks, wvs)


def mixed(values, sparse, masks, lay, l_cap):
    args = lay.n_prefix, lay.chunk_bounds, lay.sparse_offsets
    if sparse is None:
        return oracle.gather_bilevel(*values, masks, *args, lay.sparse_idx, l_cap=l_cap)
    return oracle.gather_bilevel_pooled(*values, *sparse, masks, *args, l_cap=l_cap)


def some_masks(rng, bsz, n_chunks):
    masks = rng.integers(0, 2, size=(bsz, n_chunks)).astype(np.uint8)
    masks[0] = 0
    if bsz > 1:
        masks[1] = 1
    return masks


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("pooled", [False, True])
@pytest.mark.parametrize("dtype,hkv,d,bsz,chunks,prefix", [
    ("bf16", 4, 128, 3, 11, 17), ("f32", 1, 64, 2, 5, 0), ("bf16", 3, 64, 1, 1, 300), ("f32", 2, 128, 1, 40, 5),
    ("bf16", 2, 128, 2, 0, 33), ("bf16", 8, 64, 9, 130, 1)])
def test_gather(fmt, pooled, dtype, hkv, d, bsz, chunks, prefix):
    rng = np.random.default_rng(d + 13 * chunks)
    lay = wl.random_layout(rng, prefix, chunks, 1, 60) if chunks else wl.layout_from_lists(prefix, [], [])
    cache, sparse, values, sparse_values = prompt(rng, dtype, hkv, d, fmt, lay, pooled)
    masks = some_masks(rng, bsz, max(chunks, 1))[:, :chunks]
    l_cap = lay.n_tokens + 7
    wk, wv, wlen, wsrc = mixed(values, sparse_values, masks, lay, l_cap)
    desc = vxl.make_desc(hkv, hkv, d, dtype)
    kmix = torch.full((bsz, hkv, l_cap, d), 7.0, dtype=DTYPE[dtype], device="cuda")
    vmix = torch.full_like(kmix, 7.0)
    lens, src = torch.full((bsz,), -1, dtype=torch.int32, device="cuda"), torch.full((bsz, l_cap), -5, dtype=torch.int32, device="cuda")
    dm = torch.from_numpy(np.ascontiguousarray(masks)).cuda() if chunks else None
    gl = make_layout(lay)
    for want_src in (True, False):
        kmix.fill_(7.0), vmix.fill_(7.0), lens.fill_(-1)
        vxl.gather_bilevel_kvq(gl, desc, cache, sparse, dm, kmix, vmix, lens, src if want_src else None)
        assert np.array_equal(lens.cpu().numpy(), wlen)
        for b in range(bsz):
            n = int(wlen[b])
            for got, want in ((kmix, wk), (vmix, wv)):
                got = got[b].double().cpu().numpy()
                assert np.array_equal(got[:, :n], want[b, :, :n]) and (got[:, n:] == 7.0).all()
            assert np.array_equal(src[b, :n].cpu().numpy(), wsrc[b, :n]) and (src[b, n:] == -5).all()


@pytest.mark.parametrize("fmt,pooled,dtype,hkv,d,bsz,chunks,length,groups", [
    ("fp4", False, "bf16", 4, 128, 1, 640, 28, 2), ("fp8", True, "bf16", 4, 128, 1, 640, 28, 2), ("fp8", False, "bf16", 2, 64, 3, 1500, 33, 3),
    ("fp4", True, "f32", 1, 64, 1, 1600, 20, 3), ("fp8", False, "f32", 3, 128, 1, 3000, 12, 6), ("fp4", True, "bf16", 1, 64, 2, 3500, 40, 7)])
def test_gather_of_several_passes_per_block(fmt, pooled, dtype, hkv, d, bsz, chunks, length, groups):
    """Sets of so many chunks that a block takes several passes over its rows (`groups`, as the launch counts them)."""
    rng = np.random.default_rng(chunks + d)
    lay = wl.random_layout(rng, 37, chunks, 1, 2 * length)
    l_cap = lay.n_tokens + 5
    rows = 256 // (d // (8 if dtype == "bf16" else 4))
    assert max(1, min(8, 1 + chunks // 512, -(-l_cap // rows) * bsz // 512)) == groups
    cache, sparse, values, sparse_values = prompt(rng, dtype, hkv, d, fmt, lay, pooled)
    masks = some_masks(rng, bsz, chunks)
    masks[0] = rng.integers(0, 3, size=chunks) > 0
    wk, wv, wlen, wsrc = mixed(values, sparse_values, masks, lay, l_cap)
    desc = vxl.make_desc(hkv, hkv, d, dtype)
    kmix = torch.full((bsz, hkv, l_cap, d), 7.0, dtype=DTYPE[dtype], device="cuda")
    vmix = torch.full_like(kmix, 7.0)
    lens, src = torch.full((bsz,), -1, dtype=torch.int32, device="cuda"), torch.full((bsz, l_cap), -5, dtype=torch.int32, device="cuda")
    vxl.gather_bilevel_kvq(make_layout(lay), desc, cache, sparse, torch.from_numpy(masks).cuda(), kmix, vmix, lens, src)
    assert np.array_equal(lens.cpu().numpy(), wlen)
    for b in range(bsz):
        n = int(wlen[b])
        for got, want in ((kmix, wk), (vmix, wv)):
            got = got[b].double().cpu().numpy()
            assert np.array_equal(got[:, :n], want[b, :, :n]) and (got[:, n:] == 7.0).all()
        assert np.array_equal(src[b, :n].cpu().numpy(), wsrc[b, :n]) and (src[b, n:] == -5).all()


@pytest.mark.parametrize("fmt,pooled,dtype,hkv,d,bsz", [
    ("fp4", False, "bf16", 4, 128, 8), ("fp8", True, "bf16", 4, 128, 8), ("fp4", True, "bf16", 2, 64, 20), ("fp8", False, "bf16", 3, 64, 20),
    ("fp4", False, "f32", 1, 128, 16), ("fp8", True, "f32", 4, 64, 9)])
def test_gather_past_the_caches(fmt, pooled, dtype, hkv, d, bsz):
    """Sets of 160 MB and more, whose rows are stored past the caches, beside smaller ones, which are not: every row is the one that
    the cache reads back as."""
    rng = np.random.default_rng(d + hkv)
    elem = 2 if dtype == "bf16" else 4
    row = 2 * bsz * hkv * d * elem                                  # bytes of one row of all sets
    tokens = (160 << 20) // row + 3000
    lens = [int(x) for x in np.diff(np.concatenate([[0], np.sort(rng.choice(np.arange(1, tokens), size=40, replace=False)), [tokens]]))]
    starts = 21 + np.cumsum([0] + lens[:-1])
    lay = wl.layout_from_lists(21, lens, [np.sort(rng.choice(n, size=n // 5, replace=False)).astype(np.int32) + s for n, s in zip(lens, starts)])
    desc, n, n_sparse = vxl.make_desc(hkv, hkv, d, dtype), lay.n_tokens, len(lay.sparse_idx)
    gen = torch.Generator("cuda").manual_seed(hkv)
    values = []
    caches = [vxl.KvqCache(desc, fmt, size) for size in ([n, n_sparse] if pooled else [n])]
    for c in caches:
        k, v = (torch.randn(hkv, c.capacity, d, generator=gen, device="cuda").to(DTYPE[dtype]) for _ in range(2))
        vxl.kvq_write(desc, k, v, c)
        vxl.kvq_read(desc, c, k, v)
        values.append((k, v))
    masks = some_masks(rng, bsz, lay.n_chunks)
    masks[2:] |= rng.integers(0, 50, size=masks[2:].shape) > 0
    kmix = torch.full((bsz, hkv, n + 9, d), 7.0, dtype=DTYPE[dtype], device="cuda")
    vmix, lens_got = torch.full_like(kmix, 7.0), torch.zeros(bsz, dtype=torch.int32, device="cuda")
    vxl.gather_bilevel_kvq(make_layout(lay), desc, caches[0], caches[1] if pooled else None, torch.from_numpy(masks).cuda(), kmix, vmix, lens_got)
    past = []
    for b in range(bsz):
        src = [np.arange(21)]
        for c in range(lay.n_chunks):
            dense, kept = np.arange(lay.chunk_bounds[c], lay.chunk_bounds[c + 1]), np.arange(lay.sparse_offsets[c], lay.sparse_offsets[c + 1])
            src.append(dense if masks[b, c] else n + kept if pooled else lay.sparse_idx[kept])
        src = torch.from_numpy(np.concatenate(src).astype(np.int64)).cuda()
        past.append(row * len(src) > 160 << 20)
        assert int(lens_got[b]) == len(src)
        for got, i in ((kmix, 0), (vmix, 1)):
            want = torch.cat([x[i] for x in values], 1)[:, src]
            assert same_bits(got[b, :, :len(src)], want) and (got[b, :, len(src):] == 7.0).all()
    assert any(past) and not all(past)


def test_gather_reports_an_overflow():
    rng = np.random.default_rng(3)
    lay = wl.random_layout(rng, 9, 6, 20, 50)
    cache, _, values, _ = prompt(rng, "bf16", 2, 64, "fp4", lay, False)
    masks = np.ones((2, lay.n_chunks), np.uint8)
    masks[0] = 0
    few = 9 + len(lay.sparse_idx)
    desc, gl = vxl.make_desc(2, 2, 64, "bf16"), make_layout(lay)
    kmix = torch.full((2, 2, few, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    vmix, lens = torch.full_like(kmix, 7.0), torch.zeros(2, dtype=torch.int32, device="cuda")
    vxl.gather_bilevel_kvq(gl, desc, cache, None, torch.from_numpy(masks).cuda(), kmix, vmix, lens)
    assert lens.tolist() == [few, -lay.n_tokens] and (kmix[1] == 7.0).all() and not (kmix[0] == 7.0).all()
    qd = torch.ones(2, 1, 2, 64, dtype=torch.bfloat16, device="cuda")
    out, lse = torch.full_like(qd, 5.0), torch.zeros(2, 1, 2, device="cuda")
    ws = vxl.alloc_workspace(vxl.workspace_bytes(vxl.OP_DECODE_KVQ, gl, desc, 2, 1, few))
    vxl.bilevel_decode_kvq(gl, desc, qd, cache, None, torch.from_numpy(masks).cuda(), few, out, lse, lens, ws)
    assert lens.tolist() == [few, -lay.n_tokens] and not out[1].any() and (lse[1] == -np.inf).all() and out[0].any()


# ---- decode --------------------------------------------------------------------------------------
def attention(qd, k, v, n, scale):
    """float64 (O, LSE) [T, Hq, ...] over n rows, and sum p |v| and the largest sum |q k| and |logit| of a row."""
    t, hq, d = qd.shape
    g = hq // k.shape[0]
    o, lse, av, aq = (np.zeros(s) for s in ((t, hq, d), (t, hq), (t, hq, d), (t, hq)))
    for h in range(hq):
        kk, vv = k[h // g, :n], v[h // g, :n]
        s = scale * (qd[:, h].astype(np.float64) @ kk.T)
        m = s.max(1, keepdims=True)
        e = np.exp(s - m)
        p = e / e.sum(1, keepdims=True)
        o[:, h], av[:, h] = p @ vv, p @ np.abs(vv)
        lse[:, h] = (m + np.log(e.sum(1, keepdims=True)))[:, 0]
        aq[:, h] = scale * (np.abs(qd[:, h].astype(np.float64)) @ np.abs(kk).T).max(1)
    return o, lse, av, aq


def check_decode(rng, dtype, fmt, hq, hkv, d, t, lay, masks, pooled, q_gain=1.0, scale=0.0, l_cap=None):
    cache, sparse, values, sparse_values = prompt(rng, dtype, hkv, d, fmt, lay, pooled)
    bsz = masks.shape[0]
    l_cap = lay.n_tokens if l_cap is None else l_cap
    qd = (rng.standard_normal((bsz, t, hq, d)) * q_gain).astype(np.float32)
    qd = wl.round_to_bf16(qd) if dtype == "bf16" else qd
    wk, wv, wlen, _ = mixed(values, sparse_values, masks, lay, l_cap)
    gl, desc = make_layout(lay), vxl.make_desc(hq, hkv, d, dtype, scale)
    dq = vxl.to_device(qd, dtype)
    dm = torch.from_numpy(np.ascontiguousarray(masks)).cuda() if lay.n_chunks else None
    out, lse = torch.full_like(dq, np.nan), torch.full(dq.shape[:3], np.nan, device="cuda")
    lens = torch.full((bsz,), -77, dtype=torch.int32, device="cuda")
    ws = vxl.alloc_workspace(vxl.workspace_bytes(vxl.OP_DECODE_KVQ, gl, desc, bsz, t, l_cap))
    ws.fill_(0xff)
    vxl.bilevel_decode_kvq(gl, desc, dq, cache, sparse, dm, l_cap, out, lse, lens, ws)
    assert np.array_equal(lens.cpu().numpy(), wlen)
    again, only = torch.full_like(dq, np.nan), torch.full_like(dq, np.nan)
    vxl.bilevel_decode_kvq(gl, desc, dq, cache, sparse, dm, l_cap, again, None, lens, ws, map_ready=True)
    assert same_bits(out, again)                                    # the map reused, no LSE, no lengths asked for
    vxl.bilevel_decode_kvq(gl, desc, dq, cache, sparse, dm, l_cap, only, None, None, ws)
    assert same_bits(out, only)
    got, got_lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    scale = scale or d ** -0.5
    for b in range(bsz):
        n = int(wlen[b])
        if n == 0:
            assert not got[b].any() and (got_lse[b] == -np.inf).all()
            continue
        o, wlse, av, aq = attention(qd[b], wk[b], wv[b], n, scale)
        # A logit: fp32 sums of at most 12 steps of 32 products, its product with log2(e) and the subtraction from the
        # reference, all of magnitude up to sum |q k|; an exponential 2 steps.  The sum over n keys in lanes, waves and
        # splits: n / 16 + 100 steps.  bf16: every weight and the result are rounded by half a step, 2^-8.  The weights are
        # exponentials against a reference that is a logit of the row, so that their sum is at least 1, and one below the
        # smallest normal number, 2^-126, is 0: up to n times 2^-126 |v| is missing from the result.
        logit = (44 + 4) * 2.0 ** -24 * aq * 1.5 + 2.0 ** -22
        sums = (n / 16 + 100) * 2.0 ** -24
        bound = av * (2 * logit + 2 * sums)[..., None] + n * 2.0 ** -126 * np.abs(wv[b, :, :n]).max()
        if dtype == "bf16":
            bound = bound + 1.01 * 2.0 ** -8 * (av + np.abs(o))
        assert (np.abs(got[b] - o) <= bound).all(), float((np.abs(got[b] - o) / bound).max())
        assert (np.abs(got_lse[b] - wlse) <= logit + sums + np.abs(wlse) * 2.0 ** -22).all()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("pooled", [False, True])
@pytest.mark.parametrize("dtype,hq,hkv,d,t,bsz", [
    ("bf16", 14, 2, 128, 1, 2), ("bf16", 14, 2, 64, 4, 1), ("bf16", 8, 1, 128, 2, 3), ("bf16", 4, 4, 64, 1, 9),
    ("bf16", 28, 4, 128, 5, 2), ("bf16", 14, 2, 128, 18, 2), ("bf16", 14, 2, 64, 40, 1), ("bf16", 28, 4, 128, 64, 1),
    ("bf16", 16, 1, 64, 1, 2), ("bf16", 17, 1, 128, 1, 2), ("f32", 2, 1, 64, 8, 1), ("f32", 14, 2, 128, 1, 2), ("f32", 6, 3, 64, 21, 3)])
def test_decode(fmt, pooled, dtype, hq, hkv, d, t, bsz):
    rng = np.random.default_rng(hq * 1000 + d + t)
    lay = wl.random_layout(rng, 17, 11, 1, 150)
    check_decode(rng, dtype, fmt, hq, hkv, d, t, lay, some_masks(rng, bsz, lay.n_chunks), pooled)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 130, 257])
def test_decode_of_short_sets(dtype, n):
    """A prefix alone, in buffers of its own size and in larger ones."""
    rng = np.random.default_rng(n)
    lay = wl.layout_from_lists(n, [], [])
    masks = np.zeros((1, 0), np.uint8)
    check_decode(rng, dtype, "fp4", 14, 2, 128, 1, lay, masks, False)
    check_decode(rng, dtype, "fp8", 4, 2, 64, 3, lay, masks, False, l_cap=n + 1000)


def test_decode_of_empty_sets():
    """No prefix and no kept rows: a query without dense chunks attends to nothing."""
    rng = np.random.default_rng(4)
    lay = wl.layout_from_lists(0, [40, 3, 90], [[], [], []])
    masks = np.array([[0, 0, 0], [0, 1, 0], [1, 1, 1]], np.uint8)
    for dtype in ("bf16", "f32"):
        for pooled in (False, True):
            check_decode(rng, dtype, "fp4", 6, 2, 64, 2, lay, masks, pooled)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype,d,t,tokens,bsz", [("bf16", 128, 1, 20000, 1), ("bf16", 64, 3, 30001, 2), ("f32", 128, 2, 9000, 1),
                                                  ("bf16", 128, 33, 9001, 2), ("bf16", 128, 1, 40000, 8)])
def test_decode_of_long_sets(fmt, dtype, d, t, tokens, bsz):
    """Many splits and many tiles per wave; two heads, values of wide range, logits of a few units and of dozens."""
    rng = np.random.default_rng(tokens + t)
    lens = [tokens // 7] * 7
    lay = wl.layout_from_lists(130, lens, [np.arange(130 + i * lens[0], 130 + (i + 1) * lens[0], 5) for i in range(7)])
    check_decode(rng, dtype, fmt, 4, 2, d, t, lay, some_masks(rng, bsz, 7), False, q_gain=0.02)
    if bsz < 8:
        check_decode(rng, dtype, fmt, 4, 1, d, t, lay, some_masks(rng, bsz, 7), True, q_gain=0.5)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("pooled", [False, True])
@pytest.mark.parametrize("hq,hkv,d,t,bsz,tokens,many", [
    (32, 4, 64, 129, 1, 6000, False), (32, 4, 128, 129, 1, 6000, False), (32, 4, 64, 129, 1, 16000, True), (32, 4, 128, 129, 1, 16000, True),
    (8, 4, 128, 200, 32, 700, True), (14, 2, 64, 129, 32, 700, True)])
def test_decode_of_many_rows(fmt, pooled, hq, hkv, d, t, bsz, tokens, many):
    """The kernel whose workgroups convert a tile for all their rows (`many`), and blocks of 32 rows over the same: row tiles and key
    tiles that are not full, several splits and one, splits without keys, queries without any."""
    rng = np.random.default_rng(tokens + d + t)
    cuts = np.sort(rng.choice(np.arange(1, tokens), size=6, replace=False))
    lens = np.diff(np.concatenate([[0], cuts, [tokens]]))
    starts = np.concatenate([[0], cuts])
    kept = [np.sort(rng.choice(n, size=n // 9, replace=False)).astype(np.int32) + s for n, s in zip(lens, starts)]
    lay = wl.layout_from_lists(0, [int(n) for n in lens], kept)
    masks = some_masks(rng, bsz, lay.n_chunks)
    masks[-1] = np.arange(lay.n_chunks) == 3
    desc = vxl.make_desc(hq, hkv, d, "bf16")
    kernel, n_split = vxl.debug_kvq_plan(desc, bsz, t, lay.n_tokens)
    assert kernel == (0 if many else 2) and (n_split > 1) == (bsz == 1)
    check_decode(rng, "bf16", fmt, hq, hkv, d, t, lay, masks, pooled, q_gain=0.1)


def test_plans():
    """The kernels and numbers of splits that these tests are meant to reach."""
    plan = lambda hq, hkv, d, dtype, b, t, cap: vxl.debug_kvq_plan(vxl.make_desc(hq, hkv, d, dtype), b, t, cap)  # noqa: E731
    assert plan(14, 2, 128, "bf16", 2, 1, 900)[0] == 1 and plan(14, 2, 128, "bf16", 2, 1, 900)[1] > 1
    assert plan(14, 2, 128, "bf16", 1, 1, 128) == (1, 1)
    assert plan(14, 2, 128, "bf16", 2, 18, 900)[0] == plan(28, 4, 128, "bf16", 1, 64, 900)[0] == 2
    assert plan(6, 3, 64, "f32", 3, 21, 900)[0] == 1
    assert plan(4, 2, 128, "bf16", 1, 1, 20000)[1] > 64
    assert plan(4, 1, 64, "bf16", 2, 3, 30001)[1] > 32


def test_decode_with_a_scale_of_its_own_and_steep_logits():
    rng = np.random.default_rng(21)
    lay = wl.random_layout(rng, 30, 5, 50, 200)
    for dtype in ("bf16", "f32"):
        check_decode(rng, dtype, "fp8", 6, 2, 64, 2, lay, some_masks(rng, 2, 5), False, scale=0.9)
        check_decode(rng, dtype, "fp4", 6, 2, 128, 1, lay, some_masks(rng, 2, 5), False, scale=1e-3)
        check_decode(rng, dtype, "fp4", 6, 2, 128, 1, lay, some_masks(rng, 2, 5), False, q_gain=20.0)


def test_many_chunks():
    """More chunks than a block's table of first rows holds."""
    rng = np.random.default_rng(6)
    lay = wl.random_layout(rng, 3, 4000, 1, 3)
    masks = some_masks(rng, 3, 4000)
    check_decode(rng, "bf16", "fp4", 4, 1, 64, 1, lay, masks, True)
    cache, _, values, _ = prompt(rng, "bf16", 1, 64, "fp8", lay, False)
    wk, wv, wlen, _ = mixed(values, None, masks, lay, lay.n_tokens)
    kmix = torch.zeros(3, 1, lay.n_tokens, 64, dtype=torch.bfloat16, device="cuda")
    vmix, lens = torch.zeros_like(kmix), torch.zeros(3, dtype=torch.int32, device="cuda")
    vxl.gather_bilevel_kvq(make_layout(lay), vxl.make_desc(1, 1, 64, "bf16"), cache, None, torch.from_numpy(masks).cuda(), kmix, vmix, lens)
    assert np.array_equal(lens.cpu().numpy(), wlen)
    assert np.array_equal(kmix.double().cpu().numpy(), wk) and np.array_equal(vmix.double().cpu().numpy(), wv)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("t", [1, 40])
def test_nan_rows_matter_where_they_are_attended_to(dtype, t):
    """Block 1 of token 40's value and token 200's key are NaN; token 0, which is read in the place of rows that are not there,
    is NaN altogether.  Queries with these tokens in a sparse chunk's unkept rows get the results without them."""
    rng = np.random.default_rng(40)
    lay = wl.layout_from_lists(0, [30, 70, 90, 101], [np.arange(c, c + 4) + 2 for c in (0, 30, 100, 190)])
    hq, hkv, d, fmt = 6, 2, 128, "fp4"
    k, v = random_rows(rng, (hkv, lay.n_tokens, d), dtype), random_rows(rng, (hkv, lay.n_tokens, d), dtype)
    rows, scales, wk, wv = quantised(k, v, fmt)
    scales[:, 40, 1, 1] = 255
    scales[:, 200, 0, 3] = 255
    scales[:, 0] = 255
    desc, gl = vxl.make_desc(hq, hkv, d, dtype), make_layout(lay)
    cache = device_cache(desc, fmt, rows, scales, spare=1)
    masks = np.array([[0, 0, 1, 0], [0, 1, 1, 0], [0, 0, 0, 1], [1, 0, 0, 0]], np.uint8)
    wkm, wvm, wlen, _ = oracle.gather_bilevel(wk, wv, masks, 0, lay.chunk_bounds, lay.sparse_offsets, lay.sparse_idx, l_cap=lay.n_tokens)
    qd = rng.standard_normal((4, t, hq, d)).astype(np.float32) * 0.1
    dq = vxl.to_device(wl.round_to_bf16(qd), dtype)
    out, lse = torch.zeros_like(dq), torch.zeros(dq.shape[:3], device="cuda")
    ws = vxl.alloc_workspace(vxl.workspace_bytes(vxl.OP_DECODE_KVQ, gl, desc, 4, t, lay.n_tokens))
    vxl.bilevel_decode_kvq(gl, desc, dq, cache, None, torch.from_numpy(masks).cuda(), lay.n_tokens, out, lse, None, ws)
    got, got_lse = out.double().cpu().numpy(), lse.cpu().numpy()
    want, want_lse = oracle.decode_lse(wl.round_to_bf16(qd), wkm, wvm, wlen)
    assert np.abs(got[0] - want[0]).max() <= 2.0 ** -6 * np.abs(wvm).max() and np.isfinite(got_lse[0]).all()
    assert np.isnan(got[1][..., 32:64]).all() and np.isfinite(np.delete(got[1], np.s_[32:64], -1)).all()
    assert np.abs(got_lse[1] - want_lse[1]).max() < 1e-4
    assert np.isnan(got[2]).all() and np.isnan(got_lse[2]).all()
    assert np.isnan(got[3]).all() and np.isnan(got_lse[3]).all()


def test_queries_that_are_not_finite():
    """A NaN or an infinity in one query row makes that row NaN and no other."""
    rng = np.random.default_rng(41)
    lay = wl.layout_from_lists(300, [], [])
    for dtype in ("bf16", "f32"):
        cache, _, _, _ = prompt(rng, dtype, 1, 64, "fp8", lay, False)
        desc, gl = vxl.make_desc(5, 1, 64, dtype), make_layout(lay)
        good = torch.randn(1, 7, 5, 64, device="cuda").to(DTYPE[dtype])
        bad = good.clone()
        bad[0, 2, 3, 10] = float("nan")
        bad[0, 6, 0, 63] = float("inf")
        ws = vxl.alloc_workspace(vxl.workspace_bytes(vxl.OP_DECODE_KVQ, gl, desc, 1, 7, 300))
        outs = []
        for q in (good, bad):
            outs.append((torch.zeros_like(q), torch.zeros(q.shape[:3], device="cuda")))
            vxl.bilevel_decode_kvq(gl, desc, q, cache, None, None, 300, *outs[-1], None, ws)
        hit = torch.zeros(1, 7, 5, dtype=torch.bool, device="cuda")
        hit[0, 2, 3] = hit[0, 6, 0] = True
        assert outs[1][0][hit].isnan().all() and outs[1][1][hit].isnan().all()
        assert outs[1][0][~hit].isfinite().all() and outs[1][1][~hit].isfinite().all()
        assert (outs[0][0][~hit].float() - outs[1][0][~hit].float()).abs().max() <= 2.0 ** -6 * outs[0][0].float().abs().max()


@pytest.mark.parametrize("dtype,hq,hkv,t,bsz,kernel", [("bf16", 1, 1, 1, 1, 1), ("bf16", 4, 2, 30, 1, 2), ("bf16", 8, 4, 200, 32, 0),
                                                       ("f32", 2, 2, 3, 1, 1)])
def test_logits_below_the_smallest_number(dtype, hq, hkv, t, bsz, kernel):
    """Products that overflow to -inf: these keys weigh nothing, also where they are all that a wave sees for a while, and
    where the rest of an fp32 query that bf16 does not hold overflows by itself (rounded up, it would be of the other sign)."""
    n, few, d = 700, 60, 128
    lay = wl.layout_from_lists(n, [], [])
    desc, gl = vxl.make_desc(hq, hkv, d, dtype), make_layout(lay)
    assert vxl.debug_kvq_plan(desc, bsz, t, n)[0] == kernel
    rng = np.random.default_rng(n)
    k, v = np.zeros((hkv, n, d), np.float32), random_rows(rng, (hkv, n, d), dtype)
    k[:, :n - few, 0] = -2.0 ** 100
    rows, scales, _, wv = quantised(k, v, "fp8")
    cache = device_cache(desc, "fp8", rows, scales)
    qd = np.zeros((bsz, t, hq, d), np.float32)
    qd[..., 0] = np.float32(2.0 ** 127 * (1 + 2.0 ** -7 - (2.0 ** -12 if dtype == "f32" else 0)))
    qd[..., 1:] = 1
    dq = vxl.to_device(qd, dtype)
    out, lse = torch.zeros_like(dq), torch.zeros(dq.shape[:3], device="cuda")
    ws = vxl.alloc_workspace(vxl.workspace_bytes(vxl.OP_DECODE_KVQ, gl, desc, bsz, t, n))
    vxl.bilevel_decode_kvq(gl, desc, dq, cache, None, None, n, out, lse, None, ws)
    part = wv[:, n - few:]
    # the logits that count are 0 and their weights 1: `few` additions in fp32, a division, the result's rounding
    want, sums = part.mean(1), np.abs(part).mean(1) * (few + 2) * 2.0 ** -24
    bound = sums + (np.abs(want) * 1.01 * 2.0 ** -8 if dtype == "bf16" else 0)
    got = out.double().cpu().numpy().reshape(bsz, t, hkv, hq // hkv, d)
    assert (np.abs(got - want[:, None]) <= bound[:, None]).all()
    assert (np.abs(lse.double().cpu().numpy() - np.log(few)) <= 2.0 ** -21 * np.log(few)).all()


@pytest.mark.parametrize("scale", [0.0, 4.0])
@pytest.mark.parametrize("dtype,hq,hkv,d,t,bsz,n,kernel,one", [
    ("bf16", 6, 2, 128, 1, 400, 2100, 1, True), ("bf16", 6, 2, 128, 1, 64, 2100, 1, False), ("f32", 6, 2, 128, 3, 400, 2100, 1, True),
    ("f32", 6, 2, 64, 3, 64, 2100, 1, False), ("bf16", 6, 2, 64, 20, 400, 2100, 2, True), ("bf16", 6, 2, 128, 20, 16, 2100, 2, False),
    ("bf16", 8, 4, 64, 200, 32, 2100, 0, True), ("bf16", 32, 4, 128, 129, 1, 16000, 0, False)])
def test_rows_below_the_smallest_number_beside_others(dtype, hq, hkv, d, t, bsz, n, kernel, one, scale):
    """Of three query rows that a wave has side by side one meets runs of keys whose products overflow to -inf (scale 4: whose
    products do when they are scaled) before, between and behind others, one has logits of a few units with all of them, and
    one has -inf with all: its result is NaN and its LSE -inf.  One KV head has a key of the first run that all rows can be
    compared with."""
    lay = wl.layout_from_lists(n, [], [])
    desc, gl = vxl.make_desc(hq, hkv, d, dtype, scale), make_layout(lay)
    far, gain = (2.0 ** 27, 3 / (scale * d ** 0.5)) if scale else (2.0 ** 127, 3)
    scale = scale or d ** -0.5
    plan = vxl.debug_kvq_plan(desc, bsz, t, n)
    assert plan[0] == kernel and (plan[1] == 1) == one
    rng = np.random.default_rng(n + d + t)
    k, v = rng.standard_normal((hkv, n, d)).astype(np.float32) * np.float32(0.3), random_rows(rng, (hkv, n, d), dtype)
    runs = np.arange(n) // 256 % 2 == 0                             # (eight 32-key tiles: two steps of a workgroup's four waves)
    k[..., 0] = np.where(runs, -2.0 ** 100, 0)
    k[1, 5, 0] = 0
    k[..., -1] = -2.0 ** 100
    rows, scales, wk, wv = quantised(wl.round_to_bf16(k), v, "fp8")
    cache = device_cache(desc, "fp8", rows, scales)
    some = min(bsz, 2)
    qd = rng.standard_normal((some, t, hq, d)).astype(np.float32) * np.float32(gain)
    kind = (np.arange(t)[:, None] * hq + np.arange(hq)) % 3
    qd[..., 0] = np.where(kind == 0, far, 0)
    qd[..., -1] = np.where(kind == 2, far, 0)
    qd = wl.round_to_bf16(qd) if dtype == "bf16" else qd
    dq = vxl.to_device(qd, dtype).repeat(bsz // some, 1, 1, 1)
    out, lse = torch.zeros_like(dq), torch.zeros(dq.shape[:3], device="cuda")
    ws = vxl.alloc_workspace(vxl.workspace_bytes(vxl.OP_DECODE_KVQ, gl, desc, bsz, t, n))
    vxl.bilevel_decode_kvq(gl, desc, dq, cache, None, None, n, out, lse, None, ws)
    for b in range(some, bsz, some):
        assert same_bits(out[b:b + some], out[:some]) and same_bits(lse[b:b + some], lse[:some])
    got, got_lse = out[:some].double().cpu().numpy(), lse[:some].double().cpu().numpy()
    assert np.isnan(got[:, kind == 2]).all() and (got_lse[:, kind == 2] == -np.inf).all()
    inner = qd.copy()
    inner[..., [0, -1]] = 0                                         # (the elements behind a logit that is no infinity)
    for b in range(some):
        o, wlse, av, _ = attention(np.where(kind[..., None] == 2, 0, qd[b]), wk, wv, n, scale)
        aq = attention(inner[b], wk, wv, n, scale)[3]
        # the bounds of check_decode
        logit, sums = (44 + 4) * 2.0 ** -24 * aq * 1.5 + 2.0 ** -22, (n / 16 + 100) * 2.0 ** -24
        bound = av * (2 * logit + 2 * sums)[..., None] + n * 2.0 ** -126 * np.abs(wv).max()
        if dtype == "bf16":
            bound = bound + 1.01 * 2.0 ** -8 * (av + np.abs(o))
        finite = kind < 2
        assert (np.abs(got[b] - o)[finite] <= bound[finite]).all(), float((np.abs(got[b] - o)[finite] / bound[finite]).max())
        assert (np.abs(got_lse[b] - wlse)[finite] <= (logit + sums + np.abs(wlse) * 2.0 ** -22)[finite]).all()


def test_the_largest_batch():
    """65,535 queries, each as on its own with its mask; one more is refused before anything is written."""
    rng = np.random.default_rng(17)
    lay = wl.random_layout(rng, 3, 4, 10, 20)
    cache, sparse, _, _ = prompt(rng, "bf16", 2, 64, "fp4", lay, True)
    gl, desc, cap, bsz = make_layout(lay), vxl.make_desc(2, 2, 64, "bf16"), lay.n_tokens, 65535
    masks = torch.from_numpy(some_masks(rng, 16, 4)).cuda().repeat(bsz // 16 + 1, 1).contiguous()
    few = torch.randn(16, 1, 2, 64, device="cuda").bfloat16()
    qd = few.repeat(bsz // 16 + 1, 1, 1, 1).contiguous()
    out, lens = torch.full_like(qd, 9.0), torch.full((bsz + 1,), -77, dtype=torch.int32, device="cuda")
    ws = vxl.alloc_workspace(vxl.workspace_bytes(vxl.OP_DECODE_KVQ, gl, desc, bsz + 1, 1, cap))
    with pytest.raises(vxl.VxlError) as e:
        vxl.bilevel_decode_kvq(gl, desc, qd, cache, sparse, masks, cap, out, None, lens, ws)
    torch.cuda.synchronize()
    assert e.value.status == vxl.VXL_ERR_UNSUPPORTED and (out == 9.0).all() and (lens == -77).all()
    vxl.bilevel_decode_kvq(gl, desc, qd[:bsz], cache, sparse, masks[:bsz], cap, out[:bsz], None, lens[:bsz], ws)
    want, n = torch.zeros_like(few), torch.zeros(16, dtype=torch.int32, device="cuda")
    small = vxl.alloc_workspace(vxl.workspace_bytes(vxl.OP_DECODE_KVQ, gl, desc, 16, 1, cap))
    vxl.bilevel_decode_kvq(gl, desc, few, cache, sparse, masks[:16], cap, want, None, n, small)
    assert vxl.debug_kvq_plan(desc, 16, 1, cap) == vxl.debug_kvq_plan(desc, bsz, 1, cap) == (1, 1)
    assert same_bits(out[:bsz], want.repeat(bsz // 16 + 1, 1, 1, 1)[:bsz]) and torch.equal(lens[:bsz], n.repeat(bsz // 16 + 1)[:bsz])
    assert (out[bsz:] == 9.0).all() and lens[bsz] == -77


@pytest.mark.parametrize("dtype,hq,hkv,t,bsz,kernel", [("f32", 16, 1, 14, 5000, 1), ("f32", 8, 8, 17, 33000, 1), ("bf16", 16, 1, 8, 20000, 2),
                                                       ("bf16", 16, 1, 32, 33000, 0)])
def test_more_row_tiles_than_a_grid_dimension(dtype, hq, hkv, t, bsz, kernel):
    """Queries that are fewer than 65,536, but whose row tiles together are more: each as on its own with its mask."""
    rng = np.random.default_rng(bsz)
    lay = wl.random_layout(rng, 3, 4, 5, 12)
    cache, sparse, values, sparse_values = prompt(rng, dtype, hkv, 64, "fp8", lay, True)
    gl, desc, cap, rows = make_layout(lay), vxl.make_desc(hq, hkv, 64, dtype), lay.n_tokens, hq // hkv * t
    assert vxl.debug_kvq_plan(desc, bsz, t, cap) == (kernel, 1) and bsz * -(-rows // (16 * kernel or 256)) > 65535
    masks = some_masks(rng, 16, 4)
    qd = wl.round_to_bf16(rng.standard_normal((16, t, hq, 64)).astype(np.float32))
    whole, more = bsz // 16, bsz % 16
    dm, dq = torch.from_numpy(masks).cuda().repeat(whole + 1, 1)[:bsz], vxl.to_device(qd, dtype).repeat(whole + 1, 1, 1, 1)[:bsz]
    out = torch.full((bsz + 1, t, hq, 64), 9.0, dtype=DTYPE[dtype], device="cuda")
    lens = torch.full((bsz + 1,), -77, dtype=torch.int32, device="cuda")
    ws = vxl.alloc_workspace(vxl.workspace_bytes(vxl.OP_DECODE_KVQ, gl, desc, bsz, t, cap))
    vxl.bilevel_decode_kvq(gl, desc, dq, cache, sparse, dm, cap, out[:bsz], None, lens[:bsz], ws)
    wk, wv, wlen, _ = mixed(values, sparse_values, masks, lay, cap)
    assert np.array_equal(lens[:bsz].cpu().numpy(), np.tile(wlen, whole + 1)[:bsz]) and lens[bsz] == -77 and (out[bsz] == 9.0).all()
    assert same_bits(out[16:16 * whole], out[:16].repeat(whole - 1, 1, 1, 1)) and same_bits(out[16 * whole:bsz], out[:more])
    got = out[:16].double().cpu().numpy()
    for b in range(16):
        n = int(wlen[b])
        o, _, av, aq = attention(qd[b], wk[b], wv[b], n, 64 ** -0.5)
        # the bounds of check_decode
        bound = av * (2 * ((44 + 4) * 2.0 ** -24 * aq * 1.5 + 2.0 ** -22) + 2 * (n / 16 + 100) * 2.0 ** -24)[..., None] + n * 2.0 ** -126 * np.abs(wv).max()
        bound = bound + (1.01 * 2.0 ** -8 * (av + np.abs(o)) if dtype == "bf16" else 0)
        assert (np.abs(got[b] - o) <= bound).all()


def test_the_longest_cache():
    """Rows at the end of a cache of the largest capacity, whose offsets pass 32 bits, as from one that holds them alone."""
    cap, hkv, d, p, last, fmt = 1 << 24, 2, 128, 64, 500, "fp8"
    desc = vxl.make_desc(4, hkv, d, "bf16")
    lens = [(cap - p - last) // 40] * 39
    lens += [cap - p - last - sum(lens), last]
    tail = cap - last
    long = wl.layout_from_lists(p, lens, [[]] * 40 + [np.arange(tail + 3, cap, 7)])
    short = wl.layout_from_lists(p, [last], [np.arange(p + 3, p + last, 7)])
    whole, part = vxl.KvqCache(desc, fmt, cap), vxl.KvqCache(desc, fmt, p + last)
    k, v = (torch.randn(hkv, p + last, d, device="cuda").bfloat16() for _ in range(2))
    vxl.kvq_write(desc, k, v, part)
    cut = lambda x, a, b: x[:, a:b].contiguous()  # noqa: E731
    vxl.kvq_write(desc, cut(k, 0, p), cut(v, 0, p), whole)
    vxl.kvq_write(desc, cut(k, p, p + last), cut(v, p, p + last), whole, tail)
    with pytest.raises(vxl.VxlError):
        vxl.kvq_write(desc, cut(k, 0, 1), cut(v, 0, 1), whole, cap)
    back = [torch.zeros(hkv, last, d, dtype=torch.bfloat16, device="cuda") for _ in range(4)]
    vxl.kvq_read(desc, whole, *back[:2], tail)
    vxl.kvq_read(desc, part, *back[2:], p)
    assert same_bits(back[0], back[2]) and same_bits(back[1], back[3])
    sparse = vxl.KvqCache(desc, fmt, len(short.sparse_idx))
    vxl.kvq_write(desc, *(x[:, short.sparse_idx].contiguous() for x in (v, k)), sparse)
    l_cap = p + last
    for kept in (None, sparse):
        for bsz, t in ((2, 1), (2, 40), (64, 200)):
            results = []
            for lay, cache in ((long, whole), (short, part)):
                gl = make_layout(lay)
                mask = torch.zeros(bsz, gl.n_chunks, dtype=torch.uint8, device="cuda")
                mask[::2, -1] = 1
                kmix = torch.zeros(bsz, hkv, l_cap, d, dtype=torch.bfloat16, device="cuda")
                vmix, n = torch.zeros_like(kmix), torch.zeros(bsz, dtype=torch.int32, device="cuda")
                vxl.gather_bilevel_kvq(gl, desc, cache, kept, mask, kmix, vmix, n)
                q = torch.randn(bsz, t, 4, d, generator=torch.Generator("cuda").manual_seed(t), device="cuda").bfloat16()
                ws = vxl.alloc_workspace(vxl.workspace_bytes(vxl.OP_DECODE_KVQ, gl, desc, bsz, t, l_cap))
                out, lse = torch.zeros_like(q), torch.zeros(q.shape[:3], device="cuda")
                vxl.bilevel_decode_kvq(gl, desc, q, cache, kept, mask, l_cap, out, lse, None, ws)
                results.append((kmix, vmix, n, out, lse))
            assert all(same_bits(a, b) for a, b in zip(*results)) and results[0][2][0] == l_cap
            assert results[0][3].isfinite().all() and results[0][3].any()
    assert [vxl.debug_kvq_plan(desc, b, t, l_cap)[0] for b, t in ((2, 1), (2, 40), (64, 200))] == [1, 2, 0]
    with pytest.raises(vxl.VxlError) as e:
        vxl.kvq_write(desc, cut(k, 0, 1), cut(v, 0, 1), vxl.KvqCache(desc, "fp4", cap + 1))
    assert e.value.status == vxl.VXL_ERR_UNSUPPORTED


def test_a_map_of_the_plain_cache():
    """The row map that the plain decode in place left in the workspace serves the quantised one, and the other way round."""
    rng = np.random.default_rng(19)
    lay = wl.random_layout(rng, 30, 5, 40, 90)
    hq, hkv, d, n, t = 8, 2, 128, lay.n_tokens, 3
    gl, desc = make_layout(lay), vxl.make_desc(hq, hkv, d, "bf16")
    k, v = (torch.randn(hkv, n, d, device="cuda").bfloat16() for _ in range(2))
    cache = vxl.KvqCache(desc, "fp8", n)
    vxl.kvq_write(desc, k, v, cache)
    vxl.kvq_read(desc, cache, k, v)                                 # (one set of values for both)
    qd, mask = torch.randn(2, t, hq, d, device="cuda").bfloat16(), torch.from_numpy(some_masks(rng, 2, 5)).cuda()
    need = max(vxl.workspace_bytes(op, gl, desc, 2, t, n) for op in (vxl.OP_DECODE_KVQ, vxl.OP_DECODE_INPLACE))
    plain = lambda o, ws, ready: vxl.bilevel_decode_inplace(gl, desc, qd, k, v, None, None, mask, n, o, workspace=ws, map_ready=ready)  # noqa: E731
    quant = lambda o, ws, ready: vxl.bilevel_decode_kvq(gl, desc, qd, cache, None, mask, n, o, workspace=ws, map_ready=ready)  # noqa: E731
    for first, second in ((plain, quant), (quant, plain)):
        ws, other = vxl.alloc_workspace(need), vxl.alloc_workspace(need)
        outs = [torch.zeros_like(qd) for _ in range(3)]
        first(outs[0], ws, False)
        second(outs[1], ws, True)
        second(outs[2], other, False)
        assert same_bits(outs[1], outs[2])
        assert (outs[0].float() - outs[1].float()).abs().max() <= 4 * 2.0 ** -8 * v.float().abs().max()


# ---- together, as they are used ------------------------------------------------------------------
def test_a_prompt_in_a_quantised_cache():
    """Chunk by chunk into the cache as the pre-filling ends them, pooled rows quantised beside; selection by the mean keys
    of the plain cache; gather + plain decode and the decode in place agree, the in-place one also for the next tokens."""
    rng = np.random.default_rng(99)
    hq, hkv, d, t, top_k = 14, 2, 128, 6, 3
    lay = wl.random_layout(rng, 40, 9, 60, 200)
    gl, desc = make_layout(lay), vxl.make_desc(hq, hkv, d, "bf16", token_major=True)
    n, n_sparse = lay.n_tokens, int(lay.sparse_offsets[-1])
    q, k, v = (torch.randn(n, h, d, generator=torch.Generator("cuda").manual_seed(5 + h), device="cuda").bfloat16() for h in (hq, hkv, hkv))
    out = torch.empty_like(q)
    vxl.chunk_prefill(gl, desc, q, k, v, out, None, vxl.alloc_workspace(vxl.workspace_bytes(vxl.OP_PREFILL, gl, desc)))
    cache, sparse = vxl.KvqCache(desc, "fp8", n), vxl.KvqCache(desc, "fp8", n_sparse)
    for lo, hi in zip([0, *lay.chunk_bounds[:-1]], lay.chunk_bounds):
        vxl.kvq_write(desc, k[lo:hi], v[lo:hi], cache, lo)
    ksp, vsp = (torch.empty(hkv, n_sparse, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    vxl.pool_sparse_kv(gl, desc, k, v, ksp, vsp)
    vxl.kvq_write(vxl.make_desc(hq, hkv, d, "bf16"), ksp, vsp, sparse)
    whole = vxl.KvqCache(desc, "fp8", n)
    vxl.kvq_write(desc, k, v, whole)
    assert torch.equal(cache.rows, whole.rows) and torch.equal(cache.scales, whole.scales)
    qd = torch.randn(2, t, hq, d, device="cuda").bfloat16()
    idx, mask = torch.zeros(2, top_k, dtype=torch.int32, device="cuda"), torch.zeros(2, lay.n_chunks, dtype=torch.uint8, device="cuda")
    vxl.chunk_score_topk(gl, desc, qd, k, top_k, idx, mask, workspace=vxl.alloc_workspace(
        vxl.workspace_bytes(vxl.OP_SCORE_TOPK, gl, desc, 2, t)))
    cap = gl.mixed_kv_capacity(top_k)
    kmix = torch.zeros(2, hkv, cap, d, dtype=torch.bfloat16, device="cuda")
    vmix, lens = torch.zeros_like(kmix), torch.zeros(2, dtype=torch.int32, device="cuda")
    for sp in (None, sparse):
        vxl.gather_bilevel_kvq(gl, desc, cache, sp, mask, kmix, vmix, lens)
        a, b = torch.empty_like(qd), torch.empty_like(qd)
        vxl.bilevel_decode(desc, qd, kmix, vmix, lens, a, None, vxl.alloc_workspace(vxl.workspace_bytes(vxl.OP_DECODE, None, desc, 2, t, cap)))
        ws = vxl.alloc_workspace(max(vxl.workspace_bytes(vxl.OP_DECODE_KVQ, gl, desc, 2, x, cap) for x in (1, t)))
        lens2 = torch.zeros_like(lens)
        vxl.bilevel_decode_kvq(gl, desc, qd, cache, sp, mask, cap, b, None, lens2, ws)
        assert torch.equal(lens, lens2)
        # each of the two rounds its weights and its result to bf16, by half a step (2^-8) of sum p |v| each at most
        assert (a.float() - b.float()).abs().max() <= 4 * 2.0 ** -8 * vmix.float().abs().max()
        for i in (0, t - 1):                                       # single tokens on the map that the question left
            one, got = qd[:, i:i + 1].contiguous(), torch.empty_like(qd[:, :1])
            vxl.bilevel_decode_kvq(gl, desc, one, cache, sp, mask, cap, got, None, lens2, ws, map_ready=True)
            assert (got.float() - b[:, i:i + 1].float()).abs().max() <= 4 * 2.0 ** -8 * vmix.float().abs().max()
        plain = vxl.KvqCache(desc, "fp8", n)                       # read back and written again: the same codes
        back = [torch.empty_like(k) for _ in range(2)]
        vxl.kvq_read(desc, cache, *back)
        vxl.kvq_write(desc, *back, plain)
        again = [torch.empty_like(k) for _ in range(2)]
        vxl.kvq_read(desc, plain, *again)
        assert all(torch.equal(x, y) for x, y in zip(back, again))


def test_in_a_replayed_graph():
    """Write, gather and both forms of the decode in one captured graph, replayed on new inputs with eager work in between."""
    rng = np.random.default_rng(12)
    lay = wl.random_layout(rng, 20, 6, 30, 90)
    hq, hkv, d = 8, 2, 128
    gl, desc = make_layout(lay), vxl.make_desc(hq, hkv, d, "bf16")
    n = lay.n_tokens
    k, v = (torch.randn(hkv, n, d, device="cuda").bfloat16() for _ in range(2))
    qd = torch.randn(2, 1, hq, d, device="cuda").bfloat16()
    mask = torch.from_numpy(some_masks(rng, 2, 6)).cuda()
    cache = vxl.KvqCache(desc, "fp4", n)
    kmix = torch.zeros(2, hkv, n, d, dtype=torch.bfloat16, device="cuda")
    bufs = dict(kmix=kmix, vmix=torch.zeros_like(kmix), lens=torch.zeros(2, dtype=torch.int32, device="cuda"), a=torch.zeros_like(qd),
                b=torch.zeros_like(qd), lse=torch.zeros(2, 1, hq, device="cuda"))
    ws = vxl.alloc_workspace(vxl.workspace_bytes(vxl.OP_DECODE_KVQ, gl, desc, 2, 1, n))

    def chain(x, ws):
        vxl.kvq_write(desc, k, v, cache)
        vxl.gather_bilevel_kvq(gl, desc, cache, None, mask, x["kmix"], x["vmix"], x["lens"])
        vxl.bilevel_decode_kvq(gl, desc, qd, cache, None, mask, n, x["a"], x["lse"], x["lens"], ws)
        vxl.bilevel_decode_kvq(gl, desc, qd, cache, None, mask, n, x["b"], None, x["lens"], ws, map_ready=True)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        chain(bufs, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        chain(bufs, ws)
    for i in range(4):
        for x in (k, v, qd):
            x.copy_(torch.randn_like(x))
        mask.copy_(torch.from_numpy(some_masks(rng, 2, 6)))
        want = {name: torch.zeros_like(x) for name, x in bufs.items()}
        chain(want, torch.empty_like(ws))
        torch.cuda.synchronize()
        for x in bufs.values():
            x.fill_(3)
        bufs["kmix"].zero_(), bufs["vmix"].zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(same_bits(want[name], x) for name, x in bufs.items()), i
        assert same_bits(bufs["a"], bufs["b"])


def test_on_streams_of_their_own():
    """Two streams with a workspace each, at once; results as on one."""
    rng = np.random.default_rng(15)
    lay = wl.random_layout(rng, 100, 8, 300, 900)
    cache, sparse, _, _ = prompt(rng, "bf16", 2, 128, "fp4", lay, True)
    gl, desc, n = make_layout(lay), vxl.make_desc(14, 2, 128, "bf16"), lay.n_tokens
    qs = [torch.randn(1, t, 14, 128, device="cuda").bfloat16() for t in (1, 30)]
    masks = [torch.from_numpy(m[None]).cuda() for m in some_masks(rng, 2, 8)]
    work = [vxl.alloc_workspace(vxl.workspace_bytes(vxl.OP_DECODE_KVQ, gl, desc, 1, q.shape[1], n)) for q in qs]
    want = [vxl.bilevel_decode_kvq(gl, desc, q, cache, sparse, m, n, torch.zeros_like(q), workspace=w) for q, m, w in zip(qs, masks, work)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in qs]
    for _ in range(5):
        got = [torch.zeros_like(q) for q in qs]
        torch.cuda.synchronize()
        for s, q, m, w, o in zip(streams, qs, masks, work, got):
            vxl.bilevel_decode_kvq(gl, desc, q, cache, sparse, m, n, o, workspace=w, stream=s)
        torch.cuda.synchronize()
        assert all(same_bits(a, b) for a, b in zip(want, got))


def test_rows_that_a_tensor_or_a_cache_does_not_hold():
    """Numbers of rows and strides past the tensor, first rows past 32 bits, no rows at all."""
    desc = vxl.make_desc(4, 2, 64, "bf16")
    k = torch.ones(2, 10, 64, dtype=torch.bfloat16, device="cuda")
    cache = vxl.KvqCache(desc, "fp4", 20)
    cache.rows.fill_(3), cache.scales.fill_(4)
    wide = vxl.make_desc(4, 2, 64, "bf16")
    wide.q_stride_head, wide.q_stride_tok, wide.kv_stride_head, wide.kv_stride_tok = 640, 64, 1 << 62, 1 << 62
    for d, n, first in ((desc, 11, 0), (desc, 10, 11), (desc, 10, 1 << 32), (desc, 10, -(1 << 32)), (desc, (1 << 32) + 10, 0), (desc, -1, 0),
                        (wide, 10, 0), (wide, 5, 0)):
        for call in (lambda: vxl.kvq_write(d, k, k, cache, first, n), lambda: vxl.kvq_read(d, cache, k, torch.ones_like(k), first, n)):
            with pytest.raises(vxl.VxlError) as e:
                call()
            assert e.value.status == vxl.VXL_ERR_INVALID_ARG, (n, first)
    vxl.kvq_write(desc, k, k, cache, 20, 0), vxl.kvq_read(desc, cache, k, k, 0, 0)
    torch.cuda.synchronize()
    assert (cache.rows == 3).all() and (cache.scales == 4).all() and (k == 1).all()


def test_buffers_side_by_side():
    """Keys and values of one tensor, token by token, and everything in one allocation without a gap: the same rows."""
    hkv, n, d = 4, 33, 64
    desc = vxl.make_desc(hkv, hkv, d, "bf16")
    k, v = (torch.randn(hkv, n, d, device="cuda").bfloat16() for _ in range(2))
    want = vxl.KvqCache(desc, "fp4", n)
    vxl.kvq_write(desc, k, v, want)
    pair = vxl.make_desc(hkv, hkv, d, "bf16")
    pair.q_stride_head = pair.kv_stride_head = d
    pair.q_stride_tok = pair.kv_stride_tok = 2 * hkv * d
    both = torch.stack((k, v)).permute(2, 0, 1, 3).contiguous()         # [n, 2, hkv, d]
    cache = vxl.KvqCache(desc, "fp4", n)
    flat = both.view(-1)
    vxl.kvq_write(pair, flat, flat[hkv * d:], cache, 0, n)
    assert torch.equal(cache.rows, want.rows) and torch.equal(cache.scales, want.scales)
    back = torch.zeros_like(flat)
    vxl.kvq_read(pair, cache, back, back[hkv * d:], 0, n)
    values = [torch.zeros_like(k) for _ in range(2)]
    vxl.kvq_read(desc, want, *values)
    assert same_bits(back.view(n, 2, hkv, d), torch.stack(values).permute(2, 0, 1, 3).contiguous())
    plain, codes, scales = k.numel() * 2, want.rows.numel(), want.scales.numel()
    room = torch.zeros(2 * plain + codes + scales, dtype=torch.uint8, device="cuda")
    kk, vv, rows, sc = room.split([plain, plain, codes, scales])
    near = vxl.KvqCache(desc, "fp4", rows=rows.view_as(want.rows), scales=sc.view_as(want.scales))
    kk.view(torch.bfloat16).copy_(k.view(-1)), vv.view(torch.bfloat16).copy_(v.view(-1))
    vxl.kvq_write(desc, kk.view(torch.bfloat16), vv.view(torch.bfloat16), near)
    assert torch.equal(near.rows, want.rows) and torch.equal(near.scales, want.scales)
    vxl.kvq_read(desc, near, kk.view(torch.bfloat16), vv.view(torch.bfloat16))
    assert same_bits(kk.view(torch.bfloat16).view_as(k), values[0]) and same_bits(vv.view(torch.bfloat16).view_as(v), values[1])


def test_outputs_that_overlap():
    """A mixed set, a result, an LSE, lengths or a workspace in a cache or in another of them: refused, and nothing is written."""
    rng = np.random.default_rng(29)
    lay = wl.random_layout(rng, 10, 4, 20, 40)
    cache, sparse, _, _ = prompt(rng, "bf16", 2, 64, "fp4", lay, True)
    gl, desc, n = make_layout(lay), vxl.make_desc(4, 2, 64, "bf16"), lay.n_tokens
    before = [t.clone() for c in (cache, sparse) for t in (c.rows, c.scales)]
    mask = torch.ones(1, 4, dtype=torch.uint8, device="cuda")
    size, need = 2 * n * 64 * 2, vxl.workspace_bytes(vxl.OP_DECODE_KVQ, gl, desc, 1, 3, n)

    class At:                                                           # (a tensor of this size at this address, in bounds or not)
        is_cuda = True

        def __init__(self, ptr, shape):
            self.ptr, self.shape = ptr, shape
        is_contiguous, data_ptr, numel = (lambda self: True), (lambda self: self.ptr), (lambda self: int(np.prod(self.shape)))

    part = (size + need) // 256 * 256 + 256
    room = torch.zeros(7 * part, dtype=torch.uint8, device="cuda")
    free = room.data_ptr()
    mix = lambda p: At(p, (1, 2, n, 64))  # noqa: E731
    q = lambda p: At(p, (1, 3, 4, 64))  # noqa: E731
    kmix, vmix, lens, ws, qd, out, lse = (free + i * part for i in range(7))
    gather = lambda k=kmix, v=vmix, m=lens, s=0: vxl.gather_bilevel_kvq(gl, desc, cache, sparse, mask, mix(k), mix(v), At(m, (1,)), At(s, (1, n)) if s else None)  # noqa: E731
    decode = lambda o=out, l=lse, m=lens, w=ws: vxl.bilevel_decode_kvq(gl, desc, q(qd), cache, sparse, mask, n, q(o), At(l, (1, 3, 4)), At(m, (1,)), At(w, (need,)))  # noqa: E731
    inside = [t.data_ptr() + t.numel() // 2 // 16 * 16 for c in (cache, sparse) for t in (c.rows, c.scales)]
    calls = [(gather, dict(v=kmix + 16)), (gather, dict(m=kmix + 64)), (gather, dict(s=vmix)), (gather, dict(s=lens - 4))]
    calls += [(gather, {x: p}) for x in "kvms" for p in inside] + [(decode, {x: p}) for x in "olmw" for p in inside]
    calls += [(decode, dict(o=qd + 16)), (decode, dict(l=out + 4)), (decode, dict(m=lse)), (decode, dict(w=out - 256)), (decode, dict(w=qd - need + 16)),
              (decode, dict(m=ws + need - 4))]
    for call, kw in calls:
        with pytest.raises(vxl.VxlError) as e:
            call(**kw)
        assert e.value.status == vxl.VXL_ERR_INVALID_ARG, kw
    torch.cuda.synchronize()
    assert not room.any() and all(torch.equal(a, b) for a, b in zip(before, [t for c in (cache, sparse) for t in (c.rows, c.scales)]))
    gather(), decode()
    torch.cuda.synchronize()
    assert room.any()


def test_a_cache_whose_tensors_are_replaced():
    """Written, read and attended to are the tensors that a cache has at the call; those it had before are left as they are."""
    rng = np.random.default_rng(23)
    lay = wl.random_layout(rng, 10, 4, 20, 40)
    gl, n, desc = make_layout(lay), lay.n_tokens, vxl.make_desc(4, 2, 64, "bf16")
    k, v = (torch.randn(2, n, 64, device="cuda").bfloat16() for _ in range(2))
    cache, want = vxl.KvqCache(desc, "fp4", n), vxl.KvqCache(desc, "fp4", n + 5)
    old = cache.rows.fill_(3), cache.scales.fill_(4)
    cache.rows, cache.scales = torch.zeros(2, n + 5, 2, 32, dtype=torch.uint8, device="cuda"), torch.zeros(2, n + 5, 2, 2, dtype=torch.uint8, device="cuda")
    for c in (cache, want):
        c.rows.zero_(), c.scales.zero_()
        vxl.kvq_write(desc, k, v, c, 5)
    assert cache.capacity == n + 5 and torch.equal(cache.rows, want.rows) and torch.equal(cache.scales, want.scales) and cache.rows.any()
    assert (old[0] == 3).all() and (old[1] == 4).all()
    del old
    back = [torch.zeros_like(k) for _ in range(4)]
    vxl.kvq_read(desc, cache, *back[:2], 5), vxl.kvq_read(desc, want, *back[2:], 5)
    assert same_bits(back[0], back[2]) and same_bits(back[1], back[3]) and back[0].any()
    q, mask = torch.randn(1, 2, 4, 64, device="cuda").bfloat16(), torch.ones(1, 4, dtype=torch.uint8, device="cuda")
    ws = vxl.alloc_workspace(vxl.workspace_bytes(vxl.OP_DECODE_KVQ, gl, desc, 1, 2, n))
    out = [vxl.bilevel_decode_kvq(gl, desc, q, c, None, mask, n, torch.zeros_like(q), workspace=ws) for c in (cache, want)]
    assert same_bits(*out) and out[0].any()
    cache.rows.resize_(2, n - 1, 2, 32)
    with pytest.raises(ValueError, match="do not fit"):
        vxl.kvq_write(desc, k, v, cache)
    cache.scales.resize_(2, n - 1, 2, 2)
    with pytest.raises(vxl.VxlError):                               # (fewer rows than the layout's tokens)
        vxl.bilevel_decode_kvq(gl, desc, q, cache, None, mask, n, torch.zeros_like(q), workspace=ws)


def test_caches_of_other_heads_are_refused():
    rng = np.random.default_rng(18)
    lay = wl.random_layout(rng, 10, 4, 20, 40)
    gl, n, desc = make_layout(lay), lay.n_tokens, vxl.make_desc(4, 2, 64, "bf16")
    cache = vxl.KvqCache(desc, "fp4", n)
    for hkv, d in ((1, 64), (4, 64), (2, 128)):
        other = vxl.KvqCache(vxl.make_desc(4, hkv, d, "f32"), "fp4", n)
        k = torch.zeros(2, n, 64, dtype=torch.bfloat16, device="cuda")
        mask, lens = torch.zeros(1, 4, dtype=torch.uint8, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
        q, mix = torch.zeros(1, 1, 4, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(2, 1, 2, n, 64, dtype=torch.bfloat16, device="cuda")
        ws = vxl.alloc_workspace(vxl.workspace_bytes(vxl.OP_DECODE_KVQ, gl, desc, 1, 1, n))
        for call in (lambda: vxl.kvq_write(desc, k, k, other), lambda: vxl.kvq_read(desc, other, k, torch.zeros_like(k)),
                     lambda: vxl.gather_bilevel_kvq(gl, desc, other, None, mask, mix[0], mix[1], lens),
                     lambda: vxl.gather_bilevel_kvq(gl, desc, cache, other, mask, mix[0], mix[1], lens),
                     lambda: vxl.bilevel_decode_kvq(gl, desc, q, other, None, mask, n, torch.zeros_like(q), workspace=ws),
                     lambda: vxl.bilevel_decode_kvq(gl, desc, q, cache, other, mask, n, torch.zeros_like(q), workspace=ws)):
            with pytest.raises(vxl.VxlError) as e:
                call()
            assert e.value.status == vxl.VXL_ERR_INVALID_ARG


def test_refusals_with_a_layout():
    rng = np.random.default_rng(16)
    lay = wl.random_layout(rng, 10, 4, 20, 40)
    cache, sparse, _, _ = prompt(rng, "bf16", 2, 64, "fp4", lay, True)
    other, _, _, _ = prompt(rng, "bf16", 2, 64, "fp8", lay, False)
    gl, desc, n = make_layout(lay), vxl.make_desc(4, 2, 64, "bf16"), lay.n_tokens
    short = vxl.KvqCache(desc, "fp4", n - 1)
    few = vxl.KvqCache(desc, "fp4", len(lay.sparse_idx) - 1)
    mask = torch.zeros(1, 4, dtype=torch.uint8, device="cuda")
    q = torch.zeros(1, 1, 4, 64, dtype=torch.bfloat16, device="cuda")
    kmix = torch.zeros(1, 2, n, 64, dtype=torch.bfloat16, device="cuda")
    vmix, out = torch.zeros_like(kmix), torch.full_like(q, 9.0)
    lens = torch.full((1,), 9, dtype=torch.int32, device="cuda")
    need = vxl.workspace_bytes(vxl.OP_DECODE_KVQ, gl, desc, 1, 1, n)
    ws = vxl.alloc_workspace(need)

    def refused(status, **kw):
        a = dict(cache=cache, sparse=sparse, mask=mask, kmix=kmix, vmix=vmix, lens=lens, q=q, out=out, ws=ws[:need], cap=n)
        a.update(kw)
        if not {"q", "out", "ws"} & set(kw):
            with pytest.raises(vxl.VxlError) as e:
                vxl.gather_bilevel_kvq(gl, desc, a["cache"], a["sparse"], a["mask"], a["kmix"][:, :, :a["cap"]].contiguous(), a["vmix"],
                                       a["lens"])
            assert e.value.status == status
        if not {"kmix", "vmix", "lens"} & set(kw):
            with pytest.raises(vxl.VxlError) as e:
                vxl.bilevel_decode_kvq(gl, desc, a["q"], a["cache"], a["sparse"], a["mask"], a["cap"], a["out"], None, a["lens"], a["ws"])
            assert e.value.status == status

    bad = vxl.VXL_ERR_INVALID_ARG
    refused(bad, cache=short)
    refused(bad, sparse=few)
    refused(bad, sparse=other)                                    # of another format
    refused(bad, mask=None)
    refused(bad, cap=gl.mixed_kv_capacity(0) - 1)
    refused(bad, lens=None)
    refused(bad, q=out)
    refused(vxl.VXL_ERR_WORKSPACE, ws=ws[:need - 1])
    refused(vxl.VXL_ERR_WORKSPACE, ws=None)
    torch.cuda.synchronize()
    assert (out == 9.0).all() and (lens == 9).all() and not kmix.any()
