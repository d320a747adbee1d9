"""A growing mixed set from its beginning: a prompt's keys rotated, gathered for every query, then tokens put behind, attended to and the
sets cut back, each step against the oracle run on what the step before it left."""
import numpy as np
import pytest
import torch

import oracle
from paper_2506_19225_amd import vxl, workloads as wl

from mixed_util import DTYPE, check_attend, i32, values
from test_gpu_mixed import frequencies, rotary_tol

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("pooled", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("t", [1, 4, 20])
def test_from_a_gather_to_an_eviction(t, dtype, pooled):
    rng = np.random.default_rng(t)
    hq, hkv, d, bsz, keep = 8, 2, 64, 3, 90
    lay = wl.random_layout(rng, 7, 6, 20, 45, allow_empty_kept=False)
    n, chunks = lay.n_tokens, lay.n_chunks
    desc, new = vxl.make_desc(hq, hkv, d, dtype), vxl.make_desc(hq, hkv, d, dtype, token_major=True)
    layout = vxl.Layout(lay.n_prefix, lay.chunk_bounds, lay.sparse_offsets, lay.sparse_idx)
    rotary = vxl.Rotary(torch.from_numpy(frequencies(d)).cuda())
    q0, k0, v0 = (values(rng, (h, n, d), dtype) for h in (hq, hkv, hkv))
    q, k, v = (vxl.to_device(x, dtype) for x in (q0, k0, v0))
    vxl.rotate(desc, rotary, i32(np.arange(n)), q, k, q, k)
    turned = oracle.rotate(k0, np.arange(n), frequencies(d))
    assert (np.abs(k.double().cpu().numpy() - turned) <= rotary_tol(k0, turned, frequencies(d), False, 1.0, dtype)).all()

    # what the gather reports, for the calls behind it: a row's token is its position, the same for every head; nothing received so far
    masks = (rng.random((bsz, chunks)) < 0.5).astype(np.uint8)
    masks[0], masks[1] = 0, 1
    cap = n + t + 3
    kmix, vmix = (torch.full((bsz, hkv, cap, d), float("nan"), dtype=DTYPE[dtype], device="cuda") for _ in range(2))
    lens, src = torch.empty(bsz, dtype=torch.int32, device="cuda"), torch.full((bsz, cap), -1, dtype=torch.int32, device="cuda")
    mask = torch.from_numpy(masks).cuda()
    if pooled:
        ksp, vsp = (torch.empty(hkv, int(lay.sparse_offsets[-1]), d, dtype=DTYPE[dtype], device="cuda") for _ in range(2))
        vxl.pool_sparse_kv(layout, desc, k, v, ksp, vsp)
        vxl.gather_bilevel_kv_pooled(layout, desc, k, v, ksp, vsp, mask, kmix, vmix, lens, src)
        at = torch.from_numpy(lay.sparse_idx).cuda()                         # (pooled rows have no token: the kept ones' places)
        src = torch.where(src < 0, at[(-1 - src).clamp(0, len(at) - 1).long()], src)
    else:
        vxl.gather_bilevel_kv(layout, desc, k, v, mask, kmix, vmix, lens, src)
        want = oracle.gather_bilevel(k.float().cpu().numpy(), v.float().cpu().numpy(), masks, lay.n_prefix, lay.chunk_bounds, lay.sparse_offsets,
                                     lay.sparse_idx, cap)
        assert np.array_equal(lens.cpu().numpy(), want[2]) and np.array_equal(src.cpu().numpy(), want[3])
    row_pos = src[:, None].expand(bsz, hkv, cap).contiguous()
    weight = torch.zeros(bsz, hkv, cap, device="cuda")

    before = lens.tolist()
    lens += t
    q0, k0, v0 = (values(rng, (bsz * t, h, d), dtype) for h in (hq, hkv, hkv))
    positions = n + np.arange(t, dtype=np.int32)[None].repeat(bsz, 0)
    qd = torch.empty(bsz, t, hq, d, dtype=DTYPE[dtype], device="cuda")
    vxl.mixed_append(new, rotary, i32(positions), *(vxl.to_device(x, dtype) for x in (q0, k0, v0)), qd, kmix, vmix, lens, row_pos, weight)
    turned = oracle.rotate(k0.reshape(bsz, t, hkv, d).transpose(0, 2, 1, 3), np.arange(n, n + t), frequencies(d))
    for b, m in enumerate(before):
        tol = rotary_tol(k0.reshape(bsz, t, hkv, d)[b].transpose(1, 0, 2), turned[b], frequencies(d), False, 1.0, dtype)
        assert (np.abs(kmix[b, :, m:m + t].double().cpu().numpy() - turned[b]) <= tol).all()
        assert np.array_equal(vmix[b, :, m:m + t].float().cpu().numpy(), v0.reshape(bsz, t, hkv, d)[b].transpose(1, 0, 2))
        assert np.array_equal(row_pos[b, :, m:m + t].cpu().numpy(), positions[b][None].repeat(hkv, 0))

    rule = dict(causal=True, window=120, n_always=7)
    out, lse = torch.empty_like(qd), torch.empty(bsz, t, hq, device="cuda")
    ws = vxl.alloc_workspace(vxl.workspace_bytes(vxl.OP_MIXED_ATTEND, None, new, bsz, t, cap))
    vxl.mixed_attend(new, vxl.ScoreRule(**rule), qd, i32(positions), kmix, vmix, lens, row_pos, out, lse, weight, weight, ws)
    host = [x.float().cpu().numpy() for x in (qd, kmix, vmix)]
    got = tuple(x.double().cpu().numpy() for x in (out, lse, weight))
    check_attend(got, *host, lens.tolist(), dtype, 0.0, positions, row_pos.cpu().numpy(), np.zeros((bsz, hkv, cap)), **rule)

    was, long = [x.clone() for x in (kmix, vmix, weight, row_pos)], lens.tolist()
    ws = vxl.alloc_workspace(vxl.workspace_bytes(vxl.OP_MIXED_EVICT, None, new, bsz, 0, cap))
    vxl.mixed_evict(new, kmix, vmix, lens, weight, row_pos, i32([n + t - 1] * bsz), keep, 7, t, kmix, vmix, weight, row_pos, lens, ws)
    assert lens.tolist() == [min(x, keep) for x in long] and max(long) > keep
    for b, m in enumerate(lens.tolist()):
        for g in range(hkv):
            src = oracle.evict_rows(long[b], was[2][b, g].cpu().numpy(), was[3][b, g].cpu().numpy(), n + t - 1, keep, 7, t)
            for x, y in zip((kmix, vmix, weight, row_pos), was):
                assert torch.equal(x[b, g, :m], y[b, g, torch.from_numpy(src).cuda()])
