"""Growing mixed sets on the device: every variant of a call on the same inputs, graphs and streams, large buffers."""
import numpy as np
import pytest
import torch

import oracle
from paper_2506_19225_amd import vxl

from mixed_util import DTYPE, attend, check_attend, check_evict, f32, i32, sets, values

pytestmark = pytest.mark.gpu

SLOPES = dict(causal=True, slopes=2.0 ** (-8 * (np.arange(8) + 1) / 8))


def spread_case(seed, hq, hkv, d, bsz, t, cap, lens, dtype):
    rng = np.random.default_rng(seed)
    k, v, pos = sets(rng, bsz, hkv, cap, d, dtype, lens)
    q_pos = np.stack([rng.integers(0, 3 * max(int(n), 1), t) for n in lens]).astype(np.int32)
    return values(rng, (bsz, t, hq, d), dtype), k, v, q_pos, pos, rng.random((bsz, hkv, cap)).astype(np.float32)


# ---- variants ------------------------------------------------------------------------------------
@pytest.mark.parametrize("rule", [dict(causal=True), dict(causal=True, window=70, n_always=9), dict(softcap=12.0, window=200), SLOPES])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("waves,n_split,n_part", [(4, 1, 1), (4, 3, 2), (8, 1, 3), (8, 4, 1), (4, 99, 99)])
def test_every_plan_of_many_rows(waves, n_split, n_part, d, rule):
    lens = [517, 64]
    qd, k, v, q_pos, pos, weight = spread_case(d + waves, 8, 2, d, 2, 75, 530, lens, "bf16")
    q_pos[1, 3:] = -1                                             # (blocks of rows that are padding)
    try:
        vxl.debug_mixed_force(waves, n_split, n_part)
        got = attend(qd, k, v, lens, "bf16", 0.0, q_pos, pos, weight, **rule)
    finally:
        vxl.debug_mixed_force()
    check_attend(got, qd, k, v, lens, "bf16", 0.0, q_pos, pos, weight, **rule)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("t", [1, 3, 40])
@pytest.mark.parametrize("n_split", [1, 2, 7])
def test_every_split(n_split, t, dtype):
    lens = [890, 130]
    qd, k, v, q_pos, pos, weight = spread_case(t, 8, 2, 128, 2, t, 900, lens, dtype)
    for rule in (dict(causal=True, window=300), SLOPES):
        try:
            vxl.debug_mixed_force(0, n_split, 0)
            got = attend(qd, k, v, lens, dtype, 0.0, q_pos, pos, weight, **rule)
        finally:
            vxl.debug_mixed_force()
        check_attend(got, qd, k, v, lens, dtype, 0.0, q_pos, pos, weight, **rule)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("t", [1, 21])
@pytest.mark.parametrize("d", [64, 128])
def test_row_by_row(d, t, dtype):
    lens = [140, 0, 77]
    qd, k, v, q_pos, pos, weight = spread_case(t + d, 8, 2, d, 3, t, 141, lens, dtype)
    for rule in (dict(causal=True, window=30, n_always=3, softcap=9.0), SLOPES):
        try:
            vxl.debug_force_simple(True)
            got = attend(qd, k, v, lens, dtype, 0.2, q_pos, pos, weight, **rule)
        finally:
            vxl.debug_force_simple(False)
        check_attend(got, qd, k, v, lens, dtype, 0.2, q_pos, pos, weight, **rule)


@pytest.mark.parametrize("heads", [(40, 1, 64), (33, 1, 128), (32, 1, 64), (7, 7, 128), (1, 1, 64)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_head_groups(heads, dtype):
    hq, hkv, d = heads
    qd, k, v, q_pos, pos, weight = spread_case(hq, hq, hkv, d, 2, 1, 700, [699, 12], dtype)
    got = attend(qd, k, v, [699, 12], dtype, 0.0, q_pos, pos, weight, causal=True)
    check_attend(got, qd, k, v, [699, 12], dtype, 0.0, q_pos, pos, weight, causal=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("t", [1, 50])
def test_what_a_window_leaves_out_does_not_matter(t, dtype):
    """NaN and infinities in rows that no token's window holds, on both sides of it, in every tile."""
    n = 640
    qd, k, v, _, pos, weight = spread_case(t, 8, 2, 64, 1, t, n, [n], dtype)
    pos[:] = np.arange(n) * 2
    q_pos = np.full((1, t), 700, np.int32)
    hidden = (pos > 700) | (pos <= 600)
    k[hidden], v[hidden] = np.nan, np.inf
    odd = np.zeros(n, bool)
    odd[301:350:3] = True                                         # (inside the window: empty rows)
    pos[:, :, odd], k[:, :, odd], v[:, :, odd] = -1, np.inf, np.nan
    rule = dict(causal=True, window=100)
    got = attend(qd, k, v, [n], dtype, 0.0, q_pos, pos, weight, **rule)
    assert np.isfinite(got[0]).all() and np.isfinite(got[1]).all() and np.isfinite(got[2]).all()
    check_attend(got, qd, k, v, [n], dtype, 0.0, q_pos, pos, weight, **rule)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("t", [1, 40])
@pytest.mark.parametrize("softcap", [1e-3, 0.25, 2.0, 300.0, 2e7])
def test_caps(softcap, t, dtype):
    """From a cap that all logits reach to one that none comes near (a logit of 40 is then off by 40^3 / (3 softcap^2) = 5e-11: the plain ones)."""
    lens = [300, 45]
    qd, k, v, q_pos, pos, weight = spread_case(t, 8, 2, 64, 2, t, 310, lens, dtype)
    k[0, :, 20] = 0.0                                              # (logits of exactly 0)
    got = attend(qd, k, v, lens, dtype, 0.0, q_pos, pos, weight, softcap=softcap, window=250)
    check_attend(got, qd, k, v, lens, dtype, 0.0, q_pos, pos, weight, softcap=softcap if softcap < 1e6 else 0.0, window=250)


@pytest.mark.parametrize("edge", [1024, 2048, 4096, 8192, 16384])
@pytest.mark.parametrize("more", [-1, 0, 1])
def test_eviction_at_the_borders_of_its_variants(edge, more):
    rng = np.random.default_rng(edge + more)
    cap = edge + more
    k, v, pos = sets(rng, 2, 1, cap, 64, "bf16", [cap, cap - 70])
    w = (rng.integers(0, 900, (2, 1, cap)) / 7).astype(np.float32)
    for keep in (cap // 2, cap - 1):
        check_evict(k, v, [cap, cap - 70], w, pos, np.array([3 * cap, 3 * cap]), keep, 3, 40, "bf16", out_cap=keep)
        check_evict(k, v, [cap, cap - 70], w, pos, np.array([3 * cap, 3 * cap]), keep, 3, 40, "bf16", in_place=True)


@pytest.mark.parametrize("cap", [500, 17000])
def test_eviction_that_overwrites_the_lengths_only(cap):
    """kept may be mix_len where the sets go elsewhere too."""
    rng = np.random.default_rng(cap)
    bsz, hkv, d, keep = 3, 2, 64, 200
    lens = [cap, 150, cap - 1]
    k, v, pos = sets(rng, bsz, hkv, cap, d, "bf16", lens)
    w = rng.random((bsz, hkv, cap)).astype(np.float32)
    desc = vxl.make_desc(hkv, hkv, d, "bf16")
    dk, dv, dw, dp, dl = vxl.to_device(k, "bf16"), vxl.to_device(v, "bf16"), f32(w), i32(pos), i32(lens)
    ko, vo = (torch.empty(bsz, hkv, keep, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    wo, po = torch.empty(bsz, hkv, keep, device="cuda"), torch.empty(bsz, hkv, keep, dtype=torch.int32, device="cuda")
    ws = vxl.alloc_workspace(vxl.workspace_bytes(vxl.OP_MIXED_EVICT, None, desc, bsz, 0, cap))
    vxl.mixed_evict(desc, dk, dv, dl, dw, dp, None, keep, 0, 0, ko, vo, wo, po, dl, ws)
    assert dl.tolist() == [keep, 150, keep]
    for b in range(bsz):
        for g in range(hkv):
            src = oracle.evict_rows(lens[b], w[b, g], pos[b, g], 0, keep, 0, 0)
            assert np.array_equal(po[b, g, :len(src)].cpu().numpy(), pos[b, g, src])
            assert torch.equal(ko[b, g, :len(src)], dk[b, g, torch.from_numpy(np.asarray(src)).cuda()])


def test_append_of_a_fused_projection():
    """Queries, keys and values of a token side by side: read where they are, the projection left as it was."""
    rng = np.random.default_rng(8)
    hq, hkv, d, bsz, t, cap = 6, 2, 64, 2, 3, 10
    wide = hq + 2 * hkv
    x = vxl.to_device(values(rng, (bsz * t, wide, d), "bf16"), "bf16")
    split = vxl.make_desc(hq, hkv, d, "bf16", token_major=True)
    fused = vxl.make_desc(hq, hkv, d, "bf16", token_major=True)
    fused.q_stride_tok = fused.kv_stride_tok = wide * d
    rotary = vxl.Rotary(torch.from_numpy(1e4 ** (-np.arange(d // 2) * 2.0 / d)).cuda())
    at, lens, before = i32(rng.integers(0, 9999, (bsz, t))), i32([7, 10]), x.clone()

    def run(desc, q, k, v):
        out = [torch.full(s, 5.0, dtype=torch.bfloat16, device="cuda") for s in ((bsz, t, hq, d), (bsz, hkv, cap, d), (bsz, hkv, cap, d))]
        import ctypes as C
        st = vxl.lib().vxl_mixed_append(C.byref(desc), C.byref(vxl.RotaryArg(rotary.freqs.data_ptr(), d, 0, 1.0, 0)), at.data_ptr(), bsz, t, q, k, v,
                                        *(o.data_ptr() for o in out), cap, lens.data_ptr(), None, None, vxl._stream(None))
        assert st == vxl.VXL_OK
        return out

    p, row = x.data_ptr(), d * 2
    got = run(fused, p, p + hq * row, p + (hq + hkv) * row)
    apart = [y.contiguous() for y in (x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:])]
    want = run(split, *(y.data_ptr() for y in apart))
    assert torch.equal(x, before) and all(torch.equal(a, b) for a, b in zip(got, want))


# ---- graphs and streams --------------------------------------------------------------------------
class Generation:
    """A set that grows by a token (or several) of every query, is attended to and cut back when full, in fixed buffers."""

    def __init__(self, seed, t=1, dtype="bf16", cap=200, hq=14, hkv=2, d=64, bsz=2):
        rng = np.random.default_rng(seed)
        self.t, self.desc = t, vxl.make_desc(hq, hkv, d, dtype, token_major=True)
        self.rotary = vxl.Rotary(torch.from_numpy(1e6 ** (-np.arange(d // 2) * 2.0 / d)).cuda())
        self.rule = vxl.ScoreRule(causal=True, softcap=25.0, window=150, n_always=4)
        self.q, self.k, self.v = (vxl.to_device(values(rng, (bsz * t, h, d), dtype), dtype) for h in (hq, hkv, hkv))
        k, v, pos = sets(rng, bsz, hkv, cap, d, dtype, [120] * bsz, prompt=120)
        self.kmix, self.vmix, self.pos = vxl.to_device(k, dtype), vxl.to_device(v, dtype), i32(pos)
        self.weight = f32(rng.random((bsz, hkv, cap)))
        self.lens, self.at = i32([120] * bsz), i32(np.arange(120, 120 + t)[None].repeat(bsz, 0))
        self.qd = torch.zeros(bsz, t, hq, d, dtype=DTYPE[dtype], device="cuda")
        self.out, self.lse = torch.zeros_like(self.qd), torch.zeros(bsz, t, hq, device="cuda")
        self.newest = i32([0] * bsz)
        self.keep = 120
        self.ws_a = vxl.alloc_workspace(vxl.workspace_bytes(vxl.OP_MIXED_ATTEND, None, self.desc, bsz, t, cap))
        self.ws_e = vxl.alloc_workspace(vxl.workspace_bytes(vxl.OP_MIXED_EVICT, None, self.desc, bsz, 0, cap))

    def step(self):
        self.lens.add_(self.t)
        vxl.mixed_append(self.desc, self.rotary, self.at, self.q, self.k, self.v, self.qd, self.kmix, self.vmix, self.lens, self.pos, self.weight)
        vxl.mixed_attend(self.desc, self.rule, self.qd, self.at, self.kmix, self.vmix, self.lens, self.pos, self.out, self.lse, self.weight,
                         self.weight, self.ws_a)
        self.newest.copy_(self.at[:, -1])
        vxl.mixed_evict(self.desc, self.kmix, self.vmix, self.lens, self.weight, self.pos, self.newest, self.keep, 4, 16, self.kmix, self.vmix,
                        self.weight, self.pos, self.lens, self.ws_e)
        self.at.add_(self.t)

    def state(self):
        """All that a step writes; what lies behind the lengths holds NaN."""
        n = int(self.lens[0])
        return [x.clone() for x in (self.qd, self.out, self.lse, self.kmix[:, :, :n], self.vmix[:, :, :n], self.weight[:, :, :n],
                                    self.pos[:, :, :n], self.lens, self.at)]


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("t,dtype,cap", [(1, "bf16", 200), (7, "bf16", 200), (3, "f32", 200), (9, "f32", 200), (1, "bf16", 2000), (2, "bf16", 17000)])
def test_a_replayed_step_is_the_eager_one(t, dtype, cap):
    eager, graphed = Generation(t, t, dtype, cap), Generation(t, t, dtype, cap)
    side = torch.cuda.Stream()
    warm = Generation(1, t, dtype, cap)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        warm.step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        graphed.step()
    for _ in range(5):
        graph.replay()
        eager.step()
        torch.cuda.synchronize()
        assert same(eager.state(), graphed.state())
        warm.step()                                               # (other work between the replays)
        graphed.ws_a.fill_(0xFF)
        graphed.ws_e.fill_(0xFF)                                  # (nothing is kept in a workspace from call to call)


def test_two_graphs_on_two_streams():
    """Each with buffers and a workspace of its own, replayed side by side."""
    both = [Generation(3, 1), Generation(4, 5)]
    eager = [Generation(3, 1), Generation(4, 5)]
    for g in (Generation(5, 1), Generation(6, 5)):
        g.step()
    torch.cuda.synchronize()
    graphs, streams = [], [torch.cuda.Stream() for _ in both]
    for g in both:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            g.step()
    for _ in range(4):
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
        for g in eager:
            g.step()
    torch.cuda.synchronize()
    assert all(same(a.state(), b.state()) for a, b in zip(both, eager))


def test_calls_take_the_stream_that_they_are_given():
    """On a stream that is not the current one, behind work of that stream."""
    want, got = Generation(9, 2), Generation(9, 2)
    want.step()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    late, right = torch.empty_like(got.k), got.k.clone()
    torch.cuda.synchronize()
    got.k = late
    with torch.cuda.stream(stream):
        got.lens.add_(2)
        got.newest.copy_(got.at[:, -1])
        torch.cuda._sleep(2_000_000)
        late.copy_(right)
    g = got
    vxl.mixed_append(g.desc, g.rotary, g.at, g.q, g.k, g.v, g.qd, g.kmix, g.vmix, g.lens, g.pos, g.weight, stream)
    vxl.mixed_attend(g.desc, g.rule, g.qd, g.at, g.kmix, g.vmix, g.lens, g.pos, g.out, g.lse, g.weight, g.weight, g.ws_a, stream)
    vxl.mixed_evict(g.desc, g.kmix, g.vmix, g.lens, g.weight, g.pos, g.newest, g.keep, 4, 16, g.kmix, g.vmix, g.weight, g.pos, g.lens, g.ws_e, stream)
    with torch.cuda.stream(stream):
        got.at.add_(2)
    torch.cuda.synchronize()
    assert same(want.state(), got.state())


# ---- large buffers -------------------------------------------------------------------------------
def test_offsets_past_32_bits():
    """Three sets of 2^23 rows of 256 bytes: the third lies 4 GiB behind the first, its elements 2^31.  Its last rows are appended,
    attended to and kept."""
    hq, hkv, d, cap, t = 6, 3, 128, 1 << 23, 2
    rng = np.random.default_rng(1)
    desc = vxl.make_desc(hq, hkv, d, "bf16", token_major=True)
    kmix, vmix = (torch.zeros(1, hkv, cap, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    pos = torch.arange(cap, dtype=torch.int32, device="cuda").expand(1, hkv, cap).contiguous()
    weight = torch.zeros(1, hkv, cap, device="cuda")
    seen = 40
    k, v = (values(rng, (1, hkv, seen, d), "bf16") for _ in range(2))
    kmix[:, :, -seen:], vmix[:, :, -seen:] = vxl.to_device(k, "bf16"), vxl.to_device(v, "bf16")
    q, kn, vn = (vxl.to_device(values(rng, (t, h, d), "bf16"), "bf16") for h in (hq, hkv, hkv))
    qd, out, lse = torch.empty(1, t, hq, d, dtype=torch.bfloat16, device="cuda"), torch.empty(1, t, hq, d, dtype=torch.bfloat16, device="cuda"), \
        torch.empty(1, t, hq, device="cuda")
    at, lens = i32([[cap - 2, cap - 1]]), i32([cap])
    vxl.mixed_append(desc, None, at, q, kn, vn, qd, kmix, vmix, lens, pos, weight)
    assert torch.equal(kmix[0, :, -2:], kn.transpose(0, 1)) and torch.equal(vmix[0, :, -2:], vn.transpose(0, 1))
    k[0, :, -2:], v[0, :, -2:] = kn.float().cpu().numpy().transpose(1, 0, 2), vn.float().cpu().numpy().transpose(1, 0, 2)
    for tokens in (1, t):                                          # (a few rows, and as many as the ring has)
        many = 1 if tokens == 1 else 20
        qs = qd[:, -tokens:].repeat(1, many, 1, 1).contiguous()
        qp = at[:, -tokens:].repeat(1, many).contiguous()
        o, l, w = torch.empty_like(qs), torch.empty(1, tokens * many, hq, device="cuda"), torch.full_like(weight, 3.0)
        ws = vxl.alloc_workspace(vxl.workspace_bytes(vxl.OP_MIXED_ATTEND, None, desc, 1, tokens * many, cap))
        vxl.mixed_attend(desc, vxl.ScoreRule(causal=True, window=30), qs, qp, kmix, vmix, lens, pos, o, l, weight, w, ws)
        got = o.double().cpu().numpy(), l.double().cpu().numpy(), w[:, :, -seen:].double().cpu().numpy()
        near = np.broadcast_to(np.arange(cap - seen, cap, dtype=np.int32), (1, hkv, seen))
        check_attend(got, qs.float().cpu().numpy(), k, v, [seen], "bf16", 0.0, qp.cpu().numpy(), near, np.zeros((1, hkv, seen), np.float32), causal=True,
                     window=30)
        assert (w[:, :, :-seen] == 0).all()
        del ws, w
    # distinct weights, so that what is kept is what a sort says
    for g in range(hkv):
        weight[0, g] = torch.randperm(cap, device="cuda").float()
    kmix.view(torch.int16)[..., 0] = pos.to(torch.int16)           # (a row's number in its first bytes)
    kmix.view(torch.int16)[..., 1] = (pos >> 16).to(torch.int16)
    keep = cap - 1000
    dropped = [torch.sort(weight[0, g]).indices[:1000] for g in range(hkv)]
    was = weight.clone()
    ws = vxl.alloc_workspace(vxl.workspace_bytes(vxl.OP_MIXED_EVICT, None, desc, 1, 0, cap))
    vxl.mixed_evict(desc, kmix, vmix, lens, weight, pos, None, keep, 0, 0, kmix, vmix, weight, pos, lens, ws)
    assert int(lens) == keep
    for g in range(hkv):
        stays = torch.ones(cap, dtype=torch.bool, device="cuda")
        stays[dropped[g]] = False
        src = torch.arange(keep, dtype=torch.int32, device="cuda")
        holes, movers = (~stays[:keep]).nonzero()[:, 0], stays[keep:].nonzero()[:, 0] + keep
        src[holes] = movers.int()
        assert torch.equal(pos[0, g, :keep], src) and torch.equal(weight[0, g, :keep], was[0, g, src.long()])
        marks = kmix[0, g, :keep].view(torch.int16)
        assert torch.equal(marks[:, 0], src.to(torch.int16)) and torch.equal(marks[:, 1], (src >> 16).to(torch.int16))
