"""The operators of a mixed KV set that grows with generation and is cut back, as cases that can be timed and compared.

A mixed set holds, per query of a batch and KV head, rows of keys and values (`len` of them, room for `cap`), and beside
them the position of every row's token and the attention weight that the row has received so far.

Kinds of work:
  rotate    rotary positions of a prompt's queries and keys, before its pre-filling
  append    new tokens as a projection writes them: queries and keys rotated, keys and values put behind the rows of the sets
  attend    the tokens' attention over the sets: scores capped by a tanh or biased by distance, rows visible by position;
            and the weight that every row receives, added to what it has
  evict     the rows of the largest weight kept (the first and the latest positions always) and moved together: a kept row
            below the new length stays in its place, those above fill the gaps in order
"""
import functools
import math
import types

import numpy as np
import torch

own = False

ELEM = {"bf16": 2, "f32": 4}
DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}

_DEFAULTS = dict(dtype="bf16", hq=28, hkv=4, d=128, batch=1)
_OF_KIND = {
    "rotate": dict(token_major=True, rotary=128, interleaved=False, scaling="none", far=0),
    "append": dict(token_major=True, rotary=128, interleaved=False, scaling="none", far=0, t=1),
    "attend": dict(t=1, softcap=0.0, causal=False, window=0, n_always=0, slopes=False, pos=True, weigh=True, lse=False),
    "evict": dict(n_first=0, n_recent=0),
}


def _case(name, kind, **kw):
    c = dict(_DEFAULTS, kind=kind, **dict(_OF_KIND[kind], **kw))
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # a small fp32 prompt, half of every head rotated, neighbouring elements as pairs
        _case("rotate_f32_tiny", "rotate", dtype="f32", hq=4, hkv=2, d=64, tokens=577, rotary=32, interleaved=True, token_major=False),
        # a prompt of 2,048 frames, frequencies stretched by parts for its length: the largest
        _case("rotate_131k", "rotate", tokens=131328, scaling="parts"),
        # a generated token: latency
        _case("append_token", "append", rows=4097, cap=4352, far=16640),
        # the questions of eight users, 64 tokens each
        _case("append_questions_batch8", "append", batch=8, t=64, rows=18240, cap=18432, far=164096, scaling="linear"),
        # a generated token over an evicted set of 4,096 rows: latency
        _case("attend_token_4k", "attend", rows=4097, cap=4352),
        # a generated token of eight queries over mixed sets of the longest prompt: memory
        _case("attend_tokens_18k_batch8", "attend", batch=8, rows=18177, cap=18432, causal=True, lse=True),
        # a question of 64 tokens, scores capped
        _case("attend_question_24k_capped", "attend", t=64, rows=23872, cap=24064, causal=True, softcap=50.0),
        # a few tokens of three queries of a small fp32 model, biased by distance
        _case("attend_f32_biased", "attend", dtype="f32", hq=4, hkv=2, d=64, batch=3, t=5, rows=705, cap=768, causal=True,
              slopes=True, lse=True),
        # 2,048 more tokens of a prompt, attending to what is left of 16k and to themselves: the most computation
        _case("attend_chunk_2k", "attend", t=2048, rows=18688, cap=18688, causal=True),
        # every 256 tokens a set of 2,304 rows is cut to 2,048: latency
        _case("evict_2k", "evict", rows=2304, cap=2304, keep=2048, n_first=4, n_recent=128),
        # eight ragged fp32 sets of another head count
        _case("evict_batch8_f32", "evict", dtype="f32", hq=14, hkv=2, d=64, batch=8, rows=7001, cap=7040, keep=1777, n_first=17),
        # the dense keys and values of a 131k prompt cut to 16k rows
        _case("evict_131k", "evict", rows=131328, cap=131328, keep=16384, n_first=256, n_recent=64),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Another prompt, batch, head count, rule and length of the ranges above."""
    listed_work = {}
    for x in listed():
        w = work(x)
        have = listed_work.get(x["kind"], (0, 0))
        listed_work[x["kind"]] = (max(have[0], w["bytes"]), max(have[1], w["flops"]))
    kind = rng.choice(["rotate", "append", "attend", "attend", "attend", "evict", "evict"])
    while True:
        hq, hkv, d = rng.choice([(28, 4, 128)] * 4 + [(14, 2, 128), (14, 2, 64), (8, 1, 128), (4, 4, 64), (16, 8, 128)])
        f32 = rng.random() < 0.2                              # fp32 is for small models
        kw = dict(hq=hq, hkv=hkv, d=d, dtype="f32" if f32 else "bf16")
        turned = dict(rotary=rng.choice([d, d, d, d // 2, 16, 48]), interleaved=rng.random() < 0.4,
                      scaling=rng.choice(["none", "linear", "parts"]), token_major=rng.random() < 0.7,
                      far=rng.choice([0, _log(rng, 100, 900000)]))
        if kind == "rotate":
            c = _case(None, kind, tokens=_log(rng, 1, 8000 if f32 else 131328), **turned, **kw)
        else:
            rows = _log(rng, 60, 3000 if f32 else 40000)
            kw.update(batch=rng.choice([1, 1, 1, 2, 3, 8]), cap=rows + rng.choice([0, 1, 17, 255]))
            t = min(rows, rng.choice([1, 1, 2, 4, _log(rng, 1, 128), _log(rng, 16, 64 if f32 else 2048)]))
            if kind == "append":
                c = _case(None, kind, rows=rows, t=t, **turned, **kw)
            elif kind == "attend":
                pos = rng.random() < 0.8
                c = _case(None, kind, rows=rows, t=t, softcap=rng.choice([0.0, 0.0, 15.0, 30.0, 50.0]), pos=pos,
                          causal=pos and rng.random() < 0.8, window=rng.choice([0, 0, 0, _log(rng, 16, 8 * rows)]) if pos else 0,
                          n_always=rng.choice([0, 0, 4, 64]) if pos else 0, slopes=pos and rng.random() < 0.25,
                          weigh=rng.random() < 0.8, lse=rng.random() < 0.4, **kw)
            else:
                if rng.random() < 0.2:                        # whole prompts
                    rows = _log(rng, 3000, 131328)
                    kw.update(batch=1, cap=rows)
                keep = _log(rng, 16, rows + 20)
                n_first = rng.choice([0, 4, 64])
                n_first = n_first if n_first <= keep else 0
                c = _case(None, kind, rows=rows, keep=keep, n_first=n_first,
                          n_recent=rng.choice([0, min(keep - n_first, _log(rng, 1, 200))]), **kw)
        w = work(c)
        if w["bytes"] <= listed_work[kind][0] and w["flops"] <= max(listed_work[kind][1], 1):
            return c
        if kind in ("rotate", "append") and w["bytes"] <= listed_work[kind][0]:
            return c


# ---- what a case fixes, whatever the seed --------------------------------------------------------
@functools.lru_cache(maxsize=64)
def _lens_of(batch, rows, t):
    """Rows of every query's set, the new ones among them: the first is the longest."""
    rng = np.random.default_rng([batch, rows, t])
    return np.concatenate([[rows], rng.integers(max(t, rows // 2), rows + 1, size=batch - 1)]).astype(np.int32)


def _lens(c):
    return _lens_of(c["batch"], c["rows"], c.get("t", 1))


@functools.lru_cache(maxsize=16)
def _positions_of(batch, hkv, rows, cap, t):
    """Positions of the rows int32 [B, Hkv, cap] and of the new tokens [B, T]: a head keeps rows of its own of a prompt four times
    as long, a part of them out of order as gaps are filled; then the new tokens."""
    rng = np.random.default_rng([batch, hkv, rows, t, 3])
    row_pos = np.full((batch, hkv, cap), -1, np.int32)
    q_pos = np.empty((batch, t), np.int32)
    for b, n in enumerate(_lens_of(batch, rows, t)):
        old, prompt = int(n) - t, 4 * int(n)
        q_pos[b] = prompt + np.arange(t)
        for g in range(hkv):
            p = np.sort(rng.choice(prompt, size=old, replace=False)).astype(np.int32)
            at = rng.choice(old, size=old // 4, replace=False)
            p[at] = p[rng.permutation(at)]
            row_pos[b, g, :old] = p
            row_pos[b, g, old:n] = q_pos[b]
    return row_pos, q_pos


def _positions(c):
    return _positions_of(c["batch"], c["hkv"], c["rows"], c["cap"], c.get("t", 1))


def _pairs(c):
    """(query token, row) pairs that see each other, over the batch and the KV heads."""
    total = 0
    row_pos, q_pos = _positions(c) if c["pos"] else (None, None)
    for b, n in enumerate(_lens(c)):
        if not c["pos"] or not (c["causal"] or c["window"]):
            total += c["hkv"] * c["t"] * int(n)
            continue
        for g in range(c["hkv"]):
            p = np.sort(row_pos[b, g, :n]).astype(np.int64)
            hi = np.searchsorted(p, q_pos[b], side="right") if c["causal"] else np.full(c["t"], n)
            lo = np.searchsorted(p, q_pos[b].astype(np.int64) - c["window"], side="right") if c["window"] else np.zeros(c["t"], np.int64)
            first = np.searchsorted(p, c["n_always"], side="left")
            total += int((np.maximum(hi, lo) - lo + np.minimum(first, lo) + np.maximum(first - np.maximum(hi, lo), 0)).sum())
    return total


def work(c):
    elem, hq, hkv, d = ELEM[c["dtype"]], c["hq"], c["hkv"], c["d"]
    if c["kind"] == "rotate":
        return {"bytes": 2 * c["tokens"] * (hq + hkv) * d * elem + 4 * c["tokens"], "flops": 3 * c["tokens"] * (hq + hkv) * c["rotary"]}
    if c["kind"] == "append":
        n = c["batch"] * c["t"]
        return {"bytes": n * (2 * (hq + 2 * hkv) * d * elem + 4 + 8 * hkv), "flops": 3 * n * (hq + hkv) * c["rotary"]}
    rows = int(_lens(c).sum())
    if c["kind"] == "attend":
        new = 2 * c["batch"] * c["t"] * hq * d * elem
        beside = (4 if c["pos"] else 0) + (8 if c["weigh"] else 0)
        return {"bytes": rows * hkv * (2 * d * elem + beside) + new, "flops": 4 * d * (hq // hkv) * _pairs(c)}
    kept = int(np.minimum(_lens(c), c["keep"]).sum())
    return {"bytes": hkv * (8 * rows + kept * (4 * d * elem + 8)), "flops": 0}


def _freqs(c):
    """Radians per position of every pair: float64 [rotary / 2]; stretched for long prompts, evenly or the slow ones only."""
    i = np.arange(c["rotary"] // 2, dtype=np.float64)
    f = 1e6 ** (-2 * i / c["rotary"])
    if c["scaling"] == "linear":
        return f / 8
    if c["scaling"] == "parts":
        turns = 32768 * f / (2 * math.pi)                     # (over the length before)
        mix = np.clip((turns - 1) / (32 - 1), 0, 1)
        return f / 4 * (1 - mix) + f * mix
    return f


def _magnitude(c):
    return 0.1 * math.log(4) + 1 if c["scaling"] == "parts" else 1.0


# ---- what a program holds before the call --------------------------------------------------------
def _rows_like(gen, lead, n, d, dtype):
    """Keys and values as a model has them: a few channels of the keys are much larger than the others."""
    k = torch.randn(*lead, n, d, generator=gen, device="cuda")
    gain = torch.exp(0.5 * torch.randn(*lead, 1, d, generator=gen, device="cuda"))
    return (k * gain).to(dtype), torch.randn(*lead, n, d, generator=gen, device="cuda").to(dtype)


def _inputs(c, seed):
    """What the passes of both sides start from, and nothing else."""
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    s = types.SimpleNamespace(c=c)
    dtype, b, hq, hkv, d = DTYPE[c["dtype"]], c["batch"], c["hq"], c["hkv"], c["d"]
    if c["kind"] in ("rotate", "append"):
        n = c["tokens"] if c["kind"] == "rotate" else b * c["t"]
        shape = (lambda h: (n, h, d)) if c["token_major"] else (lambda h: (h, n, d))
        s.q, s.k, s.v = (torch.randn(*shape(h), generator=gen, device="cuda").to(dtype) for h in (hq, hkv, hkv))
        s.freqs = torch.from_numpy(_freqs(c)).cuda()
        start = torch.randint(0, 100, (b, 1), generator=gen, device="cuda") + c["far"]
        s.positions = (start + torch.arange(n // b, device="cuda")).int()
    if c["kind"] == "rotate":
        s.positions = s.positions[0].contiguous()
        s.q_out, s.k_out = torch.empty_like(s.q), torch.empty_like(s.k)
        return s
    s.lens = torch.from_numpy(_lens(c)).cuda()
    if c["kind"] == "append":
        s.qd = torch.empty(b, c["t"], hq, d, dtype=dtype, device="cuda")
        s.kmix = torch.zeros(b, hkv, c["cap"], d, dtype=dtype, device="cuda")
        s.vmix = torch.zeros_like(s.kmix)
        s.row_pos = torch.full((b, hkv, c["cap"]), -1, dtype=torch.int32, device="cuda")
        s.row_weight = torch.ones(b, hkv, c["cap"], device="cuda")
        return s
    row_pos, q_pos = _positions(c)
    s.kmix, s.vmix = _rows_like(gen, (b, hkv), c["cap"], d, dtype)
    s.row_pos, s.q_pos = torch.from_numpy(row_pos).cuda(), torch.from_numpy(q_pos).cuda()
    # weights that earlier tokens left: most rows have little, some none
    s.weight = torch.exp(1.5 * torch.randn(b, hkv, c["cap"], generator=gen, device="cuda")) / 8
    s.weight[torch.rand(b, hkv, c["cap"], generator=gen, device="cuda") < 0.2] = 0
    s.weight_out = torch.zeros_like(s.weight)
    if c["kind"] == "attend":
        q = torch.randn(b, c["t"], hkv, hq // hkv, d, generator=gen, device="cuda")
        near = s.kmix[:, :, :1].float().transpose(1, 2)[:, :, :, None] / d ** 0.5     # (queries share a direction)
        s.qd = (q + near).reshape(b, c["t"], hq, d).to(dtype)
        s.slopes = 2.0 ** (-8 * (torch.arange(hq, device="cuda") + 1) / hq) if c["slopes"] else None
        s.out = torch.empty_like(s.qd)
        s.lse = torch.empty(b, c["t"], hq, device="cuda") if c["lse"] else None
        return s
    s.newest = s.q_pos[:, -1].contiguous()
    room = c["keep"] + 64                                     # (for the tokens to come)
    s.kout = torch.zeros(b, hkv, room, d, dtype=dtype, device="cuda")
    s.vout = torch.zeros_like(s.kout)
    s.weight_out = torch.zeros(b, hkv, room, device="cuda")
    s.pos_out = torch.full((b, hkv, room), -1, dtype=torch.int32, device="cuda")
    s.kept = torch.zeros(b, dtype=torch.int32, device="cuda")
    return s


def prepare(c, seed):
    s = _inputs(c, seed)
    if own:
        _prepare_own(s)
    return s


# ---- the plain form ------------------------------------------------------------------------------
def _rotated(c, x, positions, freqs):
    """x [N, H, D] at positions [N]."""
    angle = positions.double()[:, None] * freqs
    cos, sin = ((f(angle) * _magnitude(c)).float()[:, None] for f in (torch.cos, torch.sin))
    x = x.float()
    part, rest = x[..., :c["rotary"]], x[..., c["rotary"]:]
    a, b = (part[..., 0::2], part[..., 1::2]) if c["interleaved"] else part.chunk(2, -1)
    a, b = a * cos - b * sin, a * sin + b * cos
    part = torch.stack((a, b), -1).flatten(-2) if c["interleaved"] else torch.cat((a, b), -1)
    return torch.cat((part, rest), -1)


def _visible(c, q_pos, row_pos):
    """bool [B, Hkv, T, cap]"""
    p, q = row_pos[:, :, None].long(), q_pos[:, None, :, None].long()
    see = torch.ones_like(p >= q)
    if c["causal"]:
        see = see & (p <= q)
    if c["window"]:
        see = see & (q - p < c["window"])
    return (see | (p < c["n_always"])) & (p >= 0)


def run(s):
    c = s.c
    if own:
        return _run_own(s)
    dtype, b, hkv, d = DTYPE[c["dtype"]], c["batch"], c["hkv"], c["d"]
    if c["kind"] in ("rotate", "append"):
        q, k, v = (x if c["token_major"] else x.transpose(0, 1) for x in (s.q, s.k, s.v))
        at = s.positions.flatten()
        q, k = (_rotated(c, x, at, s.freqs).to(dtype) for x in (q, k))
    if c["kind"] == "rotate":
        return tuple((x if c["token_major"] else x.transpose(0, 1)).contiguous() for x in (q, k))
    there = torch.arange(c["cap"], device="cuda") < s.lens[:, None]
    if c["kind"] == "append":
        t = c["t"]
        rows = (s.lens[:, None] - t + torch.arange(t, device="cuda")).long()           # [B, T]
        which = torch.arange(b, device="cuda")[:, None].expand(b, t)
        for mix, x in ((s.kmix, k), (s.vmix, v)):
            mix[which, :, rows] = x.reshape(b, t, hkv, d)
        s.row_pos[which, :, rows] = s.positions[:, :, None].expand(b, t, hkv)
        s.row_weight[which, :, rows] = 0.0
        return q.reshape(b, t, c["hq"], d), s.kmix, s.vmix, s.row_pos, s.row_weight
    if c["kind"] == "attend":
        t, g = c["t"], c["hq"] // hkv
        q = s.qd.float().view(b, t, hkv, g, d).permute(0, 2, 3, 1, 4).reshape(b, hkv, g * t, d)
        x = torch.matmul(q, s.kmix.float().transpose(2, 3).contiguous()).view(b, hkv, g, t, -1) * d ** -0.5
        if c["softcap"]:
            x = c["softcap"] * torch.tanh(x / c["softcap"])
        if c["slopes"]:
            far = (s.q_pos[:, None, :, None].long() - s.row_pos[:, :, None].long()).abs().float()
            x = x - s.slopes.view(1, hkv, g, 1, 1) * far[:, :, None]
        see = there[:, None, None]
        if c["pos"]:
            see = see & _visible(c, s.q_pos, s.row_pos)
        x = torch.where(see[:, :, None], x, -math.inf)
        top = x.amax(-1, keepdim=True)
        top = torch.where(top == -math.inf, 0.0, top)
        p = torch.exp(x - top)
        total = p.sum(-1, keepdim=True)
        p = p / torch.where(total == 0, 1.0, total)
        o = torch.matmul(p.view(b, hkv, g * t, -1), s.vmix.float()).view(b, hkv, g, t, d)
        out = [o.permute(0, 3, 1, 2, 4).reshape(b, t, c["hq"], d).to(dtype)]
        if c["lse"]:
            out.append((top + torch.log(total))[..., 0].permute(0, 3, 1, 2).reshape(b, t, c["hq"]))
        if c["weigh"]:
            out.append(torch.where(there[:, None], s.weight + p.sum((2, 3)), 0.0))
        return tuple(out)
    there = there[:, None].expand(b, hkv, -1)
    held = ((s.row_pos < c["n_first"]) | (s.newest[:, None, None] - s.row_pos < c["n_recent"])) & there
    key = torch.where(there, torch.where(held, math.inf, s.weight), -math.inf)
    order = torch.sort(key, dim=-1, descending=True, stable=True).indices
    kept = torch.zeros_like(there).scatter_(2, order[:, :, :c["keep"]], True) & there
    n = s.lens.clamp(max=c["keep"])
    row = torch.arange(c["cap"], device="cuda")
    low = row < n[:, None, None]
    gap, mover = low & ~kept, kept & ~low
    movers = torch.sort(mover.to(torch.int8), dim=-1, descending=True, stable=True).indices        # (those first, in order)
    src = torch.where(gap, movers.gather(2, (gap.long().cumsum(2) - 1).clamp(min=0)), row)
    m = min(c["keep"], c["cap"])
    src, low = src[:, :, :m], low[:, :, :m].expand(b, hkv, m)
    for to, x, none in ((s.kout, s.kmix, 0.0), (s.vout, s.vmix, 0.0)):
        to[:, :, :m] = torch.where(low[..., None], x.gather(2, src[..., None].expand(b, hkv, m, d)), none)
    s.weight_out[:, :, :m] = torch.where(low, s.weight.gather(2, src), 0.0)
    s.pos_out[:, :, :m] = torch.where(low, s.row_pos.gather(2, src), -1)
    return s.kout, s.vout, s.weight_out, s.pos_out, n


# ---- the framework's operators -------------------------------------------------------------------
def _prepare_own(s):
    from paper_2506_19225_amd import vxl
    c = s.c
    s.vxl = vxl
    s.desc = vxl.make_desc(c["hq"], c["hkv"], c["d"], c["dtype"], token_major=c.get("token_major", False))
    if c["kind"] in ("rotate", "append"):
        s.rotary = vxl.Rotary(s.freqs, interleaved=c["interleaved"], magnitude=_magnitude(c))
    elif c["kind"] == "attend":
        s.rule = vxl.ScoreRule(softcap=c["softcap"], causal=c["causal"], window=c["window"], n_always=c["n_always"], slopes=s.slopes)
        s.ws = vxl.alloc_workspace(vxl.workspace_bytes(vxl.OP_MIXED_ATTEND, None, s.desc, c["batch"], c["t"], c["cap"]))
    else:
        s.ws = vxl.alloc_workspace(vxl.workspace_bytes(vxl.OP_MIXED_EVICT, None, s.desc, c["batch"], 0, c["cap"]))


def _run_own(s):
    c, vxl = s.c, s.vxl
    if c["kind"] == "rotate":
        vxl.rotate(s.desc, s.rotary, s.positions, s.q, s.k, s.q_out, s.k_out)
        return s.q_out, s.k_out
    if c["kind"] == "append":
        vxl.mixed_append(s.desc, s.rotary, s.positions, s.q, s.k, s.v, s.qd, s.kmix, s.vmix, s.lens, s.row_pos, s.row_weight)
        return s.qd, s.kmix, s.vmix, s.row_pos, s.row_weight
    if c["kind"] == "attend":
        vxl.mixed_attend(s.desc, s.rule, s.qd, s.q_pos if c["pos"] else None, s.kmix, s.vmix, s.lens, s.row_pos if c["pos"] else None,
                         s.out, s.lse, s.weight if c["weigh"] else None, s.weight_out if c["weigh"] else None, s.ws)
        return (s.out,) + ((s.lse,) if c["lse"] else ()) + ((s.weight_out,) if c["weigh"] else ())
    vxl.mixed_evict(s.desc, s.kmix, s.vmix, s.lens, s.weight, s.row_pos, s.newest, c["keep"], c["n_first"], c["n_recent"],
                    s.kout, s.vout, s.weight_out, s.pos_out, s.kept, workspace=s.ws)
    return s.kout, s.vout, s.weight_out, s.pos_out, s.kept


# ---- the definition in 64 bits -------------------------------------------------------------------
def _turned64(c, x, positions, freqs):
    """x [..., H, D] with positions [...], as complex numbers turned by their angle."""
    x = x.double()
    r = c["rotary"]
    pair = x[..., :r].unflatten(-1, (-1, 2)) if c["interleaved"] else x[..., :r].unflatten(-1, (2, -1)).transpose(-1, -2)
    turn = torch.polar(torch.full_like(freqs, _magnitude(c)), torch.zeros_like(freqs)) * torch.exp(1j * positions.double()[..., None] * freqs)
    pair = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * turn[..., None, :])
    pair = pair.flatten(-2) if c["interleaved"] else pair.transpose(-1, -2).flatten(-2)
    return torch.cat((pair, x[..., r:]), -1)


def exact(c, seed):
    s = _inputs(c, seed)
    b, hkv, d = c["batch"], c["hkv"], c["d"]
    if c["kind"] == "rotate":
        out = []
        for x in (s.q, s.k):
            y = _turned64(c, x if c["token_major"] else x.transpose(0, 1), s.positions, s.freqs)
            out.append(y if c["token_major"] else y.transpose(0, 1).contiguous())
        return tuple(out)
    if c["kind"] == "append":
        q, k, v = (x if c["token_major"] else x.transpose(0, 1) for x in (s.q, s.k, s.v))
        q, k, v = (x.reshape(b, c["t"], -1, d) for x in (q, k, v))
        q, k = _turned64(c, q, s.positions, s.freqs), _turned64(c, k, s.positions, s.freqs)
        kmix, vmix, row_pos, weight = s.kmix.double(), s.vmix.double(), s.row_pos.clone(), s.row_weight.double()
        for i, n in enumerate(_lens(c)):
            at = slice(int(n) - c["t"], int(n))
            kmix[i, :, at], vmix[i, :, at] = k[i].transpose(0, 1), v[i].transpose(0, 1)
            row_pos[i, :, at], weight[i, :, at] = s.positions[i], 0
        return q, kmix, vmix, row_pos, weight
    if c["kind"] == "attend":
        t, g = c["t"], c["hq"] // hkv
        o, lse, weight = (torch.zeros(x.shape, dtype=torch.float64, device="cuda") for x in (s.out, s.out[..., 0], s.weight))
        for i, n in enumerate(int(n) for n in _lens(c)):
            for h in range(c["hq"]):
                kv = h // g
                x = s.qd[i, :, h].double() @ s.kmix[i, kv, :n].double().T / math.sqrt(d)
                if c["softcap"]:
                    x = c["softcap"] * torch.tanh(x / c["softcap"])
                if c["pos"]:
                    back = s.q_pos[i].double()[:, None] - s.row_pos[i, kv, :n].double()
                    if c["slopes"]:
                        x = x - back.abs() * s.slopes[h].double()
                    hidden = torch.zeros_like(back, dtype=torch.bool)
                    if c["causal"]:
                        hidden |= back < 0
                    if c["window"]:
                        hidden |= back >= c["window"]
                    hidden &= s.row_pos[i, kv, :n] >= c["n_always"]
                    x = x.masked_fill(hidden, -math.inf)
                p = torch.nan_to_num(torch.softmax(x, 1), nan=0.0)
                o[i, :, h] = p @ s.vmix[i, kv, :n].double()
                lse[i, :, h] = torch.logsumexp(x, 1)
                weight[i, kv, :n] += p.sum(0)
            weight[i, :, :n] += s.weight[i, :, :n].double()
        return (o,) + ((lse,) if c["lse"] else ()) + ((weight,) if c["weigh"] else ())
    kout, vout, weight, pos = s.kout.double(), s.vout.double(), s.weight_out.double(), s.pos_out.clone()
    kept_len = np.minimum(_lens(c), c["keep"]).astype(np.int32)
    all_w, all_p, newest = s.weight.cpu().numpy(), s.row_pos.cpu().numpy(), s.newest.cpu().numpy()
    for i, n in enumerate(int(n) for n in _lens(c)):
        m = int(kept_len[i])
        for h in range(hkv):
            w, p = all_w[i, h, :n].astype(np.float64), all_p[i, h, :n]
            held = (p < c["n_first"]) | (int(newest[i]) - p < c["n_recent"])
            keep = np.zeros(n, bool)
            keep[np.lexsort((np.arange(n), -w, ~held))[:m]] = True
            src = np.arange(m)
            src[~keep[:m]] = m + np.nonzero(keep[m:])[0]
            at = torch.from_numpy(src).cuda()
            kout[i, h, :m], vout[i, h, :m] = s.kmix[i, h, at].double(), s.vmix[i, h, at].double()
            weight[i, h, :m], pos[i, h, :m] = s.weight[i, h, at].double(), s.row_pos[i, h, at]
    return kout, vout, weight, pos, torch.from_numpy(kept_len).cuda()
