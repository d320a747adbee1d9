"""The operators of the quantised KV cache, as cases that can be timed and compared.

A quantised cache holds keys and values in 8 bits (e4m3) or 4 bits (e2m1) with a power-of-two scale for every 32 values of
a row.  Of a block x with a = max|x| the scale is 2^e, e = floor(log2 a) - emax, one more where a / 2^floor(log2 a) is 1.75
or more (emax = 8 or 2; e is at least -110), and x / 2^e is rounded to the nearest code, ties to even.  In memory:
  rows    uint8 [Hkv, capacity, 2, D * bits / 8]   the key codes of a row, then its value codes (4 bits: the even one low)
  scales  uint8 [Hkv, capacity, 2, D / 32]         e + 127

Kinds of work:
  store     rows written into the cache and read back from it
  gather    the mixed KV set of every query from a quantised cache, ready for the decode of plain KVs
  decode    attention of the query tokens over the quantised rows in place; `map_ready`: a generated token, whose row map
            an earlier call of the same selection has left
"""
import functools
import math
import types

import numpy as np
import torch

own = False

ELEM = {"bf16": 2, "f32": 4}
DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}
BITS = {"fp8": 8, "fp4": 4}
MANT = {"fp8": 3, "fp4": 1}                # mantissa bits
LOW = {"fp8": -6, "fp4": 0}                # exponent of the smallest normal number
EMAX = {"fp8": 8, "fp4": 2}                # exponent of the largest
TOP = {"fp8": 126, "fp4": 7}               # code of the largest

_DEFAULTS = dict(dtype="bf16", fmt="fp4", hq=28, hkv=4, d=128, prefix=256, unit=1, keep=8, kept_random=False,
                 pooled=False, token_major=False, lse=False, batch=1, t=1, k=0, map_ready=False)


def _case(name, kind, **kw):
    c = dict(_DEFAULTS, kind=kind, **kw)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one more token of the prompt goes into the cache, as a projection writes it: latency
        _case("store_token_fp4", "store", rows=1, first=4097, capacity=16640, token_major=True),
        # a ragged chunk of a small fp32 model
        _case("store_chunk_f32_fp8", "store", dtype="f32", fmt="fp8", hq=4, hkv=2, d=64, rows=577, first=64, capacity=1000),
        # a prompt of 256 frames of 64 tokens after its pre-filling
        _case("store_16k_fp4", "store", rows=16640, first=0, capacity=16640, token_major=True),
        # 2,048 frames: the largest single call
        _case("store_131k_fp8", "store", fmt="fp8", rows=131328, first=0, capacity=131328),
        # the tiny fp32 prompt of the parity workloads with odd chunks
        _case("gather_f32_tiny", "gather", dtype="f32", hq=2, hkv=1, d=64, prefix=17, chunks=5, len_lo=61, len_hi=140, k=2),
        # a question on the 16k prompt, its eight most relevant chunks dense
        _case("gather_16k_fp4", "gather", chunks=64, len_lo=256, len_hi=256, k=8),
        # eight questions on a ragged prompt with pooled sparse rows
        _case("gather_66k_batch8_fp8", "gather", fmt="fp8", chunks=114, len_lo=128, len_hi=1024, unit=64, keep=0, pooled=True,
              batch=8, k=32),
        # a generated token on the 16k prompt: latency
        _case("token_16k_fp4", "decode", chunks=64, len_lo=256, len_hi=256, k=8, map_ready=True),
        # a generated token of the longest prompt, 10,240 frames in 640 chunks
        _case("token_164k_fp8", "decode", fmt="fp8", chunks=640, len_lo=256, len_hi=256, keep=16, k=32, map_ready=True),
        # a generated token of eight questions, every chunk dense
        _case("tokens_66k_batch8_fp4", "decode", chunks=114, len_lo=128, len_hi=1024, unit=64, keep=0, batch=8, k=114,
              map_ready=True),
        # a question of 64 tokens on the 131k prompt, the sparse rows pooled
        _case("question_131k_fp4", "decode", chunks=256, len_lo=512, len_hi=512, pooled=True, t=64, k=16, lse=True),
        # a question on the tiny fp32 prompt
        _case("question_f32_tiny", "decode", dtype="f32", fmt="fp8", hq=2, hkv=1, d=64, prefix=64, chunks=4, len_lo=128,
              len_hi=128, t=8, k=2, lse=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Another prompt, head count, question and format of the ranges above."""
    most = [work(c) for c in listed()]
    kind = rng.choice(["store", "store", "gather", "gather", "decode", "decode", "decode", "decode"])
    while True:
        hq, hkv, d = rng.choice([(28, 4, 128)] * 4 + [(14, 2, 128), (14, 2, 64), (8, 1, 128), (4, 4, 64), (16, 8, 128)])
        f32 = rng.random() < 0.2                              # fp32 is for small prompts
        kw = dict(hq=hq, hkv=hkv, d=d, dtype="f32" if f32 else "bf16", fmt=rng.choice(["fp4", "fp8"]))
        tokens = _log(rng, 200, 8000) if f32 else _log(rng, 600, 164000)
        if kind == "store":
            rows = _log(rng, 1, tokens)
            c = _case(None, kind, rows=rows, capacity=tokens, first=rng.randint(0, tokens - rows),
                      token_major=rng.random() < 0.5, **kw)
        else:
            mean = min(tokens, _log(rng, 64, 1024))
            chunks = max(1, round(tokens / mean))
            if rng.random() < 0.5:
                kw.update(chunks=chunks, len_lo=mean, len_hi=mean)
            else:
                kw.update(chunks=chunks, len_lo=max(1, mean // 2), len_hi=mean + mean // 2)
            kw.update(prefix=rng.choice([0, 17, 64, 256, 256, 300]), keep=rng.choice([0, 4, 8, 16, 32]),
                      kept_random=rng.random() < 0.5, pooled=rng.random() < 0.4, batch=rng.choice([1, 1, 1, 2, 3, 8]),
                      k=min(chunks, rng.choice([0, chunks] + [_log(rng, 1, 64)] * 4)))
            if kind == "decode":
                kw.update(t=rng.choice([1, 1, 1, 2, 4, _log(rng, 1, 128), _log(rng, 8, 128)]), lse=rng.random() < 0.4)
                kw.update(map_ready=kw["t"] <= 4 and rng.random() < 0.7)
            c = _case(None, kind, **kw)
        w = work(c)
        if (c.get("chunks", 1) <= 4096 and w["bytes"] <= max(m["bytes"] for m in most)
                and w["flops"] <= max(m["flops"] for m in most)):
            return c


# ---- prompts -----------------------------------------------------------------------------------
@functools.lru_cache(maxsize=64)
def _shape(prefix, chunks, lo, hi, unit, keep):
    """Chunk bounds and sparse counts of a prompt: a property of the case, not of the seed."""
    rng = np.random.default_rng([prefix, chunks, lo, hi, unit, keep])
    lens = np.full(chunks, lo, np.int64) if lo == hi else rng.integers(lo // unit, hi // unit + 1, size=chunks) * unit
    lens = np.maximum(lens, 1)
    ratio = np.full(chunks, keep, np.int64) if keep else rng.choice([4, 8, 32], size=chunks)
    counts = np.maximum(lens // ratio, 1)
    return (np.concatenate([[prefix], prefix + np.cumsum(lens)]).astype(np.int32),
            np.concatenate([[0], np.cumsum(counts)]).astype(np.int32))


def _shape_of(c):
    return _shape(c["prefix"], c["chunks"], c["len_lo"], c["len_hi"], c["unit"], c["keep"])


def _kept(c, bounds, soff, seed):
    """Token ids of the kept rows: strided from the chunk's start, or at random places."""
    lens, counts = np.diff(bounds), np.diff(soff)
    if not c["kept_random"]:
        m = np.arange(soff[-1]) - np.repeat(soff[:-1], counts)
        return (np.repeat(bounds[:-1], counts) + m * np.repeat(lens // counts, counts)).astype(np.int32)
    rng = np.random.default_rng([seed, 7])
    return np.concatenate([b + np.sort(rng.permutation(n)[:m]) for b, n, m in zip(bounds[:-1], lens, counts)]
                          ).astype(np.int32)


def _capacity(c):
    """Rows that a mixed set with k dense chunks has at most."""
    bounds, soff = _shape_of(c)
    extra = np.sort(np.diff(bounds) - np.diff(soff))[::-1]
    return int(c["prefix"] + soff[-1] + extra[:c["k"]].sum())


def _row_bytes(c):
    return 2 * (c["d"] * BITS[c["fmt"]] // 8 + c["d"] // 32)


def work(c):
    elem, hkv, d = ELEM[c["dtype"]], c["hkv"], c["d"]
    if c["kind"] == "store":                  # rows in, rows out, and the cache between them
        return {"bytes": hkv * c["rows"] * (4 * d * elem + _row_bytes(c)), "flops": 0}
    bounds, soff = _shape_of(c)
    mean = float(np.mean(np.diff(bounds) - np.diff(soff)))
    rows = c["batch"] * (c["prefix"] + int(soff[-1]) + c["k"] * mean)          # of all mixed sets
    read = min(rows, int(bounds[-1]) + (int(soff[-1]) if c["pooled"] else 0))  # (shared ones once)
    if c["kind"] == "gather":
        return {"bytes": int(hkv * (read * _row_bytes(c) + rows * 2 * d * elem) + 4 * rows), "flops": 0}
    q = 2 * c["batch"] * c["t"] * c["hq"] * d * elem
    return {"bytes": int(hkv * read * _row_bytes(c) + 4 * rows + q), "flops": int(4 * d * c["hq"] * c["t"] * rows)}


# ---- the format, in plain operations -------------------------------------------------------------
def _pow2(e):
    """2^e as float32, exactly, for int32 e of normal numbers."""
    return ((e + 127) << 23).view(torch.float32)


def _encode(x, fmt):
    """float [..., D] -> codes uint8 [..., D * bits / 8], scales uint8 [..., D / 32]."""
    b = x.float().unflatten(-1, (-1, 32))
    amax = b.abs().amax(-1)
    m, e = torch.frexp(amax)                                       # amax = m 2^e, m in [0.5, 1)
    e = e - 1 - EMAX[fmt] + (m >= 0.875).int()
    e = torch.where(amax == 0, -110, e.clamp(min=-110)).int()
    bad = ~(amax < 1.75 * 2.0 ** 127)
    e = torch.where(bad, 0, e)
    y = torch.where(bad[..., None], 0.0, b) * _pow2(-e)[..., None]
    a = y.abs()
    ex = (torch.frexp(a)[1] - 1).clamp(min=LOW[fmt]).int()
    ex = torch.where(a == 0, LOW[fmt], ex)
    k = torch.round(a * _pow2(MANT[fmt] - ex)).int()
    code = ((ex - LOW[fmt]) * (1 << MANT[fmt]) + k).clamp(max=TOP[fmt])
    code = (code | (torch.signbit(y).int() << (BITS[fmt] - 1))).flatten(-2)
    if fmt == "fp4":
        code = code[..., 0::2] | (code[..., 1::2] << 4)
    return code.to(torch.uint8), torch.where(bad, 255, e + 127).to(torch.uint8)


@functools.lru_cache(maxsize=None)
def _table(fmt):
    """The value of every code."""
    n, m = 1 << (BITS[fmt] - 1), MANT[fmt]
    v = [math.ldexp((i & ((1 << m) - 1)) + ((1 << m) if i >> m else 0), max(i >> m, 1) - 1 + LOW[fmt] - m) for i in range(n)]
    if fmt == "fp8":
        v[n - 1] = math.nan
    return torch.tensor(v + [-x for x in v], dtype=torch.float32, device="cuda")


def _decode(rows, scales, fmt):
    """Inverse of _encode: float32 [..., D]."""
    if fmt == "fp4":
        rows = torch.stack((rows & 15, rows >> 4), -1).flatten(-2)
    s = scales.int()
    scale = torch.where(s == 255, math.nan, _pow2(s - 127))
    return (_table(fmt)[rows.int()].unflatten(-1, (-1, 32)) * scale[..., None]).flatten(-2)


# ---- what a program holds before the call --------------------------------------------------------
def _rows_like(gen, hkv, n, d, dtype):
    """Keys and values as a model has them: a few channels of the keys are much larger than the others."""
    k = torch.randn(hkv, n, d, generator=gen, device="cuda")
    gain = torch.exp(0.5 * torch.randn(hkv, 1, d, generator=gen, device="cuda"))
    return (k * gain).to(dtype), torch.randn(hkv, n, d, generator=gen, device="cuda").to(dtype)


def _both(k, v, fmt):
    """Cache tensors of keys and values [Hkv, n, D]."""
    return tuple(t.contiguous() for t in _encode(torch.stack((k, v), 2), fmt))


def _inputs(c, seed):
    """What the passes of both sides start from, and nothing else."""
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    s = types.SimpleNamespace(c=c)
    dtype, hkv, d = DTYPE[c["dtype"]], c["hkv"], c["d"]
    if c["kind"] == "store":
        k, v = _rows_like(gen, hkv, c["rows"], d, dtype)
        s.k, s.v = (t.transpose(0, 1).contiguous() if c["token_major"] else t for t in (k, v))
        s.kvq = (torch.zeros(hkv, c["capacity"], 2, d * BITS[c["fmt"]] // 8, dtype=torch.uint8, device="cuda"),
                 torch.zeros(hkv, c["capacity"], 2, d // 32, dtype=torch.uint8, device="cuda"))
        return s
    bounds, soff = _shape_of(c)
    n, chunks, b = int(bounds[-1]), c["chunks"], c["batch"]
    s.bounds, s.soff, s.kept, s.cap = bounds, soff, _kept(c, bounds, soff, seed), _capacity(c)
    k, v = _rows_like(gen, hkv, n, d, torch.float32)
    # queries share a direction, and every chunk's keys carry some of it
    lean = torch.randn(hkv, 1, d, generator=gen, device="cuda")
    much = torch.randn(chunks, generator=gen, device="cuda") * 0.2
    lens = torch.from_numpy(np.diff(bounds).astype(np.int64)).cuda()
    k[:, c["prefix"]:] += lean * torch.repeat_interleave(much, lens, output_size=n - c["prefix"])[None, :, None]
    s.kvq = _both(k.to(dtype), v.to(dtype), c["fmt"])
    s.sparse = None
    if c["pooled"]:                           # (means of a chunk's groups; here of two of its rows)
        at = torch.from_numpy(s.kept.astype(np.int64)).cuda()
        s.sparse = _both((0.5 * (k[:, at] + k[:, (at + 1).clamp(max=n - 1)])).to(dtype),
                         (0.5 * (v[:, at] + v[:, (at + 1).clamp(max=n - 1)])).to(dtype), c["fmt"])
    order = torch.rand(b, chunks, generator=gen, device="cuda").argsort(1).argsort(1)
    s.mask = (order < c["k"]).to(torch.uint8)
    if c["kind"] == "decode":
        q = torch.randn(b, c["t"], hkv, c["hq"] // hkv, d, generator=gen, device="cuda") + lean[:, 0][:, None]
        s.q = q.reshape(b, c["t"], c["hq"], d).to(dtype)
    return s


def prepare(c, seed):
    s = _inputs(c, seed)
    if c["kind"] != "store":
        # rows that a mixed set can take, in its order: prefix, then per chunk its dense and its sparse ones
        bounds, soff = s.bounds.astype(np.int64), s.soff.astype(np.int64)
        lens, counts = np.diff(bounds), np.diff(soff)
        chunk = np.concatenate([np.repeat(np.arange(c["chunks"]), lens), np.repeat(np.arange(c["chunks"]), counts)])
        src = np.concatenate([np.arange(c["prefix"], bounds[-1]), -1 - np.arange(soff[-1]) if c["pooled"] else s.kept])
        kind = np.concatenate([np.ones(lens.sum(), np.int64), np.zeros(counts.sum(), np.int64)])
        at = np.argsort(chunk, kind="stable")
        pad = np.zeros(c["prefix"], np.int64)
        s.row_src = torch.from_numpy(np.concatenate([np.arange(c["prefix"]), src[at]]).astype(np.int32)).cuda()
        s.row_chunk = torch.from_numpy(np.concatenate([pad, chunk[at]])).cuda()
        s.row_kind = torch.from_numpy(np.concatenate([pad + 2, kind[at]])).cuda()
        if c["map_ready"]:
            s.map = _row_map(s)
    if own:
        _prepare_own(s)
    return s


# ---- the plain form ------------------------------------------------------------------------------
def _row_map(s):
    """Source row of every mixed row int32 [B, cap] (0 behind the last one) and the lengths."""
    dense = s.mask[:, s.row_chunk].long()
    take = (s.row_kind == 2) | (dense == s.row_kind)
    at = torch.where(take, take.long().cumsum(1) - 1, s.cap)
    src = torch.zeros(len(take), s.cap + 1, dtype=torch.int32, device="cuda")
    src.scatter_(1, at, s.row_src.expand(len(take), -1))
    return src[:, :s.cap].contiguous(), take.sum(1).int()


def _mixed(s, src):
    """Values of the mixed rows, float32 [B, Hkv, cap, D] of keys and of values."""
    rows, scales = s.kvq
    at = src.long()
    if s.sparse is not None:
        at = torch.where(at < 0, rows.shape[1] - 1 - at, at)
        rows, scales = torch.cat((rows, s.sparse[0]), 1), torch.cat((scales, s.sparse[1]), 1)
    kv = _decode(rows[:, at], scales[:, at], s.c["fmt"]).transpose(0, 1)
    return kv[..., 0, :], kv[..., 1, :]


def run(s):
    c = s.c
    if own:
        return _run_own(s)
    if c["kind"] == "store":
        span = slice(c["first"], c["first"] + c["rows"])
        k, v = (t.transpose(0, 1) if c["token_major"] else t for t in (s.k, s.v))
        for t, part in zip(s.kvq, _both(k, v, c["fmt"])):
            t[:, span] = part
        kv = _decode(s.kvq[0][:, span], s.kvq[1][:, span], c["fmt"]).to(s.k.dtype)
        return tuple((kv[:, :, i].transpose(0, 1) if c["token_major"] else kv[:, :, i]).contiguous() for i in (0, 1))
    src, length = s.map if c["map_ready"] else _row_map(s)
    k, v = _mixed(s, src)
    there = torch.arange(s.cap, device="cuda") < length[:, None]
    if c["kind"] == "gather":
        k, v = (torch.where(there[:, None, :, None], t, 0.0).to(DTYPE[c["dtype"]]) for t in (k, v))
        return k, v, length, torch.where(there, src, 0)
    b, t, g = c["batch"], c["t"], c["hq"] // c["hkv"]
    q = s.q.float().view(b, t, c["hkv"], g, c["d"]).transpose(1, 2).reshape(b, c["hkv"], t * g, c["d"])
    logits = torch.matmul(q, k.transpose(2, 3)) * c["d"] ** -0.5
    logits = torch.where(there[:, None, None], logits, -math.inf)
    top = logits.amax(-1, keepdim=True)
    p = torch.exp(logits - top)
    total = p.sum(-1, keepdim=True)
    back = lambda x: x.view(b, c["hkv"], t, g, -1).transpose(1, 2).reshape(b, t, c["hq"], -1)  # noqa: E731
    o = back(torch.matmul(p, v) / total).to(s.q.dtype)
    lse = back(top + torch.log(total))[..., 0]
    return (o, length) + ((lse,) if c["lse"] else ())


# ---- the framework's operators -------------------------------------------------------------------
def _prepare_own(s):
    from paper_2506_19225_amd import vxl
    c = s.c
    s.vxl = vxl
    s.desc = vxl.make_desc(c["hq"], c["hkv"], c["d"], c["dtype"], token_major=c["token_major"])
    s.cache = vxl.KvqCache(s.desc, c["fmt"], rows=s.kvq[0], scales=s.kvq[1])
    if c["kind"] == "store":
        s.k_back, s.v_back = torch.empty_like(s.k), torch.empty_like(s.v)
        return
    s.layout = vxl.Layout(c["prefix"], s.bounds, s.soff, s.kept)
    s.cache_sparse = vxl.KvqCache(s.desc, c["fmt"], rows=s.sparse[0], scales=s.sparse[1]) if s.sparse else None
    b = c["batch"]
    s.mix_len = torch.zeros(b, dtype=torch.int32, device="cuda")
    if c["kind"] == "gather":
        s.kmix = torch.zeros(b, c["hkv"], s.cap, c["d"], dtype=DTYPE[c["dtype"]], device="cuda")
        s.vmix = torch.zeros_like(s.kmix)
        s.src_idx = torch.zeros(b, s.cap, dtype=torch.int32, device="cuda")
        return
    s.out = torch.empty_like(s.q)
    s.lse = torch.empty(s.q.shape[:3], dtype=torch.float32, device="cuda") if c["lse"] else None
    s.ws = vxl.alloc_workspace(vxl.workspace_bytes(vxl.OP_DECODE_KVQ, s.layout, s.desc, b, c["t"], s.cap))
    if c["map_ready"]:                                     # the call before it has left the row map
        _decode_own(s, False)


def _decode_own(s, ready):
    s.vxl.bilevel_decode_kvq(s.layout, s.desc, s.q, s.cache, s.cache_sparse, s.mask, s.cap, s.out, s.lse, s.mix_len, s.ws,
                             map_ready=ready)


def _run_own(s):
    c = s.c
    if c["kind"] == "store":
        s.vxl.kvq_write(s.desc, s.k, s.v, s.cache, c["first"], c["rows"])
        s.vxl.kvq_read(s.desc, s.cache, s.k_back, s.v_back, c["first"], c["rows"])
        return s.k_back, s.v_back
    if c["kind"] == "gather":
        s.vxl.gather_bilevel_kvq(s.layout, s.desc, s.cache, s.cache_sparse, s.mask, s.kmix, s.vmix, s.mix_len, s.src_idx)
        return s.kmix, s.vmix, s.mix_len, s.src_idx
    _decode_own(s, c["map_ready"])
    return (s.out, s.mix_len) + ((s.lse,) if c["lse"] else ())


# ---- the definition in 64 bits -------------------------------------------------------------------
def _values64(fmt):
    """The numbers >= 0 of the element type, ascending, from its definition."""
    if fmt == "fp4":
        return torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device="cuda")
    sub = [m / 8 * 2.0 ** -6 for m in range(8)]
    return torch.tensor(sub + [(1 + m / 8) * 2.0 ** e for e in range(-6, 9) for m in range(8) if (e, m) != (8, 7)],
                        dtype=torch.float64, device="cuda")


def _two(e):
    """2^e in 64 bits for whole e, by its bits: the device's pow is off by a step for some."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _quantised64(x, fmt):
    """float64 [..., D]: every value replaced by the one that the cache holds for it."""
    grid = _values64(fmt)
    b = x.unflatten(-1, (-1, 32))
    peak = b.abs().amax(-1, keepdim=True)
    e = torch.floor(torch.log2(torch.where(peak > 0, peak, 1.0)))
    e = torch.where(_two(e) > peak, e - 1, torch.where(_two(e + 1) <= peak, e + 1, e))
    e = e - (8 if fmt == "fp8" else 2) + (peak / _two(e) >= 1.75).double()
    scale = _two(torch.where(peak > 0, e.clamp(min=-110), torch.full_like(e, -110)))
    y = (b / scale).abs().clamp(max=float(grid[-1]))
    above = torch.searchsorted(grid, y).clamp(min=1)               # grid[above - 1] < y <= grid[above]
    lo, hi = grid[above - 1], grid[above]
    up = (y - lo > hi - y) | ((y - lo == hi - y) & (above % 2 == 0))
    return (torch.copysign(torch.where(up, hi, lo), b) * scale).flatten(-2)


def _held64(rows, scales, fmt):
    """float64 values of the codes of a cache."""
    grid = _values64(fmt)
    if fmt == "fp4":
        rows = torch.stack((rows % 16, rows // 16), -1).flatten(-2)
    half = 1 << (7 if fmt == "fp8" else 3)
    code = rows.long()
    sign = torch.where(code >= half, -1.0, 1.0).double()
    v = grid[(code % half).clamp(max=len(grid) - 1)] * sign
    return (v.unflatten(-1, (-1, 32)) * _two(scales.long() - 127)[..., None]).flatten(-2)


def exact(c, seed):
    s = _inputs(c, seed)
    if c["kind"] == "store":
        # (head by head: 64 bits of all of them would not leave much of the memory)
        axis = 1 if c["token_major"] else 0
        return tuple(torch.stack([_quantised64(h.double(), c["fmt"]) for h in t.unbind(axis)], axis) for t in (s.k, s.v))
    mask, bounds, soff = s.mask.cpu().numpy(), s.bounds, s.soff
    outs = []
    for b in range(c["batch"]):
        ids = [np.arange(c["prefix"])]
        for j in range(c["chunks"]):
            if mask[b, j]:
                ids.append(np.arange(bounds[j], bounds[j + 1]))
            else:
                at = np.arange(soff[j], soff[j + 1])
                ids.append(-1 - at if c["pooled"] else s.kept[at])
        ids = np.concatenate(ids).astype(np.int64)
        at = torch.from_numpy(ids).cuda()
        rows, scales = (t[:, at.clamp(min=0)] for t in s.kvq)
        if c["pooled"]:
            lo = at < 0
            rows[:, lo], scales[:, lo] = s.sparse[0][:, -1 - at[lo]], s.sparse[1][:, -1 - at[lo]]
        if c["kind"] == "gather":
            kv = torch.zeros(c["hkv"], s.cap, 2, c["d"], dtype=torch.float64, device="cuda")
            kv[:, :len(ids)] = _held64(rows, scales, c["fmt"])
            src = torch.zeros(s.cap, dtype=torch.int32, device="cuda")
            src[:len(ids)] = at.int()
            outs.append((kv[:, :, 0], kv[:, :, 1], torch.tensor(len(ids), dtype=torch.int32, device="cuda"), src))
            continue
        g = c["hq"] // c["hkv"]
        o, lse = [], []
        for h in range(c["hkv"]):
            kv = _held64(rows[h], scales[h], c["fmt"])
            x = s.q[b, :, h * g:(h + 1) * g].double().reshape(-1, c["d"]) @ kv[:, 0].T / math.sqrt(c["d"])
            o.append((torch.softmax(x, 1) @ kv[:, 1]).view(c["t"], g, c["d"]))
            lse.append(torch.logsumexp(x, 1).view(c["t"], g))
        outs.append((torch.cat(o, 1), torch.tensor(len(ids), dtype=torch.int32, device="cuda"))
                    + ((torch.cat(lse, 1),) if c["lse"] else ()))
    return tuple(torch.stack(x) for x in zip(*outs))
