"""Calls on rotary positions and growing sets that are refused, before anything is launched, by the binding or by the library."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2506_19225_amd import vxl

from test_binding_native import Like, streams  # noqa: F401  (the fixture: no device is asked for a stream)

BF, F32, I32, F64, U8 = torch.bfloat16, torch.float32, torch.int32, torch.float64, torch.uint8
B, T, HQ, HKV, D, CAP, OUT = 2, 3, 4, 2, 64, 20, 12
DESC = vxl.make_desc(HQ, HKV, D, "bf16", token_major=True)
SIZE = {BF: 2, F32: 4, I32: 4, F64: 8, U8: 1}
_next = [1 << 20]


class Typed(Like):
    """Answers like a device tensor with a type, each in memory of its own."""

    def __init__(self, shape, dtype, ptr=None):
        if ptr is None:
            ptr = _next[0]
            _next[0] += (int(np.prod(shape)) * SIZE[dtype] + 4095) // 4096 * 4096 + 4096
        super().__init__(shape, ptr)
        self.dtype = dtype

    def dim(self):
        return len(self.shape)


Q, K, V = Typed((B * T, HQ, D), BF), Typed((B * T, HKV, D), BF), Typed((B * T, HKV, D), BF)
QO, KO = Typed((B * T, HQ, D), BF), Typed((B * T, HKV, D), BF)
AT, QD, OD = Typed((B, T), I32), Typed((B, T, HQ, D), BF), Typed((B, T, HQ, D), BF)
KM, VM, LEN = Typed((B, HKV, CAP, D), BF), Typed((B, HKV, CAP, D), BF), Typed((B,), I32)
POS, W, W2, LSE = Typed((B, HKV, CAP), I32), Typed((B, HKV, CAP), F32), Typed((B, HKV, CAP), F32), Typed((B, T, HQ), F32)
NEW, KEPT = Typed((B,), I32), Typed((B,), I32)
K2, V2, P2, W3 = Typed((B, HKV, OUT, D), BF), Typed((B, HKV, OUT, D), BF), Typed((B, HKV, OUT), I32), Typed((B, HKV, OUT), F32)


def rotary(dim=D, **kw):
    return vxl.Rotary(Typed((dim // 2,), F64), **kw)


ROT, RULE = rotary(), vxl.ScoreRule(causal=True)


def rotate(desc=DESC, r=ROT, at=AT, q=Q, k=K, qo=QO, ko=KO):
    vxl.rotate(desc, r, at, q, k, qo, ko)


def append(desc=DESC, r=ROT, at=AT, q=Q, k=K, v=V, qd=QD, km=KM, vm=VM, n=LEN, pos=POS, w=W):
    vxl.mixed_append(desc, r, at, q, k, v, qd, km, vm, n, pos, w)


def attend(desc=DESC, rule=RULE, qd=QD, at=AT, km=KM, vm=VM, n=LEN, pos=POS, out=OD, lse=LSE, w=W, w2=W2, ws="enough"):
    if ws == "enough":
        ws = Typed((1 << 20,), U8)
    vxl.mixed_attend(desc, rule, qd, at, km, vm, n, pos, out, lse, w, w2, ws)


def evict(desc=DESC, km=KM, vm=VM, n=LEN, w=W, pos=POS, new=NEW, keep=OUT, first=1, recent=2, ko=K2, vo=V2, wo=W3, po=P2, kept=KEPT, ws="enough"):
    if ws == "enough":
        ws = Typed((1 << 20,), U8)
    vxl.mixed_evict(desc, km, vm, n, w, pos, new, keep, first, recent, ko, vo, wo, po, kept, ws)


def refused(call, **kw):
    with pytest.raises(vxl.VxlError) as e:
        call(**kw)
    return e.value.status


def at_ptr(x, more):
    return Typed(x.shape, x.dtype, x.ptr + more)


@pytest.fixture(autouse=True)
def launches(streams, monkeypatch):  # noqa: F811
    """Calls that pass all checks would launch: they end in a library whose launches fail without a device, never on one."""
    if torch.cuda.is_available():
        pytest.skip("made-up addresses are not for a device")


def test_good_calls_reach_the_device():
    for call in (rotate, append, attend, evict):
        assert refused(call) == vxl.VXL_ERR_HIP, call.__name__
    assert refused(append, r=None) == refused(append, pos=None, w=None) == vxl.VXL_ERR_HIP
    assert refused(append, qd=Typed(QD.shape, BF, Q.ptr)) == vxl.VXL_ERR_HIP                 # queries in place
    assert refused(rotate, qo=Q, ko=K) == refused(rotate, k=None, ko=None) == vxl.VXL_ERR_HIP
    assert refused(attend, rule=None, at=None, pos=None) == refused(attend, w=W2) == refused(attend, lse=None, w=None, w2=None) == vxl.VXL_ERR_HIP
    assert refused(evict, ko=KM, vo=VM, wo=W, po=POS, kept=LEN) == refused(evict, new=None, recent=0) == vxl.VXL_ERR_HIP


@pytest.mark.parametrize("call,tensors", [(rotate, "at q k qo ko"), (append, "at q k v qd km vm n pos w"), (attend, "qd at km vm n pos out lse w w2"),
                                          (evict, "km vm n w pos new ko vo wo po kept")])
def test_types_sizes_and_places_of_tensors(call, tensors):
    import inspect
    have = {k: p.default for k, p in inspect.signature(call).parameters.items()}
    for name in tensors.split():
        x = have[name]
        for other in (BF, F32, I32, torch.int64, torch.float16):
            if other != x.dtype:
                SIZE.setdefault(other, 8)
                with pytest.raises(ValueError, match="tensor expected"):
                    call(**{name: Typed(x.shape, other)})
        with pytest.raises(AssertionError, match="contiguous CUDA tensors"):
            call(**{name: torch.zeros(x.shape, dtype=x.dtype)})
        for bad in (5, True, b"\1", "text", DESC):
            with pytest.raises((TypeError, AttributeError)):
                call(**{name: bad})
        assert refused(call, **{name: at_ptr(x, 2)}) == vxl.VXL_ERR_INVALID_ARG, name          # (of 4 or 16 bytes)
        short = Typed(x.shape[:-1] + (x.shape[-1] - 1,) if len(x.shape) < 4 else x.shape[:1] + (1,) + x.shape[2:], x.dtype)
        if not (call is rotate and name == "at"):                                             # (fewer tokens are fine)
            with pytest.raises((vxl.VxlError, IndexError)) as e:
                call(**{name: short})
            assert not isinstance(e.value, vxl.VxlError) or e.value.status == vxl.VXL_ERR_INVALID_ARG, name
        if name not in ("pos", "w", "w2", "lse", "at", "new"):
            with pytest.raises((vxl.VxlError, AttributeError)) as e:
                call(**{name: None})
            assert not isinstance(e.value, vxl.VxlError) or e.value.status == vxl.VXL_ERR_INVALID_ARG, name


def test_what_is_no_rotary_or_rule():
    for bad in (RULE, 5, "text", DESC, Q, object()):
        with pytest.raises(TypeError):
            rotate(r=bad)
    for bad in (ROT, 5, "text", DESC, Q):
        with pytest.raises(TypeError):
            attend(rule=bad)
    for bad in (Typed((D // 2,), F32), Typed((2, 4), F64)):
        with pytest.raises(ValueError):
            vxl.Rotary(bad)
    with pytest.raises(AssertionError):
        vxl.Rotary(torch.zeros(8, dtype=F64))
    with pytest.raises(ValueError):
        vxl.ScoreRule(slopes=Typed((HQ,), BF))
    for bad in (dict(window=2 ** 31), dict(n_always=-2 ** 40), dict(window=1.5)):
        with pytest.raises(ValueError):
            vxl.ScoreRule(**bad)
    with pytest.raises(AttributeError):
        ROT.freqs = Typed((4,), F64)
    with pytest.raises(ValueError, match="slope per query head"):
        attend(rule=vxl.ScoreRule(slopes=Typed((HQ + 1,), F32)))
    assert refused(rotate, r=None) == vxl.VXL_ERR_INVALID_ARG
    for call in (rotate, append):
        for r in (rotary(D + 2), rotary(magnitude=float("nan")), rotary(magnitude=float("inf")), vxl.Rotary(Typed((0,), F64)),
                  vxl.Rotary(Typed((4,), F64, (1 << 30) + 4))):
            assert refused(call, r=r) == vxl.VXL_ERR_INVALID_ARG
    for kw in (dict(softcap=-1.0), dict(softcap=float("nan")), dict(softcap=float("inf")), dict(softcap=1e-45), dict(window=-1), dict(n_always=-1)):
        assert refused(attend, rule=vxl.ScoreRule(**kw)) == vxl.VXL_ERR_INVALID_ARG, kw


def test_positions_where_a_rule_needs_them():
    for rule in (vxl.ScoreRule(causal=True), vxl.ScoreRule(window=3), vxl.ScoreRule(slopes=Typed((HQ,), F32))):
        assert refused(attend, rule=rule, at=None, pos=None) == vxl.VXL_ERR_INVALID_ARG
    assert refused(attend, at=None) == refused(attend, pos=None) == vxl.VXL_ERR_INVALID_ARG
    assert refused(attend, w2=None) == vxl.VXL_ERR_INVALID_ARG
    assert refused(evict, new=None) == vxl.VXL_ERR_INVALID_ARG


def test_workspaces():
    for call, op, shape in ((attend, vxl.OP_MIXED_ATTEND, (B, T, CAP)), (evict, vxl.OP_MIXED_EVICT, (B, 0, CAP))):
        need = vxl.workspace_bytes(op, None, DESC, *shape)
        assert need > 0
        assert refused(call, ws=None) == refused(call, ws=Typed((need - 1,), U8)) == vxl.VXL_ERR_WORKSPACE
        assert refused(call, ws=Typed((need,), U8, (1 << 40) + 8)) == vxl.VXL_ERR_WORKSPACE
        assert refused(call, ws=Typed((need,), U8)) == vxl.VXL_ERR_HIP
        assert vxl.workspace_bytes(op, None, DESC, 0, 1, CAP) == vxl.workspace_bytes(op, None, DESC, 1, 1, 0) == 0
    assert vxl.workspace_bytes(vxl.OP_MIXED_ATTEND, None, DESC, 1, 0, CAP) == 0


def test_numbers():
    for kw in (dict(keep=-1), dict(first=-1), dict(recent=-1), dict(keep=OUT + 1), dict(keep=1 << 32), dict(first=1 << 33), dict(recent=-(1 << 32))):
        assert refused(evict, **kw) == vxl.VXL_ERR_INVALID_ARG, kw
    big = vxl.make_desc(1 << 17, 1 << 16, 64, "bf16")
    lib, p = vxl.lib(), C.c_void_p
    far = [p(i << 44) for i in range(1, 20)]
    st = lib.vxl_mixed_attend(C.byref(big), None, far[0], None, 1, 1, far[1], far[2], 1, far[3], None, far[4], None, None, None, far[5], 1 << 40, None)
    assert st == vxl.VXL_ERR_UNSUPPORTED
    st = lib.vxl_mixed_evict(C.byref(big), far[0], far[1], 1, far[2], far[3], far[4], None, 1, 1, 0, 0, far[5], far[6], 1, far[7], far[8], far[9], far[10],
                             1 << 40, None)
    assert st == vxl.VXL_ERR_UNSUPPORTED
    rule = vxl.RotaryArg(1 << 20, 64, 0, 1.0, 0)
    many = lambda n: lib.vxl_rotate(C.byref(DESC), C.byref(rule), far[0], n, far[1], far[2], far[3], far[4], None)  # noqa: E731
    assert many(-1) == vxl.VXL_ERR_INVALID_ARG and many(0) == vxl.VXL_OK
    one = vxl.make_desc(2, 1, 64, "f32")
    st = lib.vxl_mixed_append(C.byref(one), None, far[0], 1 << 15, 1 << 17, far[1], far[2], far[3], far[4], far[5], far[6], 1, far[7], None, None, None)
    assert st == vxl.VXL_ERR_UNSUPPORTED


def test_outputs_that_meet():
    step = 16
    assert refused(rotate, qo=at_ptr(Q, step)) == refused(rotate, ko=at_ptr(K, step)) == refused(rotate, qo=Typed(Q.shape, BF, K.ptr)) \
        == refused(rotate, ko=Typed(K.shape, BF, QO.ptr)) == refused(rotate, qo=Typed(Q.shape, BF, AT.ptr)) == vxl.VXL_ERR_INVALID_ARG
    for name, x in (("qd", K), ("qd", V), ("qd", KM), ("km", VM), ("km", Q), ("vm", V), ("pos", LEN), ("pos", W), ("w", AT), ("km", ROT.freqs), ("qd", at_ptr(Q, step))):
        was = dict(qd=QD, km=KM, vm=VM, pos=POS, w=W)[name]
        assert refused(append, **{name: Typed(was.shape, was.dtype, x.ptr)}) == vxl.VXL_ERR_INVALID_ARG, (name, hex(x.ptr))
    head_major = vxl.make_desc(HQ, HKV, D, "bf16")
    assert refused(append, desc=head_major, qd=Typed(QD.shape, BF, Q.ptr)) == vxl.VXL_ERR_INVALID_ARG
    for name, x in (("out", QD), ("out", KM), ("out", at_ptr(VM, step)), ("lse", OD), ("w2", at_ptr(W, step)), ("w2", POS), ("lse", AT), ("lse", LEN), ("w2", KM)):
        was = dict(out=OD, lse=LSE, w2=W2)[name]
        assert refused(attend, **{name: Typed(was.shape, was.dtype, x.ptr)}) == vxl.VXL_ERR_INVALID_ARG, name
    for x in (QD, KM, VM, AT, POS, LEN, W, W2, OD, LSE):
        assert refused(attend, ws=Typed((1 << 20,), U8, x.ptr)) == vxl.VXL_ERR_INVALID_ARG
    for name, x in (("ko", KM), ("ko", V2), ("vo", at_ptr(VM, step)), ("wo", W), ("po", POS), ("kept", NEW), ("kept", P2), ("wo", KM)):
        was = dict(ko=K2, vo=V2, wo=W3, po=P2, kept=KEPT)[name]
        assert refused(evict, **{name: Typed(was.shape, was.dtype, x.ptr)}) == vxl.VXL_ERR_INVALID_ARG, name
    for kw in (dict(vo=V2), dict(wo=W3), dict(po=P2)):                        # in place: all four, of one capacity
        full = dict(vo=Typed(VM.shape, BF), wo=Typed(W.shape, F32), po=Typed(POS.shape, I32))
        assert refused(evict, **{**dict(ko=KM, vo=VM, wo=W, po=POS), **{k: full[k] for k in kw}}) == vxl.VXL_ERR_INVALID_ARG
    for x in (KM, VM, W, POS, LEN, NEW, K2, V2, W3, P2, KEPT):
        assert refused(evict, ws=Typed((1 << 20,), U8, x.ptr)) == vxl.VXL_ERR_INVALID_ARG


def test_rows_between_rows_do_not_meet():
    """Queries and keys of a fused projection side by side: in place, with rows of one between rows of the other."""
    base, row = 1 << 35, (HQ + 2 * HKV) * D
    desc = vxl.make_desc(HQ, HKV, D, "bf16")
    desc.q_stride_head = desc.kv_stride_head = D
    desc.q_stride_tok = desc.kv_stride_tok = row
    arg = vxl.RotaryArg(1 << 20, 64, 0, 1.0, 0)
    q, k = base, base + HQ * D * 2
    call = lambda qo, ko: vxl.lib().vxl_rotate(C.byref(desc), C.byref(arg), 1 << 34, 9, q, k, qo, ko, None)  # noqa: E731
    assert call(q, k) == vxl.VXL_ERR_HIP
    assert call(q, k + HKV * D * 2) == vxl.VXL_ERR_HIP                        # keys to where the values are: no input of the call
    assert call(q, q + (HQ - 1) * D * 2) == call(k, k) == call(q, k + 16) == call(q + row * 2, k) == vxl.VXL_ERR_INVALID_ARG


def test_caps_that_are_refused():
    """What the kernels make of a cap has to be numbers: beside infinities, caps that are nothing beside the scale, or all."""
    for softcap in (1e-20, 1e20, 2.0 ** 101):
        assert refused(attend, rule=vxl.ScoreRule(softcap=softcap)) == vxl.VXL_ERR_INVALID_ARG, softcap
